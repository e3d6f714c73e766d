// Log probabilities of given tokens, their ranks, the rows' entropies and top alternatives
// (taps_logprobs).
//
// With M the row's largest value, w_j = exp(x_j - M), Z = sum w_j and S = sum w_j (x_j - M):
// log p_j = x_j - M - ln Z and the entropy is ln Z - S / Z.  One workgroup a row, one pass: each
// thread keeps Z and S about a reference of its own, which moves only when a value exceeds it by
// 2^8; they are joined in 64 bits.  A weight is 2^t, t = fma(x, log2 e, c) with c = -(reference *
// log2 e) rounded: what the rounding and the constant's error add to every t of a thread is known
// and taken out in the join, so that a weight near the top is good to 2^-23.
//
// Top alternatives: the k-th largest of the threads' own maxima bounds the row's k-th value from
// below.  The few threads that reach it look again at the batch of loads that held their maximum
// (at all of them if a second batch reaches the bound), and what they find is ranked by counting.
// Rows with more than kCand values at the bound (ties), or without k values above kLow (masks),
// go value by value instead: the largest value not yet taken, then its places in index order.
//
// Bound: HBM; in bf16 the vector unit is close behind (about 12 of the 16 instructions an element
// that the memory's rate leaves).
#include <algorithm>
#include <cmath>

#include "common.h"

namespace taps {
namespace {

typedef uint32_t u32x4 __attribute__((ext_vector_type(4)));

constexpr float kLog2e = 1.4426950408889634f;
constexpr double kLog2eRest = 1.4426950408889634 - (double)kLog2e;
// Values below kLow count as kLow in the sums, NaN too: their weights are 0 all the same where the
// row's maximum is well above, and t stays finite (0 * inf).  Past 1e6 c's rounding reaches a
// unit of the exponent.  Rows whose maximum is not between are done again with care.
constexpr float kLow = -1e6f, kHigh = 1e6f;
constexpr int kCand = 512;   // candidates for the top alternatives

struct LogprobArgs {
  const unsigned char* x;
  int64_t row_bytes;
  int budget, vocab, top;
  const int32_t* n_nodes;
  const int32_t* tokens;
  float* logprob;
  float* entropy;
  int32_t* rank;
  int32_t* top_idx;
  float* top_lp;
};

template <typename T>
__device__ inline float value_at(const T* x, int i);
template <>
__device__ inline float value_at<uint16_t>(const uint16_t* x, int i) {
  return __uint_as_float((uint32_t)x[i] << 16);
}
template <>
__device__ inline float value_at<float>(const float* x, int i) { return x[i]; }

// element e of a 16-byte unit
template <typename T>
__device__ inline float unit_value(const u32x4& r, int e) {
  if constexpr (sizeof(T) == 2)
    return __uint_as_float((e & 1) ? r[e >> 1] & 0xFFFF0000u : r[e >> 1] << 16);
  else
    return __uint_as_float(r[e]);
}

// max(x, kLow), kLow for NaN
__device__ inline float lifted(float x) { return __builtin_amdgcn_fmed3f(x, kLow, INFINITY); }

// Row of `n` values: the first `head` lie before the first 16-byte boundary, then `units`
// whole 16-byte units, then `tail` values.
template <typename T>
struct Row {
  static constexpr int E = 16 / sizeof(T);
  const T* x;
  int n, head, units, tail;
  __device__ inline Row(const unsigned char* p, int vocab) {
    x = (const T*)p;
    n = vocab;
    head = min(n, (int)((0 - (uintptr_t)p & 15) / sizeof(T)));
    units = (n - head) / E;
    tail = n - head - units * E;
  }
  __device__ inline u32x4 unit(int u) const { return *(const u32x4*)(x + head + (size_t)u * E); }
  __device__ inline int index(int u, int e) const { return head + u * E + e; }
  // the values outside whole units, one per thread: thread i < head + tail
  __device__ inline int edge(int i) const { return i < head ? i : n - tail + (i - head); }
};

template <int NT>
__device__ inline double block_sum(double v, double* s) {
#pragma unroll
  for (int m = 32; m >= 1; m >>= 1) v += __shfl_xor(v, m);
  __syncthreads();
  if ((threadIdx.x & 63) == 0) s[threadIdx.x >> 6] = v;
  __syncthreads();
  double t = 0.0;
#pragma unroll
  for (int w = 0; w < NT / 64; ++w) t += s[w];
  return t;
}
__device__ inline float wave_max(float v) {
#pragma unroll
  for (int m = 32; m >= 1; m >>= 1) v = fmaxf(v, __shfl_xor(v, m));
  return v;
}

template <typename T, int NT>
__global__ __launch_bounds__(NT) void logprobs_kernel(const LogprobArgs A) {
  constexpr int E = Row<T>::E;
  constexpr int UN = 4;   // units per thread and batch
  constexpr int NW = NT / 64;
  __shared__ double s_sum[NW];
  __shared__ float s_max[NT];
  __shared__ float s_bound;
  __shared__ int s_int[NW];
  __shared__ int s_count;
  __shared__ uint64_t s_cand[kCand];

  const int tid = threadIdx.x, lane = tid & 63, wave = tid >> 6;
  const int64_t row = blockIdx.x;
  const int b = (int)(row / A.budget), i = (int)(row - (int64_t)b * A.budget);
  const int top = A.top;
  int32_t* const tidx = A.top_idx + (size_t)row * top;
  float* const tlp = A.top_lp + (size_t)row * top;
  if (A.n_nodes && i >= A.n_nodes[b]) {
    if (tid < top) tidx[tid] = -1, tlp[tid] = 0.f;
    if (tid == 0) A.logprob[row] = 0.f, A.entropy[row] = 0.f, A.rank[row] = -1;
    return;
  }
  const Row<T> R(A.x + (size_t)row * A.row_bytes, A.vocab);
  const int tok = A.tokens[row];
  const bool given = tok >= 0 && tok < A.vocab;
  const float xt = given ? value_at(R.x, tok) : 0.f;
  // values that come before the token: above it, or equal and of a lower index.  Units before
  // the token's compare with the next value below it.
  const bool plain = given && xt == xt && xt != -INFINITY;
  const float xt_below =
      xt == 0.f ? -1.4e-45f
                : __uint_as_float(__float_as_uint(xt) + (xt > 0.f ? 0xFFFFFFFFu : 1u));
  const int tok_unit = tok >= R.head ? (tok - R.head) / E : -1;   // (past the last: the tail's)

  // ---- one pass
  float Z = 0.f, S = 0.f, c = 0.f, ref = -INFINITY;
  float best = -INFINITY, rest = -INFINITY;   // largest lifted value; the largest of other batches
  int best_at = 0, before = 0;
  auto batch = [&](const float* x, int n, int at) __attribute__((always_inline)) {
    float mx = x[0];
#pragma unroll
    for (int e = 1; e < n; ++e) mx = fmaxf(mx, x[e]);
    if (__ballot(mx > ref + 5.5f)) {   // 5.5 log2 e: 2^8
      const bool upd = mx > ref + 5.5f;
      const float cn = -(mx * kLog2e);
      const float d = cn - c;
      const float a = __builtin_amdgcn_exp2f(d);
      if (upd) {
        S = ref == -INFINITY ? 0.f : a * fmaf(d, Z, S);
        Z = ref == -INFINITY ? 0.f : a * Z;
        c = cn;
        ref = mx;
      }
    }
    rest = fmaxf(rest, fminf(mx, best));
    if (mx > best) best = mx, best_at = at;
#pragma unroll
    for (int e = 0; e < n; ++e) {
      const float t = fmaf(x[e], kLog2e, c);
      const float w = __builtin_amdgcn_exp2f(t);
      Z += w;
      S = fmaf(w, t, S);
    }
  };
  {
    const int step = NT * UN;
    const int nb = (R.units + step - 1) / step;
    u32x4 cur[UN], nxt[UN];
    auto fetch = [&](int k, u32x4 (&r)[UN]) __attribute__((always_inline)) {
#pragma unroll
      for (int j = 0; j < UN; ++j) r[j] = R.unit(min(k * step + j * NT + tid, R.units - 1));
    };
    if (nb > 0) fetch(0, cur);
    for (int k = 0; k < nb; ++k) {
      if (k + 1 < nb) fetch(k + 1, nxt);
      float x[UN * E];
#pragma unroll
      for (int j = 0; j < UN; ++j) {
        const int u = k * step + j * NT + tid;
        const float thr = u < tok_unit ? xt_below : xt;
        const bool in = u < R.units;
#pragma unroll
        for (int e = 0; e < E; ++e) {
          const float v = in ? unit_value<T>(cur[j], e) : -INFINITY;
          before += v > thr;
          x[j * E + e] = lifted(v);
        }
      }
      if (k * step + tid < R.units) batch(x, UN * E, k);
#pragma unroll
      for (int j = 0; j < UN; ++j) cur[j] = nxt[j];
    }
    // (units past the row were lifted to kLow)
    if (tid < R.head + R.tail) {
      const int j = R.edge(tid);
      const float v = value_at(R.x, j);
      before += j < tok ? v >= xt : v > xt;
      const float x = lifted(v);
      batch(&x, 1, nb);
    }
    // ties in the token's own unit
    if (tid == 0 && given && tok_unit >= 0 && tok_unit < R.units)
      for (int j = R.index(tok_unit, 0); j < tok; ++j) before += value_at(R.x, j) == xt;
  }

  // ---- the row's maximum; the threads' maxima for the bound
  s_max[tid] = best;
  if (tid == 0) s_count = 0;
  __syncthreads();
  float M = -INFINITY;
#pragma unroll
  for (int w = 0; w < NW; ++w) M = fmaxf(M, s_max[w * 64 + lane]);
  M = wave_max(M);
  const bool special = !(M > kLow + 1000.f && M < kHigh);

  // ---- rank
  if (!plain && given) {   // -inf or NaN: again, by the definition
    const uint32_t kt = value_key(__float_as_uint(xt));
    before = 0;
    for (int j = tid; j < R.n; j += NT) {
      const uint32_t k = value_key(__float_as_uint(value_at(R.x, j)));
      before += k > kt || (k == kt && j < tok);
    }
  }
  for (int m = 32; m >= 1; m >>= 1) before += __shfl_xor(before, m);
  if (lane == 0) s_int[wave] = before;

  // ---- Z and S about M
  double Zd, Sd, Md = M;   // Sd in units of ln 2
  if (!special) {
    const double k = ref == -INFINITY ? 0.0 : -(double)c + (double)ref * kLog2eRest - Md * 1.4426950408889634;
    const double a = ref == -INFINITY ? 0.0 : exp2(k);
    Zd = block_sum<NT>(a * Z, s_sum);
    Sd = block_sum<NT>(a * ((double)S + k * Z), s_sum) * 0.6931471805599453;
  } else {
    // about kLow or below, or above kHigh: weights by the definition
    float m = -INFINITY;
    bool any = false;
    for (int j = tid; j < R.n; j += NT) {
      const float v = value_at(R.x, j);
      if (v == v) m = v > m ? v : m, any = true;
    }
    __syncthreads();
    s_max[tid] = m;
    const int have = __syncthreads_or(any);
    M = -INFINITY;
#pragma unroll
    for (int w = 0; w < NW; ++w) M = fmaxf(M, s_max[w * 64 + lane]);
    M = wave_max(M);
    Md = M;
    double z = 0.0, s = 0.0;
    for (int j = tid; have && j < R.n; j += NT) {
      const float v = value_at(R.x, j);
      if (v == M) {
        z += 1.0;
      } else if (v == v) {
        const double d = (double)v - Md, w = exp(d);
        z += w;
        if (w > 0.0) s += w * d;
      }
    }
    Zd = block_sum<NT>(z, s_sum);
    Sd = block_sum<NT>(s, s_sum);
  }
  const double lnz = log(Zd);
  auto lp = [&](float v) {
    if (v != v || Zd == 0.0) return -INFINITY;
    return v == M ? (float)-lnz : (float)(((double)v - Md) - lnz);
  };
  if (tid == 0) {
    int r = 0;
#pragma unroll
    for (int w = 0; w < NW; ++w) r += s_int[w];
    A.rank[row] = given ? r : -1;
    A.logprob[row] = given ? lp(xt) : -INFINITY;
    A.entropy[row] = Zd == 0.0 ? 0.f : (float)(lnz - Sd / Zd);
  }
  if (top == 0) return;

  // ---- top alternatives: the bound, by the first wave
  bool fallback = special;
  if (!special) {
    if (wave == 0) {
      float v[NW];
#pragma unroll
      for (int w = 0; w < NW; ++w) v[w] = s_max[w * 64 + lane];
      float bound = 0.f;
      for (int r = 0; r < top; ++r) {
        float m = v[0];
#pragma unroll
        for (int w = 1; w < NW; ++w) m = fmaxf(m, v[w]);
        bound = wave_max(m);
        const uint64_t who = __ballot(m == bound);
        if (lane == __ffsll((long long)who) - 1) {   // one of the equal ones goes
          bool gone = false;
#pragma unroll
          for (int w = 0; w < NW; ++w) {
            const bool hit = !gone && v[w] == bound;
            v[w] = hit ? -INFINITY : v[w];
            gone = gone || hit;
          }
        }
      }
      if (lane == 0) s_bound = bound;
    }
    __syncthreads();
    const float bound = s_bound;
    fallback = !(bound > kLow);
    if (!fallback) {
      auto add = [&](float v, int j) {
        if (v >= bound) {
          const int at = atomicAdd(&s_count, 1);
          if (at < kCand) s_cand[at] = cand_key(value_key(__float_as_uint(v)), (uint32_t)j);
        }
      };
      if (best >= bound) {
        const int step = NT * UN, nb = (R.units + step - 1) / step;
        const bool all = rest >= bound;
        for (int k = all ? 0 : best_at; k < (all ? nb : min(best_at + 1, nb)); ++k) {
#pragma unroll
          for (int j = 0; j < UN; ++j) {
            const int u = k * step + j * NT + tid;
            if (u < R.units) {
              const u32x4 r = R.unit(u);
#pragma unroll
              for (int e = 0; e < E; ++e) add(unit_value<T>(r, e), R.index(u, e));
            }
          }
        }
        if (tid < R.head + R.tail) add(value_at(R.x, R.edge(tid)), R.edge(tid));
      }
      __syncthreads();
      const int n = s_count;
      fallback = n > kCand;
      if (!fallback) {
        for (int q = tid; q < n; q += NT) {
          const uint64_t mine = s_cand[q];
          int r = 0;
          for (int j = 0; j < n; ++j) r += s_cand[j] > mine;
          if (r < top) {
            const int j = (int)cand_index(mine);
            tidx[r] = j;
            tlp[r] = lp(value_at(R.x, j));
          }
        }
      }
    }
  }
  if (!fallback) return;

  // ---- value by value: the largest key below the last one, then its indices in order
  uint64_t last = 1ull << 32;   // above every value's key
  for (int have = 0; have < top;) {
    uint32_t m = 0;
    bool any = false;
    for (int j = tid; j < R.n; j += NT) {
      const uint32_t k = value_key(__float_as_uint(value_at(R.x, j)));
      if (k < last) m = max(m, k), any = true;
    }
#pragma unroll
    for (int o = 32; o >= 1; o >>= 1) m = max(m, (uint32_t)__shfl_xor((int)m, o));
    __syncthreads();
    if (lane == 0) s_int[wave] = (int)m;
    if (!__syncthreads_or(any)) break;   // (top <= vocab: never)
    m = 0;
#pragma unroll
    for (int w = 0; w < NW; ++w) m = max(m, (uint32_t)s_int[w]);
    for (int j0 = 0; j0 < R.n && have < top; j0 += NT) {
      const int j = j0 + tid;
      const float v = j < R.n ? value_at(R.x, j) : 0.f;
      const bool hit = j < R.n && value_key(__float_as_uint(v)) == m;
      const uint64_t mask = __ballot(hit);
      __syncthreads();
      if (lane == 0) s_int[wave] = __popcll(mask);
      __syncthreads();
      int at = have, total = 0;
#pragma unroll
      for (int w = 0; w < NW; ++w) {
        if (w < wave) at += s_int[w];
        total += s_int[w];
      }
      at += __popcll(mask & ((1ull << lane) - 1));
      if (hit && at < top) tidx[at] = j, tlp[at] = lp(v);
      have += total;
    }
    last = m;
  }
}

}  // namespace

hipError_t launch_logprobs(const void* logits, int64_t row_bytes, int batch, int budget,
                           int vocab, int dtype, const int32_t* n_nodes, const int32_t* tokens,
                           int top, float* logprob, float* entropy, int32_t* rank,
                           int32_t* top_idx, float* top_logprob, hipStream_t s) {
  const int64_t rows = (int64_t)batch * budget;
  if (rows <= 0) return hipSuccess;
  LogprobArgs A;
  A.x = (const unsigned char*)logits, A.row_bytes = row_bytes;
  A.budget = budget, A.vocab = vocab, A.top = top, A.n_nodes = n_nodes, A.tokens = tokens;
  A.logprob = logprob, A.entropy = entropy, A.rank = rank, A.top_idx = top_idx, A.top_lp = top_logprob;
  const unsigned grid = (unsigned)rows;
  if (dtype == TAPS_BF16) logprobs_kernel<uint16_t, 512><<<grid, 512, 0, s>>>(A);
  else logprobs_kernel<float, 512><<<grid, 512, 0, s>>>(A);
  return hipGetLastError();
}

}  // namespace taps

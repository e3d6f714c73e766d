// Log probabilities of given tokens, their ranks, the rows' entropies and top alternatives
// (taps_logprobs).
//
// With M the row's largest value, w_j = exp(x_j - M), Z = sum w_j and S = sum w_j (x_j - M): log
// p_j = x_j - M - ln Z and the entropy is ln Z - S / Z.  One pass by one workgroup a row, or, of
// few rows, one for each of a row's parts, which a second kernel joins: each thread keeps Z and S
// about a reference of its own, which moves only when a value exceeds it by 2^8; they are joined in
// 64 bits.  A weight is 2^t, t = fma(x, log2 e, c) with c = -(reference * log2 e) rounded: what the
// rounding and the constant's error add to every t of a thread is known and taken out in the join,
// so that a weight near the top is good to 2^-23.  The largest value's own weight is 1 without a
// rounding: a thread that holds it takes what it added for it out again.  So Z >= 1, no log
// probability is above 0, and a row of which a mask leaves one value gives exactly 0.
//
// The pass takes values as they are.  An infinity or NaN makes S one too: a wave that ends with
// such a sum goes over its values again with those below kLow, and NaN, lifted to kLow (a wave
// that meets one in its first loads does so at once), and rows whose maximum is not an ordinary
// number are summed by the definition.
//
// Top alternatives: the k-th largest of 64 groups' maxima (of 256 from 49 alternatives on: the
// smallest of 64 groups' maxima leaves hundreds; 48 take 20.5 us for 23.5) bounds the row's k-th
// value from below.  The few threads that reach it look again at the batch of loads that held their
// maximum (at all of them if a second batch reaches the bound), and what they find is ranked by
// counting.  More than kCand values at the bound raise it: to the k-th of those kept, or past it
// where it occurs too often.  Places that are left (ties, masked values) go value by value: the
// largest value not yet taken, then its places in index order.  Rows whose maximum is not an
// ordinary number have no such bound and find all their alternatives so, a scan of the row for each
// distinct value: 64 fp32 rows of 151,936 205 us with 5 alternatives, 2070 with 64 (ordinary ones
// 19.5 and 27).
//
// Bound: HBM; in bf16 the vector unit is close behind (7.7 instructions an element, one of them the
// exponential).  2048 rows of 151,936 in bf16 (622 MB) take 121 us, 5.1 TB/s; 64 of them, in four
// parts each, 16 us with the join's 4 and two launches.
#include <algorithm>
#include <cmath>

#include "common.h"

namespace taps {
namespace {

typedef uint32_t u32x4 __attribute__((ext_vector_type(4)));

constexpr float kLog2e = 1.4426950408889634f;
constexpr double kLog2eRest = 1.4426950408889634 - (double)kLog2e;
// Values below kLow count as kLow in the careful sums, NaN too: their weights are 0 all the same
// where the row's maximum is well above, and t stays finite (0 * inf).  Past 1e6 c's rounding
// reaches a unit of the exponent.  Rows whose maximum is not between go by the definition.
constexpr float kLow = -1e6f, kHigh = 1e6f;
constexpr int kThreads = 512, kUnits = 4;   // 16-byte units per thread in a batch of loads
constexpr int kCand = kThreads;             // candidates for the top alternatives
constexpr int kFewTop = 48;                 // up to here 64 groups' maxima bound them well

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
  // parts > 1: what each part of a row leaves, [rows][parts] and [rows][parts][top]
  int parts;
  struct Part* part;
  uint64_t* keys;
};

// Maximum of a part, its sums about it, the values before the token, the token's value
struct Part {
  double Z, S;
  float M;
  int before;
  float token;
  int given;
};

template <typename T>
__device__ inline float value_at(const T* x, int i);
template <>
__device__ inline float value_at<uint16_t>(const uint16_t* x, int i) {
  return __uint_as_float((uint32_t)x[i] << 16);
}
template <>
__device__ inline float value_at<float>(const float* x, int i) { return x[i]; }

template <bool B>
struct Flag {
  static constexpr bool value = B;
};

// element e of a 16-byte unit
template <typename T>
__device__ inline float unit_value(const u32x4& r, int e) {
  if constexpr (sizeof(T) == 2)
    return __uint_as_float((e & 1) ? r[e >> 1] & 0xFFFF0000u : r[e >> 1] << 16);
  else
    return __uint_as_float(r[e]);
}

// max(x, kLow), kLow for NaN
__device__ inline float lifted(float x) { return x > kLow ? x : kLow; }

// max by the bare instruction (fmaxf quiets its operands first, an instruction each); NaN operands
// give either operand or NaN
__device__ inline float max3(float a, float b, float c) {
  float r;
  asm("v_max3_f32 %0, %1, %2, %3" : "=v"(r) : "v"(a), "v"(b), "v"(c));
  return r;
}

// Row (or part of one) of `n` values: the first `head` lie before the first 16-byte boundary, then
// `units` whole 16-byte units, then `tail` values.
template <typename T>
struct Row {
  static constexpr int E = 16 / sizeof(T);
  const T* x;
  int n, head, units, tail;
  __device__ inline Row(const T* p, int len) {
    x = p;
    n = len;
    head = min(n, (int)((0 - (uintptr_t)p & 15) / sizeof(T)));
    units = (n - head) / E;
    tail = n - head - units * E;
  }
  __device__ inline u32x4 unit(int u) const { return *(const u32x4*)(x + head + (size_t)u * E); }
  __device__ inline int index(int u, int e) const { return head + u * E + e; }
  // the values outside whole units, one per thread: thread i < head + tail
  __device__ inline int edge(int i) const { return i < head ? i : n - tail + (i - head); }
};

// over the lanes of a wave, in each of them (DPP row shifts, then row broadcasts)
template <int CTRL, int ROWS>
__device__ inline float dpp_max(float v) {
  return fmaxf(v, __uint_as_float(__builtin_amdgcn_update_dpp(
                      __float_as_uint(v), __float_as_uint(v), CTRL, ROWS, 0xf, false)));
}
__device__ inline float wave_max(float v) {
  v = dpp_max<0x111, 0xf>(v);
  v = dpp_max<0x112, 0xf>(v);
  v = dpp_max<0x114, 0xf>(v);
  v = dpp_max<0x118, 0xf>(v);
  v = dpp_max<0x142, 0xa>(v);
  v = dpp_max<0x143, 0xc>(v);
  return __uint_as_float(__builtin_amdgcn_readlane(__float_as_uint(v), 63));
}
template <int CTRL, int ROWS>
__device__ inline double dpp_add(double v) {
  const uint64_t u = __builtin_bit_cast(uint64_t, v);
  const uint32_t lo = __builtin_amdgcn_update_dpp(0u, (uint32_t)u, CTRL, ROWS, 0xf, false);
  const uint32_t hi = __builtin_amdgcn_update_dpp(0u, (uint32_t)(u >> 32), CTRL, ROWS, 0xf, false);
  return v + __builtin_bit_cast(double, ((uint64_t)hi << 32) | lo);
}
__device__ inline double wave_sum(double v) {
  v = dpp_add<0x111, 0xf>(v);
  v = dpp_add<0x112, 0xf>(v);
  v = dpp_add<0x114, 0xf>(v);
  v = dpp_add<0x118, 0xf>(v);
  v = dpp_add<0x142, 0xa>(v);
  v = dpp_add<0x143, 0xc>(v);
  const uint64_t u = __builtin_bit_cast(uint64_t, v);
  const uint32_t lo = __builtin_amdgcn_readlane((uint32_t)u, 63);
  const uint32_t hi = __builtin_amdgcn_readlane((uint32_t)(u >> 32), 63);
  return __builtin_bit_cast(double, ((uint64_t)hi << 32) | lo);
}
// 2^k, good to 2^-23: the whole part exactly, the rest by the fp32 instruction
// (0 for -inf)
__device__ inline double power(double k) {
  k = fmax(k, -4000.0);
  const double n = __builtin_rint(k);
  return __builtin_ldexp((double)__builtin_amdgcn_exp2f((float)(k - n)), (int)n);
}
// the next float above x (finite)
__device__ constexpr float next_up(float x) {
  const uint32_t b = __builtin_bit_cast(uint32_t, x);
  return __builtin_bit_cast(float, x == 0.f ? 1u : x > 0.f ? b + 1 : b - 1);
}
// ln p of the value v, from the row's maximum and sum
__device__ inline float log_prob(float v, float M, double Z, double lnz) {
  if (v != v || Z == 0.0) return -INFINITY;
  return v == M ? (float)(0.0 - lnz) : (float)(((double)v - (double)M) - lnz);   // (no -0)
}
// the value of a value_key
__device__ inline float key_value(uint32_t k) {
  return __uint_as_float((k & 0x80000000u) ? k & 0x7FFFFFFFu : ~k);
}

template <typename T>
__global__ __launch_bounds__(kThreads) void logprobs_kernel(const LogprobArgs A) {
  constexpr int E = Row<T>::E;
  constexpr int NT = kThreads, UN = kUnits, NW = NT / 64;
  __shared__ double s_z[NW], s_s[NW];
  __shared__ float s_m[NW];
  __shared__ float s_max[NT];
  __shared__ float s_bound;
  __shared__ int s_int[NW];
  __shared__ int s_count;
  __shared__ uint64_t s_cand[kCand];

  const int tid = threadIdx.x, lane = tid & 63;
  const int wave = __builtin_amdgcn_readfirstlane(tid >> 6);
  const int row = blockIdx.x, part = blockIdx.y;
  const int top = A.top;
  int32_t* const tidx = A.top_idx + (size_t)row * top;
  float* const tlp = A.top_lp + (size_t)row * top;
  const size_t at_part = (size_t)row * A.parts + part;
  uint64_t* const keys = A.keys + at_part * top;
  if (A.n_nodes && row % A.budget >= A.n_nodes[row / A.budget]) {
    if (part > 0) return;   // (part 0 writes such a row, the second kernel leaves it as it is)
    if (tid < top) tidx[tid] = -1, tlp[tid] = 0.f;
    if (tid == 0) A.logprob[row] = 0.f, A.entropy[row] = 0.f, A.rank[row] = -1;
    return;
  }
  // the values from j0 on: parts begin at whole units, the first and the last take the edges
  int j0 = 0, j1 = A.vocab;
  const T* const x0 = (const T*)(A.x + (size_t)row * A.row_bytes);
  if (A.parts > 1) {
    const Row<T> all(x0, A.vocab);
    auto begin = [&](int q) { return all.head + all.units * q / A.parts * E; };
    if (part > 0) j0 = begin(part);
    if (part < A.parts - 1) j1 = begin(part + 1);
  }
  const Row<T> R(x0 + j0, j1 - j0);
  constexpr int step = NT * UN;
  const int whole = R.units / step, nb = (R.units + step - 1) / step;   // batches
  u32x4 cur[UN], nxt[UN];
  auto fetch = [&](int k, u32x4 (&r)[UN]) __attribute__((always_inline)) {
#pragma unroll
    for (int j = 0; j < UN; ++j) r[j] = R.unit(min(k * step + j * NT + tid, R.units - 1));
  };
  if (nb > 0) fetch(0, cur);
  auto each = [&](auto f) {   // f(value, index) of the thread's values, a unit at a time
    for (int u = tid; u < R.units; u += NT) {
      const u32x4 r = R.unit(u);
#pragma unroll
      for (int e = 0; e < E; ++e) f(unit_value<T>(r, e), R.index(u, e));
    }
    if (tid < R.head + R.tail) f(value_at(R.x, R.edge(tid)), R.edge(tid));
  };

  const int token = A.tokens[row];
  const bool given = token >= 0 && token < A.vocab;
  const float xt = given ? value_at(x0, token) : 0.f;
  const int tok = token - j0;   // (among this part's values, or before or past them)
  // values that come before the token: above it, or equal and of a lower index.  Units before
  // the token's compare with the next value below it.
  const bool ordinary = given && xt == xt && xt != -INFINITY;
  const float xt_below =
      xt == 0.f ? -1.4e-45f
                : __uint_as_float(__float_as_uint(xt) + (xt > 0.f ? 0xFFFFFFFFu : 1u));
  const int tok_unit = tok >= R.head ? (tok - R.head) / E : -1;   // (past the last: the tail's)

  // ---- one pass
  float Z, S, c, ref, best, rest;   // best: largest value; rest: the largest of other batches
  int best_at, before;              // before: of the wave's values
  // mx: the largest of the values that come next, of batch `at`
  auto expect = [&](float mx, int at) __attribute__((always_inline)) {
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
  };
  auto add = [&](const float* x, int n) __attribute__((always_inline)) {
#pragma unroll
    for (int e = 0; e < n; ++e) {
      const float t = fmaf(x[e], kLog2e, c);
      const float w = __builtin_amdgcn_exp2f(t);
      Z += w;
      S = fmaf(w, t, S);
    }
  };
  // batch k in r; careful: values lifted, units past the row as kLow, where a whole round of them
  // is past it left out
  auto batch = [&](auto careful, const u32x4 (&r)[UN], int k) __attribute__((always_inline)) {
    constexpr bool C = decltype(careful)::value;
    const int rounds = C ? min(UN, (R.units - k * step + NT - 1) / NT) : UN;
    float x[UN * E], m[2] = {-INFINITY, -INFINITY};
#pragma unroll
    for (int j = 0; j < UN; ++j) {
      if (C && j >= rounds) break;
      const int u = k * step + j * NT + tid;
      const float thr = u < tok_unit ? xt_below : xt;
#pragma unroll
      for (int e = 0; e < E; ++e) {
        float v = unit_value<T>(r[j], e);
        if constexpr (C) v = u < R.units ? v : -INFINITY;
        before += __popcll(__ballot(v > thr));
        x[j * E + e] = C ? lifted(v) : v;
      }
      asm volatile("" : "+s"(before));   // counted now: masks kept for later were spilled
#pragma unroll
      for (int e = 0; e < E; e += 2)
        m[(e >> 1) & 1] = max3(m[(e >> 1) & 1], x[j * E + e], x[j * E + e + 1]);
    }
    expect(max3(m[0], m[1], m[1]), k);
#pragma unroll
    for (int j = 0; j < UN; ++j) {
      if (C && j >= rounds) break;
      add(x + j * E, E);
    }
  };
  auto pass = [&](auto careful) __attribute__((always_inline)) {
    Z = S = c = 0.f;
    ref = best = rest = -INFINITY;
    best_at = before = 0;
    int k = 0;
    if constexpr (!decltype(careful)::value) {
      for (; k + 1 < whole; k += 2) {   // (fetch: past the last the same again)
        fetch(k + 1, nxt);
        batch(careful, cur, k);
        fetch(k + 2, cur);
        batch(careful, nxt, k + 1);
      }
      if (k < whole) {
        fetch(k + 1, nxt);
        batch(careful, cur, k++);
#pragma unroll
        for (int j = 0; j < UN; ++j) cur[j] = nxt[j];
      }
    }
    for (; k < nb; ++k) {
      fetch(k + 1, nxt);
      batch(Flag<true>(), cur, k);
#pragma unroll
      for (int j = 0; j < UN; ++j) cur[j] = nxt[j];
    }
    // the edges; ties in the token's own unit
    const bool in = tid < R.head + R.tail;
    const int j = R.edge(in ? tid : 0);
    const float v = in ? value_at(R.x, j) : -INFINITY;
    before += __popcll(__ballot(in && (j < tok ? v >= xt : v > xt)));
    if (__ballot(in)) {
      const float x = lifted(v);
      if (in) expect(x, nb), add(&x, 1);
    }
    if (wave == 0 && given && tok_unit >= 0 && tok_unit < R.units) {
      const int u0 = R.index(tok_unit, 0);
      before += __popcll(__ballot(lane < tok - u0 && value_at(R.x, u0 + min(lane, E - 1)) == xt));
    }
  };
  {
    bool odd = false;
    if (nb > 0) {
#pragma unroll
      for (int e = 0; e < E; ++e) odd = odd || !(fabsf(unit_value<T>(cur[0], e)) < INFINITY);
    }
    bool careful = __ballot(odd) != 0;
    if (!careful) {
      pass(Flag<false>());
      careful = __ballot(!(fabsf(S) < INFINITY && fabsf(Z) < INFINITY)) != 0;
      if (careful && nb > 0) fetch(0, cur);
    }
    if (careful) pass(Flag<true>());
  }
  if (!ordinary && given) {   // a token of -inf or NaN: its rank by the definition
    const uint32_t kt = value_key(__float_as_uint(xt));
    int mine = 0;
    each([&](float v, int j) {
      const uint32_t k = value_key(__float_as_uint(v));
      mine += k > kt || (k == kt && j < tok);
    });
    before = (int)wave_sum((double)mine);
  }

  // ---- the waves' sums about their own maxima (ref -inf: a thread without values)
  {
    const float m = wave_max(best);
    double a = 0.0, k = 0.0, rz = Z, rs = S;
    if (ref != -INFINITY) {
      k = -(double)c + (double)ref * kLog2eRest - (double)m * 1.4426950408889634;
      a = power(k);
    }
    // (`best` was added about the reference that is in force: a larger one moves it)
    const bool holds = best == m && ref != -INFINITY;
    if (holds) {
      const float t = fmaf(best, kLog2e, c), w = __builtin_amdgcn_exp2f(t);
      rz -= w, rs -= fmaf(w, t, 0.f);
    }
    const double z = wave_sum(a * rz + (holds ? 1.0 : 0.0)), sn = wave_sum(a * (rs + k * rz));
    s_max[tid] = best;
    if (lane == 0) s_m[wave] = m, s_z[wave] = z, s_s[wave] = sn, s_int[wave] = before;
    if (tid == 0) s_count = 0;
  }
  __syncthreads();
  float M;
  double Zd, Sd, Md;
  int rank = 0;
  {
    const int w = min(lane, NW - 1);
    const float m = s_m[w];
    M = wave_max(m);
    Md = M;
    const double k = ((double)m - Md) * 1.4426950408889634;
    const bool in = lane < NW && m != -INFINITY;
    const double a = in ? power(k) : 0.0;
    Zd = wave_sum(in ? a * s_z[w] : 0.0);
    Sd = wave_sum(in ? a * (s_s[w] + k * s_z[w]) : 0.0) * 0.6931471805599453;
#pragma unroll
    for (int q = 0; q < NW; ++q) rank += s_int[q];
  }
  const bool special = !(M > kLow + 1000.f && M < kHigh);
  if (special) {
    // about kLow or below, or above kHigh: weights by the definition
    float m = -INFINITY;
    bool any = false;
    each([&](float v, int) {
      if (v == v) m = v > m ? v : m, any = true;
    });
    m = wave_max(m);
    __syncthreads();
    if (lane == 0) s_m[wave] = m;
    const int have = __syncthreads_or(any);
    M = -INFINITY;
#pragma unroll
    for (int w = 0; w < NW; ++w) M = fmaxf(M, s_m[w]);
    Md = M;
    double z = 0.0, sn = 0.0;
    if (have) each([&](float v, int) {
      if (v == M) {
        z += 1.0;
      } else if (v == v && !isinf(M)) {
        const double d = (double)v - Md, w = exp(d);
        z += w;
        if (w > 0.0) sn += w * d;
      }
    });
    z = wave_sum(z), sn = wave_sum(sn);
    if (lane == 0) s_z[wave] = z, s_s[wave] = sn;
    __syncthreads();
    Zd = Sd = 0.0;
#pragma unroll
    for (int w = 0; w < NW; ++w) Zd += s_z[w], Sd += s_s[w];
  }
  const double lnz = A.parts == 1 ? log(Zd) : 0.0;   // (parts: the second kernel takes it)
  auto lp = [&](float v) { return log_prob(v, M, Zd, lnz); };
  auto found = [&](int r, uint64_t key) {   // the row's (part's) r-th value
    if (A.parts > 1) {
      keys[r] = key;
    } else {
      tidx[r] = (int)cand_index(key);
      tlp[r] = lp(key_value((uint32_t)(key >> 32)));
    }
  };
  if (tid == 0 && A.parts > 1) A.part[at_part] = Part{Zd, Sd, M, rank, xt, given};
  if (tid == 0 && A.parts == 1) {
    A.rank[row] = given ? rank : -1;
    A.logprob[row] = given ? lp(xt) : -INFINITY;
    A.entropy[row] = Zd == 0.0 ? 0.f : (float)fmax(lnz - Sd / Zd, 0.0);
  }
  if (top == 0) return;

  // ---- top alternatives: a bound from below, the smallest maximum that fewer than `top` groups of
  // threads exceed
  float bound = -INFINITY;
  if (!special) {
    if (top <= kFewTop) {   // 64 groups, by the first wave
      if (wave == 0) {
        float v = s_max[lane];
#pragma unroll
        for (int w = 1; w < NW; ++w) v = fmaxf(v, s_max[w * 64 + lane]);
        int above = 0;
#pragma unroll
        for (int q = 0; q < 64; ++q)
          above += __uint_as_float(__builtin_amdgcn_readlane(__float_as_uint(v), q)) > v;
        const float low = -wave_max(above < top ? -v : -INFINITY);
        if (lane == 0) s_bound = low;
      }
    } else {                // NT / 2, by their threads
      float v = INFINITY;
      if (tid < NT / 2) s_max[tid] = v = fmaxf(s_max[tid], s_max[tid + NT / 2]);
      __syncthreads();
      int above = 0;
#pragma unroll 8
      for (int q = 0; q < NT / 2; ++q) above += s_max[q] > v;
      const float low = wave_max(tid < NT / 2 && above < top ? -v : -INFINITY);
      if (lane == 0) s_m[wave] = low;
      __syncthreads();
      if (wave == 0) {
        const float all = -wave_max(s_m[min(lane, NW - 1)]);
        if (lane == 0) s_bound = all;
      }
    }
    __syncthreads();
    bound = s_bound;
  }
  uint64_t last = 1ull << 32;   // values below this key are still to be found: all of them
  int have = 0;
  auto rank_found = [&](int n) {   // the n candidates in LDS
    for (int q = tid; q < n; q += NT) {
      const uint64_t mine = s_cand[q];
      int r = 0;
#pragma unroll 8
      for (int j = 0; j < n; ++j) r += s_cand[j] > mine;
      if (r < top) found(r, mine);
    }
    have = min(n, top);
  };
  if (!(bound > kLow) && R.n <= kCand) {   // few values: all of them
    for (int j = tid; j < R.n; j += NT)
      s_cand[j] = cand_key(value_key(__float_as_uint(value_at(R.x, j))), (uint32_t)(j0 + j));
    __syncthreads();
    rank_found(R.n);
    last = 0;
  } else if (!special) {
    bound = fmaxf(bound, next_up(kLow));   // masked rows: the values above kLow
    for (;;) {
      auto offer = [&](float v, int j) {
        if (v >= bound) {
          const int at = atomicAdd(&s_count, 1);
          if (at < kCand) s_cand[at] = cand_key(value_key(__float_as_uint(v)), (uint32_t)(j0 + j));
        }
      };
      if (best >= bound) {
        const bool all = rest >= bound;
        for (int k = all ? 0 : best_at; k < (all ? nb : min(best_at + 1, nb)); ++k) {
          u32x4 r[UN];
          fetch(k, r);
#pragma unroll
          for (int j = 0; j < UN; ++j) {
            const int u = k * step + j * NT + tid;
            if (u < R.units) {
#pragma unroll
              for (int e = 0; e < E; ++e) offer(unit_value<T>(r[j], e), R.index(u, e));
            }
          }
        }
        if (tid < R.head + R.tail) offer(value_at(R.x, R.edge(tid)), R.edge(tid));
      }
      __syncthreads();
      const int n = s_count;
      if (n <= kCand) {
        rank_found(n);
        last = value_key(__float_as_uint(bound));
        break;
      }
      // too many: from the `top`-th of those that were kept, or, where the bound itself occurs too
      // often, above it (its places follow in index order)
      static_assert(kCand == NT, "a candidate per thread");
      const uint64_t mine = s_cand[tid];
      int r = 0;
      for (int j = 0; j < kCand; ++j) r += s_cand[j] > mine;
      __syncthreads();
      if (r == top - 1) s_bound = key_value((uint32_t)(mine >> 32));
      if (tid == 0) s_count = 0;
      __syncthreads();
      bound = s_bound > bound ? s_bound : next_up(bound);
    }
  }

  // ---- the rest value by value: the largest key below the last one, then its indices in order
  while (have < top) {
    uint32_t m = 0;
    bool any = false;
    each([&](float v, int) {
      const uint32_t k = value_key(__float_as_uint(v));
      if (k < last) m = max(m, k), any = true;
    });
#pragma unroll
    for (int o = 32; o >= 1; o >>= 1) m = max(m, (uint32_t)__shfl_xor((int)m, o));
    __syncthreads();
    if (lane == 0) s_int[wave] = (int)m;
    if (!__syncthreads_or(any)) break;   // a part of fewer values
    m = 0;
#pragma unroll
    for (int w = 0; w < NW; ++w) m = max(m, (uint32_t)s_int[w]);
    for (int q = 0; q < R.n && have < top; q += NT * 8) {   // 8 neighbours a thread
      uint32_t hits = 0;
#pragma unroll
      for (int e = 0; e < 8; ++e) {
        const int j = q + tid * 8 + e;
        if (j < R.n && value_key(__float_as_uint(value_at(R.x, j))) == m) hits |= 1u << e;
      }
      int incl = __popc(hits);
      const int mine = incl;
#pragma unroll
      for (int o = 1; o < kWave; o <<= 1) {
        const int below = __shfl_up(incl, o);
        if (lane >= o) incl += below;
      }
      __syncthreads();
      if (lane == kWave - 1) s_int[wave] = incl;
      __syncthreads();
      int at = have + incl - mine, total = 0;
#pragma unroll
      for (int w = 0; w < NW; ++w) {
        if (w < wave) at += s_int[w];
        total += s_int[w];
      }
      for (; hits != 0 && at < top; ++at, hits &= hits - 1)
        found(at, cand_key(m, (uint32_t)(j0 + q + tid * 8 + __ffs((int)hits) - 1)));
      have += total;
    }
    last = m;
  }
  if (A.parts > 1 && tid >= have && tid < top) keys[tid] = 0;   // (no value's key)
}

// A row from its parts: a workgroup a row.
constexpr int kJoinThreads = 256, kMaxParts = 16;
__global__ __launch_bounds__(kJoinThreads) void logprobs_join_kernel(const LogprobArgs A) {
  __shared__ uint64_t s_key[kMaxParts * TAPS_MAX_LOGPROB_TOP];
  const int tid = threadIdx.x, lane = tid & 63, top = A.top;
  const int row = blockIdx.x;
  const int n = A.parts * top;
  for (int q = tid; q < n; q += kJoinThreads) s_key[q] = A.keys[(size_t)row * n + q];
  const Part p = A.part[(size_t)row * A.parts + min(lane, A.parts - 1)];
  if (A.n_nodes && row % A.budget >= A.n_nodes[row / A.budget]) return;   // written
  const bool in = lane < A.parts;
  const float M = wave_max(p.M);
  // parts without values but NaN have Z 0; equal maxima may be infinite
  const double d = p.M == M ? 0.0 : (double)p.M - (double)M;
  const double a = in && p.Z > 0.0 ? power(d * 1.4426950408889634) : 0.0;
  const double Z = wave_sum(a * p.Z), S = wave_sum(a > 0.0 ? a * (p.S + d * p.Z) : 0.0);
  const int rank = (int)wave_sum(in ? (double)p.before : 0.0);
  const double lnz = log(Z);
  if (tid == 0) {
    A.rank[row] = p.given ? rank : -1;
    A.logprob[row] = p.given ? log_prob(p.token, M, Z, lnz) : -INFINITY;
    A.entropy[row] = Z == 0.0 ? 0.f : (float)fmax(lnz - S / Z, 0.0);
  }
  __syncthreads();
  for (int q = tid; q < n; q += kJoinThreads) {
    const uint64_t mine = s_key[q];
    int r = 0;
    if (n <= 64) {
#pragma unroll 8
      for (int j = 0; j < n; ++j) r += s_key[j] > mine;
    } else {   // each part's are in order: by bisection
      for (int p = 0; p < n; p += top) {
        int lo = 0, hi = top;
        while (lo < hi) {
          const int mid = (lo + hi) >> 1;
          if (s_key[p + mid] > mine) lo = mid + 1;
          else hi = mid;
        }
        r += lo;
      }
    }
    if (r >= top || mine == 0) continue;
    A.top_idx[(size_t)row * top + r] = (int)cand_index(mine);
    A.top_lp[(size_t)row * top + r] = log_prob(key_value((uint32_t)(mine >> 32)), M, Z, lnz);
  }
}

}  // namespace

// Parts of a row: a workgroup for each CU where the rows are few (two, for more than 64 long rows),
// none with less than a whole batch of values.  The vector unit of one CU bounds a row on its own
// (152K values in bf16: 8 us); the join costs 4 us and more workgroups contend.  us a call (5
// alternatives, from graphs) with 1 / 2 / 4 / 8 parts, bf16 rows of 151,936: one row 16.8 / 14.6 /
// 12.3 / 11.5, 64 rows 25.9 / 19.3 / 14.6 / 15.0, 96 rows 25.7 / 19.5 / 18.1 / 17.9, 160 rows (1 /
// 2 / 3 / 4) 27.0 / 26.3 / 22.8 / 22.4, 256 rows 29.0 / 28.5 / 28.7 / 36.4; fp32 rows of 50,257:
// one 10.1 / 10.6 / 10.1 / 9.7, 96 rows 13.2 / 12.7 / 13.4 / 14.6, 256 rows 17.3 / 19.5 / 21.5 /
// 29.0; 64 bf16 rows of 100,000 19.4 / 15.4 / 13.5 / 15.0; bf16 rows of 32,000: one 9.1 / 10.7 /
// 9.9 / 9.5.
int logprobs_parts(int64_t rows, int vocab, int dtype) {
  if (rows <= 0) return 1;
  const int64_t batch = kThreads * kUnits * (dtype == TAPS_BF16 ? 8 : 4);
  const int64_t most = std::min<int64_t>(kMaxParts, vocab / batch);
  const int wgs = rows > 64 && most >= 8 ? 512 : 256;
  return (int)std::max<int64_t>(1, std::min<int64_t>(most, wgs / rows));
}
size_t logprobs_ws_bytes(int64_t rows, int vocab, int dtype, int top) {
  const int parts = logprobs_parts(rows, vocab, dtype);
  return parts > 1 ? (size_t)rows * parts * (sizeof(Part) + (size_t)top * sizeof(uint64_t)) : 0;
}

hipError_t launch_logprobs(const void* logits, int64_t row_bytes, int batch, int budget,
                           int vocab, int dtype, const int32_t* n_nodes, const int32_t* tokens,
                           int top, float* logprob, float* entropy, int32_t* rank,
                           int32_t* top_idx, float* top_logprob, void* ws, hipStream_t s) {
  const int64_t rows = (int64_t)batch * budget;
  if (rows <= 0) return hipSuccess;
  LogprobArgs A;
  A.x = (const unsigned char*)logits, A.row_bytes = row_bytes;
  A.budget = budget, A.vocab = vocab, A.top = top, A.n_nodes = n_nodes, A.tokens = tokens;
  A.logprob = logprob, A.entropy = entropy, A.rank = rank;
  A.top_idx = top_idx, A.top_lp = top_logprob;
  A.parts = logprobs_parts(rows, vocab, dtype);
  A.part = (Part*)ws;
  A.keys = (uint64_t*)(A.part + rows * A.parts);
  const dim3 grid((unsigned)rows, (unsigned)A.parts);
  if (dtype == TAPS_BF16) logprobs_kernel<uint16_t><<<grid, kThreads, 0, s>>>(A);
  else logprobs_kernel<float><<<grid, kThreads, 0, s>>>(A);
  const hipError_t e = hipGetLastError();
  if (e != hipSuccess || A.parts == 1) return e;
  logprobs_join_kernel<<<(unsigned)rows, kJoinThreads, 0, s>>>(A);
  return hipGetLastError();
}

}  // namespace taps

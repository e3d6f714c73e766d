// Token sampling with temperature, top-k, top-p and min-p from given random numbers
// (taps_sample).
//
// A row's tokens in rank order (value descending, index ascending, NaN last) have weights
//   W_r = rint(2^43 exp((x_r - x_0) / T)),
// integers, so that every sum below is exact: the result does not depend on the order in which
// a kernel adds, and 2^20 weights stay below 2^63.  top-k, top-p and min-p each keep a prefix
// of the rank order, so the sum S over the kept set is the smallest of the prefixes' sums
//   S_k = sum over the first top_k,   S_p = the first sum that reaches top_p * S_k,
//   S_m = sum over weights >= min_p,
// and the token is the first whose running sum exceeds floor(u S).  Each of these is one
// question: at which token does the running count or sum in rank order pass a target?
#include "common.h"

namespace taps {

namespace {

constexpr int kThreads = 1024;
constexpr int kWaves = kThreads / kWave;
constexpr double kOne = 8796093022208.0;   // 2^43, the weight of the largest value

// 2^y for -45 < y <= 0: y = k + r, |r| <= 1/2, e^(r ln 2) by its Taylor series to the 12th power
// (remainder below 2^-52), exact at y = 0.
__device__ inline double exp2_neg(double y) {
  const double k = rint(y);
  const double t = (y - k) * 0.69314718055994530942;
  double p = 1.0 / 479001600.0;
  p = fma(p, t, 1.0 / 39916800.0);
  p = fma(p, t, 1.0 / 3628800.0);
  p = fma(p, t, 1.0 / 362880.0);
  p = fma(p, t, 1.0 / 40320.0);
  p = fma(p, t, 1.0 / 5040.0);
  p = fma(p, t, 1.0 / 720.0);
  p = fma(p, t, 1.0 / 120.0);
  p = fma(p, t, 1.0 / 24.0);
  p = fma(p, t, 1.0 / 6.0);
  p = fma(p, t, 0.5);
  p = fma(p, t, 1.0);
  p = fma(p, t, 1.0);
  return ldexp(p, (int)k);
}

// the float whose value_key is `key`
__device__ inline float key_value(uint32_t key) {
  return __uint_as_float((key & 0x80000000u) ? (key & 0x7FFFFFFFu) : ~key);
}

struct Weights {
  float top;       // the row's largest value
  uint32_t key;    // its key
  double scale;    // log2(e) / T
  // log2 of the weight relative to the largest one's; 0 for equal values (infinities too)
  __device__ inline double log2w(uint32_t k) const {
    return k == key ? 0.0 : ((double)key_value(k) - (double)top) * scale;
  }
  __device__ inline uint64_t operator()(uint32_t k) const {   // k != 0 (not NaN)
    const double y = log2w(k);
    return y > -44.5 ? (uint64_t)rint(exp2_neg(y) * kOne) : 0ull;
  }
};

__device__ inline uint64_t wave_sum_u64(uint64_t v) {
#pragma unroll
  for (int m = 32; m >= 1; m >>= 1) {
    const uint32_t lo = __shfl_xor((uint32_t)v, m), hi = __shfl_xor((uint32_t)(v >> 32), m);
    v += ((uint64_t)hi << 32) | lo;
  }
  return v;
}

constexpr int kBins = 2048;

struct Shared {
  uint64_t mass[kBins];
  uint32_t count[kBins];
  uint64_t red[kWaves];
  uint32_t red32[kWaves];
  uint64_t out64[2];
  uint32_t out32[4];
};

// One row of logits, read 16 bytes at a time; f(key, index) for the elements of this thread.
template <int DT>
struct Row {
  static constexpr int U = DT == TAPS_BF16 ? 8 : 4;   // elements per 16 bytes
  const char* base;
  int vocab, lead, units;   // lead: elements that the first unit lacks

  __device__ inline Row(const void* p, int v) : base((const char*)p), vocab(v) {
    constexpr int es = 16 / U;
    lead = (int)(((uintptr_t)p & 15) / es);
    units = (v + lead + U - 1) / U;
  }
  __device__ inline uint32_t key_at(int i) const {
    return value_key(DT == TAPS_BF16 ? (uint32_t)((const uint16_t*)base)[i] << 16
                                     : ((const uint32_t*)base)[i]);
  }
  template <class F>
  __device__ inline void unit(int u, F&& f) const {
    const int e0 = u * U - lead;
    if (e0 >= 0 && e0 + U <= vocab) {
      const uint4 w = *(const uint4*)(base + (int64_t)e0 * (16 / U));
      const uint32_t ww[4] = {w.x, w.y, w.z, w.w};
#pragma unroll
      for (int q = 0; q < 4; ++q) {
        if (DT == TAPS_BF16) {
          f(value_key(ww[q] << 16), e0 + 2 * q);
          f(value_key(ww[q] & 0xFFFF0000u), e0 + 2 * q + 1);
        } else {
          f(value_key(ww[q]), e0 + q);
        }
      }
    } else {
      for (int e = max(e0, 0); e < min(e0 + U, vocab); ++e) f(key_at(e), e);
    }
  }
  template <class F>
  __device__ inline void each(F&& f) const {
    for (int u = threadIdx.x; u < units; u += kThreads) unit(u, f);
  }
};

__device__ inline uint64_t block_sum_u64(uint64_t v, Shared& sh) {
  v = wave_sum_u64(v);
  const int lane = threadIdx.x & (kWave - 1), wave = threadIdx.x / kWave;
  __syncthreads();
  if (lane == 0) sh.red[wave] = v;
  __syncthreads();
  uint64_t s = 0;
#pragma unroll
  for (int w = 0; w < kWaves; ++w) s += sh.red[w];
  return s;
}

__device__ inline uint32_t block_max_u32(uint32_t v, Shared& sh) {
#pragma unroll
  for (int m = 32; m >= 1; m >>= 1) v = max(v, (uint32_t)__shfl_xor(v, m));
  const int lane = threadIdx.x & (kWave - 1), wave = threadIdx.x / kWave;
  __syncthreads();
  if (lane == 0) sh.red32[wave] = v;
  __syncthreads();
  uint32_t s = 0;
#pragma unroll
  for (int w = 0; w < kWaves; ++w) s = max(s, sh.red32[w]);
  return s;
}

// Where the running sum of the weights (or, with `by_count`, the count) in rank order first
// exceeds `target`: the value's key, the sum and the count above it, and its ties.  `target` is
// below the whole sum (count).  Radix descent over the key, 11 + 11 + 10 bits from the top (the
// 16 bits that bf16 keys have: 11 + 5).
struct Crossing {
  uint32_t key;
  uint64_t above;    // sum (count) of the elements whose key is larger
  uint32_t ties;     // elements with this key
};

template <int DT>
__device__ Crossing find_crossing(const Row<DT>& row, const Weights& w, uint64_t target,
                                  bool by_count, Shared& sh) {
  const int tid = threadIdx.x;
  uint32_t prefix = 0;
  uint64_t above = 0;
  uint32_t ties = 0;
  int low = 32;
  while (low > (DT == TAPS_BF16 ? 16 : 0)) {
    const int bits = low == 10 ? 10 : (DT == TAPS_BF16 && low == 21 ? 5 : 11);
    const int high = low;
    low -= bits;
    for (int i = tid; i < kBins; i += kThreads) sh.mass[i] = 0ull, sh.count[i] = 0u;
    __syncthreads();
    row.each([&](uint32_t k, int) {
      if (k == 0u || (high < 32 && (k >> high) != prefix)) return;   // NaN has no weight
      const uint32_t bin = (k >> low) & ((1u << bits) - 1u);
      const uint64_t m = by_count ? 1ull : w(k);
      if (m) {
        atomicAdd((unsigned long long*)&sh.mass[bin], (unsigned long long)m);
        atomicAdd(&sh.count[bin], 1u);
      }
    });
    __syncthreads();
    if (tid < kWave) {   // one wave walks the bins from the top, 64 at a time
      uint64_t acc = above;
      bool found = false;
      for (int c = (1 << bits) - kWave; !found && c > -kWave; c -= kWave) {
        const int bin = c + (kWave - 1 - tid);        // lane 0 holds the highest
        const uint64_t m = bin >= 0 ? sh.mass[bin] : 0ull;
        uint64_t incl = m;
#pragma unroll
        for (int d = 1; d < kWave; d <<= 1) {
          const uint32_t lo = __shfl_up((uint32_t)incl, d), hi = __shfl_up((uint32_t)(incl >> 32), d);
          if (tid >= d) incl += ((uint64_t)hi << 32) | lo;
        }
        const uint64_t hit = __ballot(acc + incl > target);
        if (hit) {
          const int l = __ffsll((long long)hit) - 1;
          if (tid == l) {
            sh.out32[0] = (uint32_t)bin;
            sh.out32[1] = sh.count[bin];
            sh.out64[0] = acc + incl - m;
          }
          found = true;
        }
        const uint32_t lo = __shfl((uint32_t)incl, kWave - 1), hi = __shfl((uint32_t)(incl >> 32), kWave - 1);
        acc += ((uint64_t)hi << 32) | lo;
      }
    }
    __syncthreads();
    prefix = (prefix << bits) | sh.out32[0];
    ties = sh.out32[1];
    above = sh.out64[0];
    __syncthreads();
  }
  // a bf16 value's key ends in 16 zeros, or ones where the value is negative
  if (DT == TAPS_BF16) prefix = (prefix << 16) | ((prefix & 0x8000u) ? 0u : 0xFFFFu);
  return {prefix, above, ties};
}

// index of the nth (from 0) element whose key is `key`, in index order
template <int DT>
__device__ int nth_index(const Row<DT>& row, uint32_t key, uint32_t nth, Shared& sh) {
  const int tid = threadIdx.x, lane = tid & (kWave - 1), wave = tid / kWave;
  uint32_t seen = 0;
  for (int u0 = 0; u0 < row.units; u0 += kThreads) {
    uint32_t n = 0;
    if (u0 + tid < row.units) row.unit(u0 + tid, [&](uint32_t k, int) { n += k == key ? 1u : 0u; });
    uint32_t incl = n;
#pragma unroll
    for (int d = 1; d < kWave; d <<= 1) {
      const uint32_t o = __shfl_up(incl, d);
      if (lane >= d) incl += o;
    }
    __syncthreads();
    if (lane == kWave - 1) sh.red32[wave] = incl;
    __syncthreads();
    uint32_t before = seen, all = 0;
#pragma unroll
    for (int v = 0; v < kWaves; ++v) {
      if (v < wave) before += sh.red32[v];
      all += sh.red32[v];
    }
    before += incl - n;
    if (before <= nth && nth < before + n) {
      uint32_t c = before;
      row.unit(u0 + tid, [&](uint32_t k, int e) {
        if (k == key && c++ == nth) sh.out32[2] = (uint32_t)e;
      });
    }
    seen += all;
    if (seen > nth) break;
  }
  __syncthreads();
  return (int)sh.out32[2];
}

struct Settings {
  const float *temperature, *top_p, *min_p;
  const int32_t* top_k;
};

template <int DT>
__global__ __launch_bounds__(kThreads) void sample_kernel(
    const void* __restrict__ logits, int64_t row_bytes, int budget, int vocab,
    const int32_t* __restrict__ n_nodes, const Settings st, const float* __restrict__ u,
    int32_t* __restrict__ tokens, float* __restrict__ probs) {
  __shared__ Shared sh;
  const int r = blockIdx.x, b = r / budget, tid = threadIdx.x;
  if (n_nodes && r - b * budget >= n_nodes[b]) {
    if (tid == 0) {
      tokens[r] = -1;
      if (probs) probs[r] = 0.f;
    }
    return;
  }
  const Row<DT> row((const char*)logits + (size_t)r * row_bytes, vocab);
  uint32_t best = 0;
  row.each([&](uint32_t k, int) { best = max(best, k); });
  best = block_max_u32(best, sh);

  const float T = st.temperature ? st.temperature[b] : 1.f;
  if (!(T > 0.f) || best == 0u) {   // greedy, or a row of NaN
    const int tok = nth_index<DT>(row, best, 0, sh);
    if (tid == 0) {
      tokens[r] = tok;
      if (probs) probs[r] = best ? 1.f : 0.f;
    }
    return;
  }
  Weights w;
  w.key = best;
  w.top = key_value(best);
  w.scale = 1.4426950408889634074 / (double)T;

  const int k = st.top_k ? st.top_k[b] : 0;
  const float p = st.top_p ? st.top_p[b] : 1.f, mp = st.min_p ? st.min_p[b] : 0.f;
  const double least = mp > 0.f ? fmin(log2((double)mp), 0.0) : -INFINITY;
  uint64_t S = 0, Sm = 0, have = 0;
  row.each([&](uint32_t key, int) {
    const uint64_t m = key ? w(key) : 0ull;
    S += m;
    have += m ? 1 : 0;
    if (m && w.log2w(key) >= least) Sm += m;
  });
  S = block_sum_u64(S, sh);
  Sm = block_sum_u64(Sm, sh);
  have = block_sum_u64(have, sh);
  if (k > 0 && (uint64_t)k < have) {
    // the k-th token's value; its larger ones and the first of its ties are kept
    const Crossing c = find_crossing<DT>(row, w, (uint64_t)(k - 1), true, sh);
    uint64_t sum = 0;
    row.each([&](uint32_t key, int) { sum += key > c.key ? w(key) : 0ull; });
    S = block_sum_u64(sum, sh) + ((uint64_t)k - c.above) * w(c.key);
  }
  if (p < 1.f) {
    const double need = ceil((double)fmaxf(p, 0.f) * (double)S);
    const uint64_t P = min(max((uint64_t)need, 1ull), S);
    const Crossing c = find_crossing<DT>(row, w, P - 1, false, sh);
    const uint64_t W = w(c.key);
    S = c.above + ((P - 1 - c.above) / W + 1) * W;
  }
  S = min(S, Sm);
  const float uf = u[r];
  const double t = floor((double)fminf(fmaxf(uf, 0.f), 1.f) * (double)S);
  const uint64_t target = min((uint64_t)t, S - 1);
  const Crossing c = find_crossing<DT>(row, w, target, false, sh);
  const uint64_t W = w(c.key);
  const int tok = nth_index<DT>(row, c.key, (uint32_t)((target - c.above) / W), sh);
  if (tid == 0) {
    tokens[r] = tok;
    if (probs) probs[r] = (float)((double)W / (double)S);
  }
}

}  // namespace

hipError_t launch_sample(const void* logits, int64_t row_bytes, int batch, int budget, int vocab,
                         int dtype, const int32_t* n_nodes, const taps_sampling& s,
                         const float* u, int32_t* tokens, float* probs, hipStream_t stream) {
  if (batch <= 0) return hipSuccess;
  const Settings st{s.temperature, s.top_p, s.min_p, s.top_k};
  const unsigned rows = (unsigned)(batch * budget);
  if (dtype == TAPS_BF16)
    sample_kernel<TAPS_BF16><<<rows, kThreads, 0, stream>>>(logits, row_bytes, budget, vocab,
                                                            n_nodes, st, u, tokens, probs);
  else
    sample_kernel<TAPS_FP32><<<rows, kThreads, 0, stream>>>(logits, row_bytes, budget, vocab,
                                                            n_nodes, st, u, tokens, probs);
  return hipGetLastError();
}

}  // namespace taps

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

constexpr int kBins = 2048;         // radix digits of the general path
constexpr int kWindow = 36864;      // bf16 values counted one by one, from the largest down
constexpr int kWindowRows = kWindow / kWave;
constexpr int kPerOctave = 32;      // fp32: bins of the weight per factor of two
constexpr int kWeightBins = 1424;   // 44.5 octaves: smaller weights round to 0
constexpr int kList = 1024;         // elements that are ranked one by one
constexpr int kGroups = kThreads / 4;
constexpr int kFewTopK = 192;       // top_k up to which the groups' maxima bound the window

// Scratch of the three paths, which a row takes one after the other at most
struct GeneralScratch {
  uint64_t mass[kBins];
  uint32_t count[kBins];
};
struct CountScratch {
  uint32_t count[kWindow];          // elements per value, the largest value first
  uint64_t mass[kWindowRows];       // sums of 64 values each; then those before them
  uint32_t num[kWindowRows];
};
struct BinScratch {
  uint64_t mass[kWeightBins];
  uint64_t before[kWeightBins];
  uint64_t list[kList], sorted[kList], cum[kList];
};
template <int DT>
union PathScratch {
  GeneralScratch g;
  CountScratch c;
};
template <>
union PathScratch<TAPS_FP32> {
  GeneralScratch g;
  BinScratch b;
};

template <int DT>
struct Shared {
  PathScratch<DT> u;
  uint32_t group[kGroups];
  uint64_t red[kWaves];
  uint32_t red32[kWaves];
  uint64_t out64[2];
  uint32_t out32[4];
  uint32_t n;
  uint32_t ties[kList];
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

template <int DT>
__device__ inline uint64_t block_sum_u64(uint64_t v, Shared<DT>& sh) {
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

template <int DT>
__device__ inline uint32_t block_max_u32(uint32_t v, Shared<DT>& sh) {
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
                                  bool by_count, Shared<DT>& sh) {
  const int tid = threadIdx.x;
  uint32_t prefix = 0;
  uint64_t above = 0;
  uint32_t ties = 0;
  int low = 32;
  while (low > (DT == TAPS_BF16 ? 16 : 0)) {
    const int bits = low == 10 ? 10 : (DT == TAPS_BF16 && low == 21 ? 5 : 11);
    const int high = low;
    low -= bits;
    for (int i = tid; i < kBins; i += kThreads) sh.u.g.mass[i] = 0ull, sh.u.g.count[i] = 0u;
    __syncthreads();
    row.each([&](uint32_t k, int) {
      if (k == 0u || (high < 32 && (k >> high) != prefix)) return;   // NaN has no weight
      const uint32_t bin = (k >> low) & ((1u << bits) - 1u);
      const uint64_t m = by_count ? 1ull : w(k);
      if (m) {
        atomicAdd((unsigned long long*)&sh.u.g.mass[bin], (unsigned long long)m);
        atomicAdd(&sh.u.g.count[bin], 1u);
      }
    });
    __syncthreads();
    if (tid < kWave) {   // one wave walks the bins from the top, 64 at a time
      uint64_t acc = above;
      bool found = false;
      for (int c = (1 << bits) - kWave; !found && c > -kWave; c -= kWave) {
        const int bin = c + (kWave - 1 - tid);        // lane 0 holds the highest
        const uint64_t m = bin >= 0 ? sh.u.g.mass[bin] : 0ull;
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
            sh.out32[1] = sh.u.g.count[bin];
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
__device__ __attribute__((noinline)) int nth_index(const Row<DT>& row, uint32_t key, uint32_t nth, Shared<DT>& sh) {
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

struct RowSettings {
  float T, p, mp, u;
  int k;
  // rows for the ranked few: what lies below the bounds of a small top_k, or of min_p unless
  // top_p needs the sum over more, does not matter
  __device__ inline bool few() const { return k > 0 && k <= kFewTopK; }
  __device__ inline bool cut_by_min_p() const { return mp > 0.f && !(p < 1.f); }
  // log2 of the smallest weight that min_p keeps, relative to the largest
  __device__ inline double least() const {
    return mp > 0.f ? fmin(log2((double)mp), 0.0) : -INFINITY;
  }
};

struct Drawn {
  int token;
  float prob;
};

// floor(u S), below S
__device__ inline uint64_t draw_target(float u, uint64_t S) {
  const double t = floor((double)fminf(fmaxf(u, 0.f), 1.f) * (double)S);
  return min((uint64_t)t, S - 1);
}
// the running sum that top_p asks for: ceil(p S), 1 .. S
__device__ inline uint64_t top_p_sum(float p, uint64_t S) {
  return min(max((uint64_t)ceil((double)fmaxf(p, 0.f) * (double)S), (uint64_t)1), S);
}

// Any row: every question by a radix descent over the row in memory
template <int DT>
__device__ __attribute__((noinline)) Drawn sample_general(const Row<DT> row, const RowSettings st,
                                                          Shared<DT>& sh) {
  uint32_t best = 0;
  row.each([&](uint32_t k, int) { best = max(best, k); });
  best = block_max_u32(best, sh);
  if (!(st.T > 0.f) || best == 0u)   // greedy, or a row of NaN
    return {nth_index<DT>(row, best, 0, sh), best ? 1.f : 0.f};
  const Weights w{key_value(best), best, 1.4426950408889634074 / (double)st.T};
  const double least = st.least();
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
  if (st.k > 0 && (uint64_t)st.k < have) {
    // the k-th token's value; its larger ones and the first of its ties are kept
    const Crossing c = find_crossing<DT>(row, w, (uint64_t)(st.k - 1), true, sh);
    uint64_t sum = 0;
    row.each([&](uint32_t key, int) { sum += key > c.key ? w(key) : 0ull; });
    S = block_sum_u64(sum, sh) + ((uint64_t)st.k - c.above) * w(c.key);
  }
  if (st.p < 1.f) {
    const uint64_t P = top_p_sum(st.p, S);
    const Crossing c = find_crossing<DT>(row, w, P - 1, false, sh);
    const uint64_t W = w(c.key);
    S = c.above + ((P - 1 - c.above) / W + 1) * W;
  }
  S = min(S, Sm);
  const uint64_t target = draw_target(st.u, S);
  const Crossing c = find_crossing<DT>(row, w, target, false, sh);
  const uint64_t W = w(c.key);
  return {nth_index<DT>(row, c.key, (uint32_t)((target - c.above) / W), sh),
          (float)((double)W / (double)S)};
}

// ----------------------------------------------------------------------------------
// Passes over a row: its whole aligned 16-byte units, kAhead of them in flight per thread, and
// the elements of its unaligned ends, one per thread.  Places without an element are NaN, which
// no pass counts.  A row is read from HBM once; the passes after the first find it in the
// caches.  (A workgroup's registers would hold a row of 150000 bf16 values, but the passes need
// the rest of them: at every share kept there, the compiler spilled as much.)
constexpr int kAhead = 4;

template <int DT>
struct Passes {
  static constexpr int U = Row<DT>::U;
  static constexpr uint32_t kNone = DT == TAPS_BF16 ? 0x7FC07FC0u : 0x7FC00000u;
  const Row<DT>& row;
  int head, full;      // elements before the first whole unit, whole units

  __device__ inline explicit Passes(const Row<DT>& x) : row(x) {
    head = x.lead ? min(U - x.lead, x.vocab) : 0;
    full = (x.vocab - head) / U;
  }
  // f(unit's 16 bytes, index of its first element); the trip count is the workgroup's
  template <class F>
  __device__ __attribute__((always_inline)) inline void units(F&& f) const {
    const int tid = threadIdx.x;
    const char* const first = row.base + (int64_t)head * (16 / U);
    for (int u0 = 0; u0 < full; u0 += kAhead * kThreads) {
      uint4 x[kAhead];
#pragma unroll
      for (int j = 0; j < kAhead; ++j)
        x[j] = *(const uint4*)(first + (int64_t)min(u0 + j * kThreads + tid, full - 1) * 16);
#pragma unroll
      for (int j = 0; j < kAhead; ++j) {
        const int u = u0 + j * kThreads + tid;
        if (u0 + j * kThreads >= full) break;   // uniform
        if (u >= full) x[j] = make_uint4(kNone, kNone, kNone, kNone);
        f(x[j], u * U + head);
      }
    }
    if (row.vocab != full * U) {
      const int rest = head + full * U;
      int e = -1;
      if (tid < U && tid < head) e = tid;
      if (tid >= U && rest + tid - U < row.vocab) e = rest + tid - U;   // fewer than U of them
      uint32_t b = kNone;
      if (e >= 0)
        b = DT == TAPS_BF16 ? 0x7FC00000u | ((const uint16_t*)row.base)[e]
                            : ((const uint32_t*)row.base)[e];
      f(make_uint4(b, kNone, kNone, kNone), max(e, 0));
    }
  }
  // the largest value (NaN left out; -inf where there is none)
  __device__ __attribute__((always_inline)) inline float max_value() const {
    float mx = -INFINITY;
    units([&](const uint4& w, int) {
      const uint32_t ww[4] = {w.x, w.y, w.z, w.w};
#pragma unroll
      for (int q = 0; q < 4; ++q) {
        if (DT == TAPS_BF16)
          mx = fmaxf(mx, fmaxf(__uint_as_float(ww[q] << 16), __uint_as_float(ww[q] & 0xFFFF0000u)));
        else
          mx = fmaxf(mx, __uint_as_float(ww[q]));
      }
    });
    return mx;
  }
  // f(value, index) for the elements whose value is at least `thr`; units without any are
  // passed over with two instructions per element
  template <class F>
  __device__ __attribute__((always_inline)) inline void at_least(float thr, F&& f) const {
    units([&](const uint4& w, int e0) {
      const uint32_t ww[4] = {w.x, w.y, w.z, w.w};
      bool any = false;
#pragma unroll
      for (int q = 0; q < 4; ++q) {
        if (DT == TAPS_BF16)
          any |= __uint_as_float(ww[q] << 16) >= thr || __uint_as_float(ww[q] & 0xFFFF0000u) >= thr;
        else
          any |= __uint_as_float(ww[q]) >= thr;
      }
      if (!any) return;
#pragma unroll
      for (int q = 0; q < U; ++q) {
        const uint32_t b = DT == TAPS_BF16
                               ? ((q & 1) ? ww[q >> 1] & 0xFFFF0000u : ww[q >> 1] << 16)
                               : ww[q & 3];
        const float x = __uint_as_float(b);
        if (x >= thr) f(x, e0 + q);
      }
    });
  }
};

__device__ inline uint64_t wave_scan_u64(uint64_t v) {
  const int lane = threadIdx.x & (kWave - 1);
#pragma unroll
  for (int d = 1; d < kWave; d <<= 1) {
    const uint32_t lo = __shfl_up((uint32_t)v, d), hi = __shfl_up((uint32_t)(v >> 32), d);
    if (lane >= d) v += ((uint64_t)hi << 32) | lo;
  }
  return v;
}
__device__ inline uint32_t wave_scan_u32(uint32_t v) {
  const int lane = threadIdx.x & (kWave - 1);
#pragma unroll
  for (int d = 1; d < kWave; d <<= 1) {
    const uint32_t o = __shfl_up(v, d);
    if (lane >= d) v += o;
  }
  return v;
}
__device__ inline uint64_t shfl_u64(uint64_t v, int lane) {
  const uint32_t lo = __shfl((uint32_t)v, lane), hi = __shfl((uint32_t)(v >> 32), lane);
  return ((uint64_t)hi << 32) | lo;
}

template <int DT>
__device__ inline uint64_t block_scan_u64(uint64_t v, Shared<DT>& sh, uint64_t* total) {
  const int lane = threadIdx.x & (kWave - 1), wave = threadIdx.x / kWave;
  v = wave_scan_u64(v);
  __syncthreads();
  if (lane == kWave - 1) sh.red[wave] = v;
  __syncthreads();
  uint64_t before = 0, all = 0;
#pragma unroll
  for (int w = 0; w < kWaves; ++w) {
    if (w < wave) before += sh.red[w];
    all += sh.red[w];
  }
  *total = all;
  return v + before;
}

template <int DT>
__device__ inline float block_max_f32(float v, Shared<DT>& sh) {
#pragma unroll
  for (int m = 32; m >= 1; m >>= 1) v = fmaxf(v, __shfl_xor(v, m));
  const int lane = threadIdx.x & (kWave - 1), wave = threadIdx.x / kWave;
  __syncthreads();
  if (lane == 0) sh.red32[wave] = __float_as_uint(v);
  __syncthreads();
#pragma unroll
  for (int w = 0; w < kWaves; ++w) v = fmaxf(v, __uint_as_float(sh.red32[w]));
  return v;
}

// A key that at least k elements reach: the k-th largest of the maxima of groups of four
// threads (0 where fewer groups hold a value).  k <= kFewTopK.
template <int DT>
__device__ inline uint32_t top_k_bound(float mx, int k, Shared<DT>& sh) {
  const int tid = threadIdx.x, lane = tid & (kWave - 1);
  uint32_t key = mx > -INFINITY ? value_key(__float_as_uint(mx)) : 0u;
  key = max(key, (uint32_t)__shfl_xor(key, 1));
  key = max(key, (uint32_t)__shfl_xor(key, 2));
  if ((tid & 3) == 0) sh.group[tid >> 2] = key;
  __syncthreads();
  uint32_t g[kGroups / kWave];
#pragma unroll
  for (int i = 0; i < kGroups / kWave; ++i) g[i] = sh.group[i * kWave + lane];
  uint32_t T = 0;
  for (int bit = 31; bit >= (DT == TAPS_BF16 ? 16 : 0); --bit) {
    const uint32_t c = T | (1u << bit);
    int n = 0;
#pragma unroll
    for (int i = 0; i < kGroups / kWave; ++i) n += __popcll(__ballot(g[i] >= c));
    if (n >= k) T = c;
  }
  return T;
}

// The nth (from 0) in index order of the `ties` elements equal to `value`
template <int DT>
__device__ __attribute__((always_inline)) inline int nth_equal(const Passes<DT>& passes, float value, uint32_t nth, uint32_t ties,
                                Shared<DT>& sh) {
  if (ties > (uint32_t)kList)
    return nth_index<DT>(passes.row, value_key(__float_as_uint(value)), nth, sh);
  if (threadIdx.x == 0) sh.n = 0u;
  __syncthreads();
  passes.units([&](const uint4& w, int e0) {
    const uint32_t ww[4] = {w.x, w.y, w.z, w.w};
    bool any = false;
#pragma unroll
    for (int q = 0; q < 4; ++q) {
      if (DT == TAPS_BF16)
        any |= __uint_as_float(ww[q] << 16) == value || __uint_as_float(ww[q] & 0xFFFF0000u) == value;
      else
        any |= __uint_as_float(ww[q]) == value;
    }
    if (!any) return;
#pragma unroll
    for (int q = 0; q < Passes<DT>::U; ++q) {
      const uint32_t b = DT == TAPS_BF16 ? ((q & 1) ? ww[q >> 1] & 0xFFFF0000u : ww[q >> 1] << 16)
                                         : ww[q & 3];
      if (__uint_as_float(b) == value) sh.ties[atomicAdd(&sh.n, 1u)] = (uint32_t)(e0 + q);
    }
  });
  __syncthreads();
  const uint32_t n = sh.n;
  for (uint32_t i = threadIdx.x; i < n; i += kThreads) {
    const uint32_t mine = sh.ties[i];
    uint32_t before = 0;
    for (uint32_t j = 0; j < n; ++j) before += sh.ties[j] < mine ? 1u : 0u;
    if (before == nth) sh.out32[3] = mine;
  }
  __syncthreads();
  return (int)sh.out32[3];
}

// ----------------------------------------------------------------------------------
// bf16: a row holds few distinct values, so the elements are counted by value (16-bit keys from
// the largest down, as far as weights reach) and every sum is over values: one exponential per
// value that occurs, none per element, and a crossing is exact at once.
// Returns false where the window is too wide (or nothing exceeds -inf): the general path's.
constexpr uint32_t kLowest16 = 0x007Fu;   // the key of -inf; smaller ones are NaN
__device__ inline uint32_t key16(float x) { return value_key(__float_as_uint(x)) >> 16; }

template <int DT>
__device__ __attribute__((always_inline)) inline bool sample_counted(const Passes<DT>& passes, float mx_thread, float M,
                                      const RowSettings& st, Shared<DT>& sh, Drawn* out) {
  const int tid = threadIdx.x, lane = tid & (kWave - 1), wave = tid / kWave;
  const uint32_t kM = key16(M);
  CountScratch& cs = sh.u.c;
  const Weights w{M, value_key(__float_as_uint(M)), 1.4426950408889634074 / (double)st.T};
  // values that can have a weight, and that the filters can keep (a little more never hurts:
  // the bounds are rounded to bf16, so two more keys)
  const double least = st.least();
  const double reach = st.cut_by_min_p() ? fmax(least, -44.5) : -44.5;
  const float low = (float)((double)M + reach / w.scale);
  uint32_t klow = low > -INFINITY ? key16(low) : 0u;
  klow = klow > kLowest16 + 2u ? klow - 2u : kLowest16;
  if (st.few()) klow = max(klow, top_k_bound<DT>(mx_thread, st.k, sh) >> 16);
  if (klow == 0x8000u) klow = 0x7FFFu;   // +0 and -0 are equal
  klow = min(klow, kM);
  const uint32_t Wn = kM - klow + 1u;
  if (Wn > (uint32_t)kWindow) return false;
  for (uint32_t i = tid; i < (Wn + kWave - 1) / kWave * kWave; i += kThreads) cs.count[i] = 0u;
  __syncthreads();
  if (st.few() || st.cut_by_min_p()) {
    // few elements: compare first.  The value of the lowest key
    const float thr = __uint_as_float((klow & 0x8000u) ? (klow & 0x7FFFu) << 16 : (~klow & 0xFFFFu) << 16);
    passes.at_least(thr, [&](float x, int) {
      const uint32_t i = kM - key16(x);
      if (i < Wn) atomicAdd(&cs.count[i], 1u);
    });
  } else {
    passes.units([&](const uint4& v, int) {
      const uint32_t ww[4] = {v.x, v.y, v.z, v.w};
      typedef short s16x2 __attribute__((ext_vector_type(2)));
      typedef unsigned short u16x2 __attribute__((ext_vector_type(2)));
      const u16x2 top = {(unsigned short)kM, (unsigned short)kM};
#pragma unroll
      for (int q = 0; q < 4; ++q) {
        // both halves: key = sign ? ~bits : bits | 0x8000; NaN keys fall outside the window
        const s16x2 b = __builtin_bit_cast(s16x2, ww[q]);
        const uint32_t sign = __builtin_bit_cast(uint32_t, (s16x2)(b >> 15));
        const u16x2 key = __builtin_bit_cast(u16x2, ww[q] ^ (sign | 0x80008000u));
        const uint32_t idx = __builtin_bit_cast(uint32_t, (u16x2)(top - key));
        const uint32_t i0 = idx & 0xFFFFu, i1 = idx >> 16;
        if (i0 < Wn) atomicAdd(&cs.count[i0], 1u);
        if (i1 < Wn) atomicAdd(&cs.count[i1], 1u);
      }
    });
  }
  __syncthreads();
  if (tid == 0 && kM >= 0x8000u) {   // -0 counts as +0
    const uint32_t z = kM - 0x8000u;
    if (z + 1u < Wn) {
      cs.count[z] += cs.count[z + 1u];
      cs.count[z + 1u] = 0u;
    }
  }
  __syncthreads();

  // weight of the value at window position i
  auto weight = [&](uint32_t i) -> uint64_t {
    const uint32_t k = kM - i;   // 16 bits; the value's full key
    return w((k << 16) | ((k & 0x8000u) ? 0u : 0xFFFFu));
  };
  const int rows = (int)((Wn + kWave - 1) / kWave);
  for (int r = wave; r < rows; r += kWaves) {
    const uint32_t c = cs.count[r * kWave + lane];
    uint64_t m = 0;
    uint32_t n = 0;
    if (__ballot(c != 0u)) {
      m = c ? (uint64_t)c * weight(r * kWave + lane) : 0ull;
      m = wave_sum_u64(m);
      n = c;
#pragma unroll
      for (int d = 32; d >= 1; d >>= 1) n += __shfl_xor(n, d);
    }
    if (lane == 0) cs.mass[r] = m, cs.num[r] = n;
  }
  __syncthreads();
  uint64_t S, have;
  {
    const uint64_t m = tid < rows ? cs.mass[tid] : 0ull;
    const uint64_t n = tid < rows ? cs.num[tid] : 0ull;
    const uint64_t pm = block_scan_u64(m, sh, &S) - m, pn = block_scan_u64(n, sh, &have) - n;
    if (tid < rows) cs.mass[tid] = pm, cs.num[tid] = (uint32_t)pn;
  }
  __syncthreads();

  struct Cross {
    uint32_t pos, ties, nth;     // window position, elements there, the crossing one among them
    uint64_t above, W;           // sum (count) before them, weight of each
  };
  // where the running sum (count) first exceeds target
  auto crossing = [&](uint64_t target, bool by_count) -> Cross {
    if (tid < rows) {
      const uint64_t a = by_count ? cs.num[tid] : cs.mass[tid];
      const uint64_t b = tid + 1 < rows ? (by_count ? cs.num[tid + 1] : cs.mass[tid + 1])
                                        : (by_count ? have : S);
      if (a <= target && target < b) sh.out32[0] = (uint32_t)tid;
    }
    __syncthreads();
    const int r = (int)sh.out32[0];
    __syncthreads();
    const uint32_t i = (uint32_t)(r * kWave + lane), c = cs.count[i];
    const uint64_t W = c ? weight(i) : 0ull;
    const uint64_t m = by_count ? (uint64_t)c : (uint64_t)c * W;
    const uint64_t incl = (by_count ? (uint64_t)cs.num[r] : cs.mass[r]) + wave_scan_u64(m);
    const int l = __ffsll((long long)__ballot(incl > target)) - 1;
    Cross x;
    x.pos = (uint32_t)(r * kWave + l);
    x.ties = __shfl(c, l);
    x.W = shfl_u64(W, l);
    x.above = shfl_u64(incl - m, l);
    x.nth = by_count ? (uint32_t)(target - x.above) : (uint32_t)((target - x.above) / x.W);
    return x;
  };
  // sum of the weights before window position i
  auto sum_before = [&](uint32_t i) -> uint64_t {
    const int r = (int)(i / kWave);
    const uint32_t at = (uint32_t)(r * kWave + lane), c = cs.count[at];
    const uint64_t m = c && at < i ? (uint64_t)c * weight(at) : 0ull;
    return cs.mass[r] + wave_sum_u64(m);
  };

  uint64_t kept = S;
  if (st.k > 0 && (uint64_t)st.k < have) {
    const Cross c = crossing((uint64_t)(st.k - 1), true);
    kept = sum_before(c.pos) + (uint64_t)(c.nth + 1u) * c.W;
  }
  if (st.p < 1.f) {
    const Cross c = crossing(top_p_sum(st.p, kept) - 1, false);
    kept = c.above + (uint64_t)(c.nth + 1u) * c.W;
  }
  if (st.mp > 0.f) {
    uint32_t lo = 0, hi = Wn;   // positions below lo are kept, those from hi on are not
    while (hi - lo > 1u) {
      const uint32_t mid = (lo + hi) / 2u, k = kM - mid;
      if (w.log2w((k << 16) | ((k & 0x8000u) ? 0u : 0xFFFFu)) >= least) lo = mid;
      else hi = mid;
    }
    if (hi < Wn) kept = min(kept, sum_before(hi));
  }
  const Cross c = crossing(draw_target(st.u, kept), false);
  const uint32_t k = kM - c.pos;
  out->token = nth_equal<DT>(
      passes, __uint_as_float((k & 0x8000u) ? (k & 0x7FFFu) << 16 : (~k & 0xFFFFu) << 16), c.nth,
      c.ties, sh);
  out->prob = (float)((double)c.W / (double)kept);
  return true;
}

// ----------------------------------------------------------------------------------
// fp32, few candidates (a small top_k, or min_p): the elements above a bound, ranked one by
// one.  False: more than kList of them.
template <int DT>
__device__ inline void sort_list(uint32_t n, Shared<DT>& sh) {
  BinScratch& bs = sh.u.b;
  const uint32_t i = threadIdx.x;
  if (i < n) {
    const uint64_t mine = bs.list[i];
    uint32_t rank = 0;
    for (uint32_t j = 0; j < n; ++j) rank += bs.list[j] > mine ? 1u : 0u;
    bs.sorted[rank] = mine;
  }
  __syncthreads();
}

// the first position of cum[0 .. n) that exceeds target (one does)
template <int DT>
__device__ inline uint32_t first_above(uint64_t target, uint32_t n, Shared<DT>& sh) {
  const BinScratch& bs = sh.u.b;
  const uint32_t i = threadIdx.x;
  if (i < n && bs.cum[i] > target && (i == 0 || bs.cum[i - 1] <= target)) sh.out32[1] = i;
  __syncthreads();
  const uint32_t r = sh.out32[1];
  __syncthreads();
  return r;
}

template <int DT>
__device__ __attribute__((always_inline)) inline bool sample_listed(const Passes<DT>& passes, float mx_thread, float M,
                                     const RowSettings& st, Shared<DT>& sh, Drawn* out) {
  const int tid = threadIdx.x;
  BinScratch& bs = sh.u.b;
  const Weights w{M, value_key(__float_as_uint(M)), 1.4426950408889634074 / (double)st.T};
  const double least = st.least();
  float thr = -INFINITY;
  if (st.cut_by_min_p()) {   // rounded down by more than the arithmetic can be off
    const double low = (double)M + least / w.scale;
    thr = (float)(low - 1e-6 * (fabs(low) + fabs((double)M)));
    if (thr != thr) thr = M;   // an infinite maximum
  }
  if (st.few()) {
    const uint32_t key = top_k_bound<DT>(mx_thread, st.k, sh);
    if (key) thr = fmaxf(thr, key_value(key));
  }
  if (tid == 0) sh.n = 0u;
  __syncthreads();
  passes.at_least(thr, [&](float x, int e) {
    const uint32_t i = atomicAdd(&sh.n, 1u);
    if (i < (uint32_t)kList) bs.list[i] = cand_key(value_key(__float_as_uint(x)), (uint32_t)e);
  });
  __syncthreads();
  const uint32_t n = sh.n;
  if (n > (uint32_t)kList) return false;
  sort_list<DT>(n, sh);
  const uint32_t key = (uint32_t)tid < n ? (uint32_t)(bs.sorted[tid] >> 32) : 0u;
  const uint64_t W = key ? w(key) : 0ull;
  uint64_t all;
  const uint64_t cum = block_scan_u64(W, sh, &all);
  if ((uint32_t)tid < n) bs.cum[tid] = cum;
  uint64_t Sm = block_sum_u64(key && w.log2w(key) >= least ? W : 0ull, sh);   // also a barrier
  uint64_t S = st.k > 0 && (uint32_t)st.k < n ? bs.cum[st.k - 1] : all;
  if (st.p < 1.f) S = bs.cum[first_above<DT>(top_p_sum(st.p, S) - 1, n, sh)];
  S = min(S, Sm);
  const uint32_t r = first_above<DT>(draw_target(st.u, S), n, sh);
  out->token = (int)cand_index(bs.sorted[r]);
  out->prob = (float)((double)(bs.cum[r] - (r ? bs.cum[r - 1] : 0ull)) / (double)S);
  return true;
}

// fp32, the whole vocabulary's sum (top_p or no filter): weights are added up by bins of 1/32
// octave.  Weight 2^-(z / 32), z = 32 log2(e) (M - x) / T, is the bin's 2^-(b / 32), b = floor z,
// times a factor 2^-((z - b) / 32) from a short series; a bin adds up its factors (integers of
// 2^-43), and its sum is that times 2^-(b / 32), rounded down.  The bin where a running sum passes its
// target is then ranked one by one.  False: more than kList elements in it.
template <int DT>
__device__ __attribute__((always_inline)) inline bool sample_binned(const Passes<DT>& passes, float M, const RowSettings& st,
                                     Shared<DT>& sh, Drawn* out) {
  const int tid = threadIdx.x;
  BinScratch& bs = sh.u.b;
  const double scale = kPerOctave * 1.4426950408889634074 / (double)st.T;
  for (int i = tid; i < kWeightBins; i += kThreads) bs.mass[i] = 0ull;
  __syncthreads();
  auto depth = [&](float x) -> double { return x == M ? 0.0 : ((double)M - (double)x) * scale; };
  // the factor in units of 2^-43
  auto factor = [&](double z, int b) -> uint64_t {
    const double t = (z - (double)b) * (-0.69314718055994530942 / kPerOctave);
    double p = 1.0 / 720.0;
    p = fma(p, t, 1.0 / 120.0);
    p = fma(p, t, 1.0 / 24.0);
    p = fma(p, t, 1.0 / 6.0);
    p = fma(p, t, 0.5);
    p = fma(p, t, 1.0);
    p = fma(p, t, 1.0);
    // the sum with 512 has steps of 2^-43: its low bits are the rounded integer
    return (uint64_t)(__double_as_longlong(p + 512.0) - __double_as_longlong(512.0));
  };
  passes.units([&](const uint4& v, int) {
    const uint32_t ww[4] = {v.x, v.y, v.z, v.w};
#pragma unroll
    for (int q = 0; q < 4; ++q) {
      const double z = depth(__uint_as_float(ww[q]));
      if (z < (double)kWeightBins) {
        const int b = (int)z;
        atomicAdd((unsigned long long*)&bs.mass[b], (unsigned long long)factor(z, b));
      }
    }
  });
  __syncthreads();
  auto bin_scale = [&](int b) -> double { return exp2_neg(-(double)b / kPerOctave); };
  uint64_t S;
  {
    const int b0 = 2 * tid;
    uint64_t m0 = 0, m1 = 0;
    if (b0 < kWeightBins) {
      m0 = (uint64_t)(bin_scale(b0) * (double)bs.mass[b0]);
      m1 = (uint64_t)(bin_scale(b0 + 1) * (double)bs.mass[b0 + 1]);
    }
    const uint64_t incl = block_scan_u64(m0 + m1, sh, &S);
    if (b0 < kWeightBins) bs.before[b0] = incl - m0 - m1, bs.before[b0 + 1] = incl - m1;
  }
  __syncthreads();
  static_assert(kWeightBins % 2 == 0 && kWeightBins <= 2 * kThreads, "two bins per thread");

  // Ranks the elements of a bin: sorted[], and the running sums with each of them in cum[].
  // Returns their number; above kList nothing is ranked.
  auto rank_bin = [&](int bin) -> uint32_t {
    if (tid == 0) sh.n = 0u;
    __syncthreads();
    passes.units([&](const uint4& v, int e0) {
      const uint32_t ww[4] = {v.x, v.y, v.z, v.w};
#pragma unroll
      for (int q = 0; q < 4; ++q) {
        const double z = depth(__uint_as_float(ww[q]));
        if (z >= (double)bin && z < (double)(bin + 1)) {
          const uint32_t i = atomicAdd(&sh.n, 1u);
          if (i < (uint32_t)kList) bs.list[i] = cand_key(value_key(ww[q]), (uint32_t)(e0 + q));
        }
      }
    });
    __syncthreads();
    const uint32_t n = sh.n;
    if (n > (uint32_t)kList) return n;
    sort_list<DT>(n, sh);
    uint64_t f = 0;
    if ((uint32_t)tid < n) f = factor(depth(key_value((uint32_t)(bs.sorted[tid] >> 32))), bin);
    uint64_t all;
    const uint64_t cum = block_scan_u64(f, sh, &all);
    if ((uint32_t)tid < n) bs.cum[tid] = bs.before[bin] + (uint64_t)(bin_scale(bin) * (double)cum);
    __syncthreads();
    return n;
  };
  // the bin where the running sum first exceeds target
  auto bin_of = [&](uint64_t target) -> int {
    for (int b = tid; b < kWeightBins; b += kThreads) {
      const uint64_t hi = b + 1 < kWeightBins ? bs.before[b + 1] : S;
      if (bs.before[b] <= target && target < hi) sh.out32[0] = (uint32_t)b;
    }
    __syncthreads();
    return (int)sh.out32[0];
  };
  uint64_t kept = S;
  if (st.p < 1.f) {
    const uint64_t target = top_p_sum(st.p, S) - 1;
    const uint32_t n = rank_bin(bin_of(target));
    if (n > (uint32_t)kList) return false;
    kept = bs.cum[first_above<DT>(target, n, sh)];
  }
  if (st.mp > 0.f) {
    const double last = -kPerOctave * st.least();   // the depth down to which tokens are kept
    if (last < (double)kWeightBins) {
      const uint32_t n = rank_bin((int)last);
      if (n > (uint32_t)kList) return false;
      // kept ones of the bin come first; without any, all before it
      bool in = false;
      if ((uint32_t)tid < n) in = depth(key_value((uint32_t)(bs.sorted[tid] >> 32))) <= last;
      const uint32_t num = (uint32_t)block_sum_u64(in ? 1ull : 0ull, sh);
      kept = min(kept, num ? bs.cum[num - 1] : bs.before[(int)last]);
      __syncthreads();
    }
  }
  const uint64_t target = draw_target(st.u, kept);
  const int bin = bin_of(target);
  const uint32_t n = rank_bin(bin);
  if (n > (uint32_t)kList) return false;
  const uint64_t key = bs.sorted[first_above<DT>(target, n, sh)];
  out->token = (int)cand_index(key);
  out->prob = (float)(bin_scale(bin) *
                      (double)factor(depth(key_value((uint32_t)(key >> 32))), bin) / (double)kept);
  return true;
}

template <int DT>
__global__ __launch_bounds__(kThreads) void sample_kernel(
    const void* __restrict__ logits, int64_t row_bytes, int budget, int vocab,
    const int32_t* __restrict__ n_nodes, const Settings s, const float* __restrict__ u,
    int32_t* __restrict__ tokens, float* __restrict__ probs) {
  __shared__ Shared<DT> sh;
  const int r = blockIdx.x, b = r / budget, tid = threadIdx.x;
  if (n_nodes && r - b * budget >= n_nodes[b]) {
    if (tid == 0) {
      tokens[r] = -1;
      if (probs) probs[r] = 0.f;
    }
    return;
  }
  const Row<DT> row((const char*)logits + (size_t)r * row_bytes, vocab);
  const Passes<DT> passes(row);
  RowSettings st;
  st.T = s.temperature ? s.temperature[b] : 1.f;
  st.k = s.top_k ? s.top_k[b] : 0;
  st.p = s.top_p ? s.top_p[b] : 1.f;
  st.mp = s.min_p ? s.min_p[b] : 0.f;
  st.u = u[r];
  const float mx = passes.max_value();
  float M = block_max_f32(mx, sh);
  if (M == 0.f) M = 0.f;   // not -0
  Drawn d;
  bool done = false;
  if (M > -INFINITY) {
    if (!(st.T > 0.f)) {
      if (tid == 0) sh.n = 0xFFFFFFFFu;
      __syncthreads();
      passes.at_least(M, [&](float, int e) { atomicMin(&sh.n, (uint32_t)e); });
      __syncthreads();
      d = {(int)sh.n, 1.f};
      done = true;
    } else if constexpr (DT == TAPS_BF16) {
      done = sample_counted<DT>(passes, mx, M, st, sh, &d);
    } else if (st.few() || st.cut_by_min_p()) {
      done = sample_listed<DT>(passes, mx, M, st, sh, &d);
    } else if (st.k <= 0 || st.k >= vocab) {
      done = sample_binned<DT>(passes, M, st, sh, &d);
    }
  }
  if (!done) {   // uniform
    __syncthreads();
    d = sample_general<DT>(row, st, sh);
  }
  if (tid == 0) {
    tokens[r] = d.token;
    if (probs) probs[r] = d.prob;
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

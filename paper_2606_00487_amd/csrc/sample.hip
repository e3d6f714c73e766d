// Token sampling with temperature, top-k, top-p and min-p from given random numbers
// (taps_sample).
//
// A row's tokens in rank order (value descending, index ascending, NaN last) have weights
//   W_r = 2^43 exp((x_r - x_0) / T),
// added up as integers: a sum does not depend on the order in which a kernel adds (atomics
// included), and 2^20 weights stay below 2^64.  top-k, top-p and min-p each keep a prefix of the
// rank order, so the sum S over the kept set is the smallest of the prefixes' sums
//   S_k = sum over the first top_k,   S_p = the first sum that reaches top_p * S_k,
//   S_m = sum over weights >= min_p,
// and the token is the first whose running sum exceeds floor(u S).  Each of these is one
// question: at which token does the running count or sum in rank order pass a target?
//
// One workgroup per row, by one of four paths:
//   sample_listed   a small top_k, or min_p without top_p: the elements above a bound that the
//                   thread groups' largest values (or min_p) give, ranked one by one;
//   sample_counted  bf16 otherwise: the elements counted by value;
//   sample_binned   fp32 otherwise: weights added up by bins of 1/32 octave, the bin that a
//                   question leads to ranked;
//   sample_general  what those decline (thousands of equal bf16 values past 16-bit counts, an
//                   infinite temperature or fp32 maximum, fp32 rows too dense to bin): a radix
//                   descent over the row for each question.
// Bound: reading the row where nothing is added up for every element (2048 rows x 151936 bf16,
// top_k 40: 134 us; their bytes at 5.8 TB/s take 107); the LDS additions beside it otherwise (no
// filter 191, top_p 190; 64 additions of 32 bits take 12 clocks of a CU, of 64 bits 20); for few
// rows the chain of about twenty barriers with small work between them (16 rows x 1000: 10 to 15
// us).  A small top_k over a row whose finite values (a mask leaves the others -inf) are in fewer
// thread groups than that finds no bound, and the row is read three times (2048 rows, top_k 40 of
// 40 finite values: 334 us; top_k 20: 131).  Two workgroups a CU where there are rows for that: one's questions beside the other's
// reading.  Rows shared out over several workgroups, with a second kernel for the questions, took
// longer even for 32 rows (33 against 29 us).
#include "common.h"
#include "scan.h"

namespace taps {

namespace {

// 2^y for -45 <= y <= 0: y = k + r, |r| <= 1/2, e^(r ln 2) by its Taylor series to the 12th power
// (remainder below 2^-52), exact at y = 0.
// (The coefficients are pinned to scalar registers: from vector ones every product copied its own.)
__device__ inline double scalar(double c) {
  asm("" : "+s"(c));
  return c;
}
__device__ inline double exp2_neg(double y) {
  const double k = rint(y);
  const double t = (y - k) * 0.69314718055994530942;
  double p = 1.0 / 479001600.0;
  p = fma(p, t, scalar(1.0 / 39916800.0));
  p = fma(p, t, scalar(1.0 / 3628800.0));
  p = fma(p, t, scalar(1.0 / 362880.0));
  p = fma(p, t, scalar(1.0 / 40320.0));
  p = fma(p, t, scalar(1.0 / 5040.0));
  p = fma(p, t, scalar(1.0 / 720.0));
  p = fma(p, t, scalar(1.0 / 120.0));
  p = fma(p, t, scalar(1.0 / 24.0));
  p = fma(p, t, scalar(1.0 / 6.0));
  p = fma(p, t, 0.5);
  p = fma(p, t, 1.0);
  p = fma(p, t, 1.0);
  return ldexp(p, (int)k);
}
// x in [0, 1] in units of 2^-43, rounded: doubles between 512 and 1024 have steps of 2^-43, so
// the low bits of 512 + x are that integer
__device__ inline uint64_t fixed43(double x512) {
  return (uint64_t)(__double_as_longlong(x512) - __double_as_longlong(512.0));
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
  // (no branch: several weights of a thread are evaluated side by side; NaN counts as -45)
  __device__ inline uint64_t operator()(uint32_t k) const {
    return fixed43(512.0 + exp2_neg(fmax(log2w(k), -45.0)));
  }
};

__device__ inline uint64_t wave_sum_u64(uint64_t v) {
  return lane_u64(wave_scan_u64(v), kWave - 1);
}
// the same over rows of 16 lanes
__device__ inline uint32_t row_scan_u32(uint32_t x) {
  int v = (int)x;
  v += __builtin_amdgcn_update_dpp(0, v, 0x111, 0xf, 0xf, false);
  v += __builtin_amdgcn_update_dpp(0, v, 0x112, 0xf, 0xf, false);
  v += __builtin_amdgcn_update_dpp(0, v, 0x114, 0xf, 0xf, false);
  v += __builtin_amdgcn_update_dpp(0, v, 0x118, 0xf, 0xf, false);
  return (uint32_t)v;
}
__device__ inline uint64_t row_scan_u64(uint64_t v) {
  const uint32_t a = row_scan_u32((uint32_t)v & 0x3FFFFFu);
  const uint32_t b = row_scan_u32((uint32_t)(v >> 22) & 0x3FFFFFu);
  const uint32_t c = row_scan_u32((uint32_t)(v >> 44));
  return (uint64_t)a + ((uint64_t)b << 22) + ((uint64_t)c << 44);
}
// maximum over the lanes, in the last one (a lane without a source compares with itself)
template <int CTRL, int ROWS>
__device__ inline float dpp_max(float v) {
  const int x = (int)__float_as_uint(v);
  return fmaxf(v, __uint_as_float((uint32_t)__builtin_amdgcn_update_dpp(x, x, CTRL, ROWS, 0xf, false)));
}
__device__ inline float row_max_f32(float v) {
  v = dpp_max<0x111, 0xf>(v);
  v = dpp_max<0x112, 0xf>(v);
  v = dpp_max<0x114, 0xf>(v);
  return dpp_max<0x118, 0xf>(v);
}
__device__ inline float lane_f32(float v, int lane) {
  return __uint_as_float(__builtin_amdgcn_readlane(__float_as_uint(v), lane));
}

constexpr int kBins = 2048;         // radix digits of the general path
constexpr int kWindow = 36864;      // bf16 values counted one by one, from the largest down
constexpr int kRun = 256;           // values whose sums are kept together: four per lane
constexpr int kRuns = kWindow / kRun;
constexpr int kPerOctave = 32;      // fp32: bins of the weight per factor of two
constexpr int kOctaves = 44;        // smaller weights round to 0: at most half of 2^-43
constexpr int kWeightBins = kOctaves * kPerOctave + 1;   // the last one's upper half lies below
constexpr int kSub = 1024;          // parts of a bin with more elements than the list takes
constexpr int kList = 1024;         // elements that are ranked one by one
constexpr int kGroups = 256;        // thread groups whose maxima bound a small top_k
// ... up to this one.  us with top_k 192 / 193: 512 rows of 151,936 fp32 100 / 140, 32 of 50,257 17 /
// 26, 64 of 151,936 bf16 22 / 28; 2048 of those 185 / 164 (148 with 100, 165 with 150).
constexpr int kFewTopK = 192;

// Scratch of the paths, which a row takes one after the other at most
struct GeneralScratch {
  uint64_t mass[kBins];
  uint32_t count[kBins];
};
struct alignas(16) ListScratch {
  uint64_t list[kList], sorted[kList], cum[kList];
};
// (the elements outside a histogram are added too, into a word per lane behind it: a branch for
// each element costs more, and one word for all of them would take them one by one)
struct CountScratch {
  uint32_t count[kWindow / 2 + kWave];   // elements per value, 16 bits each, the largest first
  uint64_t mass[kRuns];             // sums of the runs; then those before them
  uint32_t num[kRuns];
};
struct BinScratch {
  ListScratch l;
  uint64_t mass[kWeightBins + kWave];   // sums of the bins; then those before them
  uint32_t num[kWeightBins + kWave];    // elements, the same way
  uint64_t sub[kSub];
  uint32_t sub_num[kSub];
};
template <int DT>
union PathScratch {
  GeneralScratch g;
  ListScratch l;
  CountScratch c;
};
template <>
union PathScratch<TAPS_FP32> {
  GeneralScratch g;
  ListScratch l;
  BinScratch b;
};

template <int DT, int NT>
struct Shared {
  PathScratch<DT> u;
  uint32_t group[kGroups];
  uint64_t red[NT / kWave];
  uint32_t red32[NT / kWave], other32[NT / kWave];
  uint64_t out64[2];
  uint32_t out32[4];
  uint32_t n, n_hot;
  uint16_t hot[4 * NT];
};

// Over the workgroup: each wave's sum through LDS, one read per wave and a scan over its lanes
// (every wave adding up all of them: 16 reads each, a microsecond of LDS time a call).
template <class S, int NT>
__device__ inline uint64_t block_scan_u64(uint64_t v, S& sh, uint64_t* total) {
  constexpr int kWaves = NT / kWave;
  static_assert(kWaves <= 16 && (kWaves & (kWaves - 1)) == 0, "one row of lanes holds the waves");
  const int lane = threadIdx.x & (kWave - 1);
  const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x / kWave);
  v = wave_scan_u64(v);
  __syncthreads();
  if (lane == kWave - 1) sh.red[wave] = v;
  __syncthreads();
  const uint64_t x = sh.red[lane & (kWaves - 1)], incl = row_scan_u64(x);
  *total = lane_u64(incl, kWaves - 1);
  return v + lane_u64(incl - x, wave);
}

template <class S, int NT>
__device__ inline uint64_t block_sum_u64(uint64_t v, S& sh) {
  uint64_t total;
  block_scan_u64<S, NT>(v, sh, &total);
  return total;
}

template <class S, int NT>
__device__ inline float block_max_f32(float v, S& sh) {
  constexpr int kWaves = NT / kWave;
  v = row_max_f32(v);
  v = dpp_max<0x142, 0xa>(v);
  v = dpp_max<0x143, 0xc>(v);
  const int lane = threadIdx.x & (kWave - 1), wave = threadIdx.x / kWave;
  __syncthreads();
  if (lane == kWave - 1) sh.red32[wave] = __float_as_uint(v);
  __syncthreads();
  return lane_f32(row_max_f32(__uint_as_float(sh.red32[lane & (kWaves - 1)])), kWaves - 1);
}

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
  template <int NT, class F>
  __device__ inline void each(F&& f) const {
    for (int u = threadIdx.x; u < units; u += NT) unit(u, f);
  }
};

// Where the running sum of the weights (or, with `by_count`, the count) in rank order first
// exceeds `target`: the value's key, the sum and the count above it, and its ties.  `target` is
// below the whole sum (count).  Radix descent over the key, 11 + 11 + 10 bits from the top (the
// 16 bits that bf16 keys have: 11 + 5).
struct Crossing {
  uint32_t key;
  uint64_t above;    // sum (count) of the elements whose key is larger
  uint32_t ties;     // elements with this key
};

template <int DT, int NT>
__device__ Crossing find_crossing(const Row<DT>& row, const Weights& w, uint64_t target,
                                  bool by_count, Shared<DT, NT>& sh) {
  const int tid = threadIdx.x;
  uint32_t prefix = 0;
  uint64_t above = 0;
  uint32_t ties = 0;
  int low = 32;
  while (low > (DT == TAPS_BF16 ? 16 : 0)) {
    const int bits = low == 10 ? 10 : (DT == TAPS_BF16 && low == 21 ? 5 : 11);
    const int high = low;
    low -= bits;
    for (int i = tid; i < kBins; i += NT) sh.u.g.mass[i] = 0ull, sh.u.g.count[i] = 0u;
    __syncthreads();
    row.template each<NT>([&](uint32_t k, int) {
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
        const uint64_t incl = wave_scan_u64(m);
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
        acc += lane_u64(incl, kWave - 1);
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
template <int DT, int NT>
__device__ __attribute__((noinline)) int nth_index(const Row<DT>& row, uint32_t key, uint32_t nth, Shared<DT, NT>& sh) {
  const int tid = threadIdx.x, lane = tid & (kWave - 1), wave = tid / kWave;
  uint32_t seen = 0;
  for (int u0 = 0; u0 < row.units; u0 += NT) {
    uint32_t n = 0;
    if (u0 + tid < row.units) row.unit(u0 + tid, [&](uint32_t k, int) { n += k == key ? 1u : 0u; });
    const uint32_t incl = wave_scan_u32(n);
    __syncthreads();
    if (lane == kWave - 1) sh.red32[wave] = incl;
    __syncthreads();
    uint32_t before = seen, all = 0;
#pragma unroll
    for (int v = 0; v < (NT / kWave); ++v) {
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

// a / b where the quotient is below 2^31
__device__ inline uint32_t quotient(uint64_t a, uint64_t b) {
  uint32_t q = (uint32_t)((double)a / (double)b);
  if (q * b > a) --q;
  else if ((q + 1ull) * b <= a) ++q;
  return q;
}

struct Drawn {
  int token;
  float prob;
};

// floor(u S), below S; NaN counts as 0
__device__ inline uint64_t draw_target(float u, uint64_t S) {
  const double t = floor((u > 0.f ? (double)fminf(u, 1.f) : 0.0) * (double)S);
  return min((uint64_t)t, S - 1);
}
// the running sum that top_p asks for: ceil(p S), 1 .. S
__device__ inline uint64_t top_p_sum(float p, uint64_t S) {
  return min(max((uint64_t)ceil((p > 0.f ? (double)p : 0.0) * (double)S), (uint64_t)1), S);
}

// Any row: every question by a radix descent over the row in memory
template <int DT, int NT>
__device__ __attribute__((noinline)) Drawn sample_general(const Row<DT> row, const RowSettings st,
                                                          Shared<DT, NT>& sh) {
  uint32_t best = 0;
  row.template each<NT>([&](uint32_t k, int) { best = max(best, k); });
#pragma unroll
  for (int m = 32; m >= 1; m >>= 1) best = max(best, (uint32_t)__shfl_xor(best, m));
  __syncthreads();
  if ((threadIdx.x & (kWave - 1)) == 0) sh.red32[threadIdx.x / kWave] = best;
  __syncthreads();
#pragma unroll
  for (int w = 0; w < NT / kWave; ++w) best = max(best, sh.red32[w]);
  if (!(st.T > 0.f) || best == 0u)   // greedy, or a row of NaN
    return {nth_index<DT, NT>(row, best, 0, sh), best ? 1.f : 0.f};
  const Weights w{key_value(best), best, 1.4426950408889634074 / (double)st.T};
  const double least = st.least();
  uint64_t S = 0, Sm = 0, have = 0;
  row.template each<NT>([&](uint32_t key, int) {
    const uint64_t m = key ? w(key) : 0ull;
    S += m;
    have += m ? 1 : 0;
    if (m && w.log2w(key) >= least) Sm += m;
  });
  S = block_sum_u64<Shared<DT, NT>, NT>(S, sh);
  Sm = block_sum_u64<Shared<DT, NT>, NT>(Sm, sh);
  have = block_sum_u64<Shared<DT, NT>, NT>(have, sh);
  if (st.k > 0 && (uint64_t)st.k < have) {
    // the k-th token's value; its larger ones and the first of its ties are kept
    const Crossing c = find_crossing<DT, NT>(row, w, (uint64_t)(st.k - 1), true, sh);
    uint64_t sum = 0;
    row.template each<NT>([&](uint32_t key, int) { sum += key > c.key ? w(key) : 0ull; });
    S = block_sum_u64<Shared<DT, NT>, NT>(sum, sh) + ((uint64_t)st.k - c.above) * w(c.key);
  }
  if (st.p < 1.f) {
    const uint64_t P = top_p_sum(st.p, S);
    const Crossing c = find_crossing<DT, NT>(row, w, P - 1, false, sh);
    const uint64_t W = w(c.key);
    S = c.above + ((P - 1 - c.above) / W + 1) * W;
  }
  S = min(S, Sm);
  const uint64_t target = draw_target(st.u, S);
  const Crossing c = find_crossing<DT, NT>(row, w, target, false, sh);
  const uint64_t W = w(c.key);
  return {nth_index<DT, NT>(row, c.key, (uint32_t)((target - c.above) / W), sh),
          (float)((double)W / (double)S)};
}

constexpr uint32_t kLowest16 = 0x007Fu;   // the key of -inf; smaller ones are NaN
__device__ inline uint32_t key16(float x) { return value_key(__float_as_uint(x)) >> 16; }
// the whole key of a 16-bit one: it ends in zeros, or ones where the value is negative
__device__ inline uint32_t key32(uint32_t k) { return (k << 16) | ((k & 0x8000u) ? 0u : 0xFFFFu); }
// the 16-bit keys of both halves: sign ? ~bits : bits | 0x8000
typedef short s16x2 __attribute__((ext_vector_type(2)));
typedef unsigned short u16x2 __attribute__((ext_vector_type(2)));
__device__ inline u16x2 keys16(uint32_t w) {
  const uint32_t sign = __builtin_bit_cast(uint32_t, (s16x2)(__builtin_bit_cast(s16x2, w) >> 15));
  return __builtin_bit_cast(u16x2, w ^ (sign | 0x80008000u));
}

// Passes over a row: its whole aligned 16-byte units, several of them in flight per thread, and
// the elements of its unaligned ends, one per thread.  Places without an element are negative
// NaN, whose key is the smallest and which no pass counts.  A row is read from HBM once; the
// passes after the first find it in the caches, and most of them read only the units of the
// threads that hold values above a bound.
// (Registers for a row of 150000 bf16 values leave too few for the passes: at every share kept
// there, the compiler spilled as much.)
constexpr int kParts = 4;   // a thread's unit j counts to its part j % kParts
struct Maxima {
  float part[kParts], all;   // largest values of the parts, and of all
};

template <int DT, int NT>
struct Passes {
  static constexpr int U = Row<DT>::U;
  static constexpr uint32_t kNone = 0xFFFFFFFFu;
  const Row<DT>& row;
  int head, full;      // elements before the first whole unit, whole units

  __device__ inline explicit Passes(const Row<DT>& x) : row(x) {
    head = x.lead ? min(U - x.lead, x.vocab) : 0;
    full = (x.vocab - head) / U;
  }
  __device__ inline const char* first() const { return row.base + (int64_t)head * (16 / U); }
  // f(unit's 16 bytes, index of its first element, part); the trip count is the workgroup's.
  // A unit's registers take the one A later as soon as it is done with; loads past the row read
  // its last unit.  (A loads, all waited for, then their work: the memory idles meanwhile.  A 8
  // where a unit is little work, 4 otherwise; 16 and 8 take as long.)
  template <int A, class F>
  __device__ __attribute__((always_inline)) inline void units(F&& f) const {
    int tid = threadIdx.x;
    asm volatile("" : "+v"(tid));   // (or the addresses of every pass are kept from the start)
    static_assert(A % kParts == 0, "a unit's part is known when the loop is unrolled");
    if (full > 0) {
      const uint32_t last = (uint32_t)(full - 1) * 16u;   // a row is below 2^32 bytes
      const char* const p = first();
      auto load = [&](int u) { return *(const uint4*)(p + min((uint32_t)u * 16u, last)); };
      uint4 x[A];
#pragma unroll
      for (int j = 0; j < A; ++j) x[j] = load(j * NT + tid);
      int u0 = 0;
      for (; u0 + A * NT <= full; u0 += A * NT) {
#pragma unroll
        for (int j = 0; j < A; ++j) {
          const int u = u0 + j * NT + tid;
          f(x[j], u * U + head, j % kParts);
          x[j] = load(u + A * NT);
          __builtin_amdgcn_sched_barrier(0);   // (or the loads gather at the loop's end)
        }
      }
#pragma unroll
      for (int j = 0; j < A; ++j) {
        if (u0 + j * NT >= full) break;
        const int u = u0 + j * NT + tid;
        if (u >= full) x[j] = make_uint4(kNone, kNone, kNone, kNone);
        f(x[j], u * U + head, j % kParts);
      }
    }
    ends(f);
  }
  template <class F>
  __device__ __attribute__((always_inline)) inline void ends(F&& f) const {
    if (row.vocab == full * U) return;
    const int tid = threadIdx.x, rest = head + full * U;
    int e = -1;
    if (tid < U && tid < head) e = tid;
    if (tid >= U && rest + tid - U < row.vocab) e = rest + tid - U;   // fewer than U of them
    uint32_t b = kNone;
    if (e >= 0)
      b = DT == TAPS_BF16 ? 0xFFFF0000u | ((const uint16_t*)row.base)[e]
                          : ((const uint32_t*)row.base)[e];
    f(make_uint4(b, kNone, kNone, kNone), max(e, 0), 0);
  }
  __device__ static inline u16x2 unit_max(const uint4& w) {
    return __builtin_elementwise_max(__builtin_elementwise_max(keys16(w.x), keys16(w.y)),
                                     __builtin_elementwise_max(keys16(w.z), keys16(w.w)));
  }
  // false (in all threads) where a positive NaN is among the workgroup's largest keys
  __device__ static inline bool from_keys(const u16x2 (&mk)[kParts], Maxima* m) {
    uint32_t top = 0;
#pragma unroll
    for (int s = 0; s < kParts; ++s) {
      const uint32_t k = max((uint32_t)mk[s][0], (uint32_t)mk[s][1]);
      top = max(top, k);
      // -inf's key is 0x7F (smaller: NaN or nothing)
      m->part[s] = k > 0x7Fu ? key_value(key32(k)) : -INFINITY;
    }
    m->all = fmaxf(fmaxf(m->part[0], m->part[1]), fmaxf(m->part[2], m->part[3]));
    return !__syncthreads_or(top > 0xFF80u);   // +inf's key
  }
  // The largest value of the first units, one per thread; NaN where a positive NaN is there
  __device__ __attribute__((always_inline)) inline float first_max(Shared<DT, NT>& sh) const {
    u16x2 mk[kParts] = {};
    mk[0] = unit_max(*(const uint4*)(first() + min((uint32_t)threadIdx.x, (uint32_t)(full - 1)) * 16u));
    Maxima m;
    if (!from_keys(mk, &m)) return NAN;
    return block_max_f32<Shared<DT, NT>, NT>(m.all, sh);
  }
  // The largest values of this thread's units (NaN left out; -inf where there is none).  bf16:
  // the largest 16-bit key, two at a time (three instructions; as floats the halves would be
  // unpacked and made quiet first, five); a positive NaN in any unit sends the workgroup through
  // the floats after all.
  __device__ __attribute__((always_inline)) inline Maxima max_value() const {
    Maxima m;
    bool done = false;
    if constexpr (DT == TAPS_BF16) {
      u16x2 mk[kParts] = {};
      units<8>([&](const uint4& w, int, int s) {
        mk[s] = __builtin_elementwise_max(mk[s], unit_max(w));
      });
      done = from_keys(mk, &m);
    }
    if (!done) {
#pragma unroll
      for (int s = 0; s < kParts; ++s) m.part[s] = -INFINITY;
      units<DT == TAPS_FP32 ? 8 : 4>([&](const uint4& w, int, int s) {
        const uint32_t ww[4] = {w.x, w.y, w.z, w.w};
        // (compared and selected: the compiler leaves operands of a maximum of three unquieted,
        // and a signalling NaN among them becomes the result)
#pragma unroll
        for (int q = 0; q < U; ++q) {
          const float x = __uint_as_float(
              DT == TAPS_BF16 ? ((q & 1) ? ww[q >> 1] & 0xFFFF0000u : ww[q >> 1] << 16) : ww[q & 3]);
          m.part[s] = x > m.part[s] ? x : m.part[s];
        }
      });
    }
    m.all = fmaxf(fmaxf(m.part[0], m.part[1]), fmaxf(m.part[2], m.part[3]));
    return m;
  }
  // f(values, whether each has lo <= value <= hi, index of the first) for the units that hold such
  // elements: only the parts (of a thread's
  // units) whose largest value reaches lo can hold one.  They are shared out to all threads;
  // where they are most of the parts, every unit is read.  Callers synchronize before the next
  // call.  (Whole threads instead of quarters: with 60 of 512 threads in question, their units
  // touch two thirds of the row's cache lines again.)
  template <class F>
  __device__ __attribute__((always_inline)) inline void between(const Maxima& mx, float lo,
                                                                float hi, Shared<DT, NT>& sh,
                                                                F&& f) const {
    const int tid = threadIdx.x;
    if (tid == 0) sh.n_hot = 0u;
    __syncthreads();
    if (__ballot(mx.all >= lo)) {
      uint64_t hot[kParts];
      uint32_t num = 0;
#pragma unroll
      for (int s = 0; s < kParts; ++s) {
        hot[s] = __ballot(mx.part[s] >= lo);
        num += (uint32_t)__popcll(hot[s]);
      }
      uint32_t at = 0;
      if ((tid & (kWave - 1)) == 0) at = atomicAdd(&sh.n_hot, num);
      at = __builtin_amdgcn_readfirstlane(at);
#pragma unroll
      for (int s = 0; s < kParts; ++s) {
        const uint32_t i =
            at + __builtin_amdgcn_mbcnt_hi((uint32_t)(hot[s] >> 32),
                                           __builtin_amdgcn_mbcnt_lo((uint32_t)hot[s], 0u));
        if (mx.part[s] >= lo) sh.hot[i] = (uint16_t)(s * NT + tid);
        at += (uint32_t)__popcll(hot[s]);
      }
    }
    __syncthreads();
    auto one = [&](const uint4& w, int e0, int) {
      const uint32_t ww[4] = {w.x, w.y, w.z, w.w};
      float x[U];
      bool in[U], any = false;   // one branch for the unit, which mostly holds none
#pragma unroll
      for (int q = 0; q < U; ++q) {
        x[q] = __uint_as_float(DT == TAPS_BF16
                                   ? ((q & 1) ? ww[q >> 1] & 0xFFFF0000u : ww[q >> 1] << 16)
                                   : ww[q & 3]);
        in[q] = x[q] >= lo && x[q] <= hi;
        any |= in[q];
      }
      if (any) f(x, in, e0);
    };
    constexpr int kAll = kParts * NT;
    const int n = (int)sh.n_hot, per = (full + kAll - 1) / kAll;
    if (2 * n > kAll) {
      units<4>(one);
      return;
    }
    // (neighbours take the same unit of their parts, whose cache lines many parts share)
    for (int i = tid; i < n * per; i += NT) {
      const int j = i / n, u = j * kAll + (int)sh.hot[i - j * n];
      if (u < full) one(*(const uint4*)(first() + (int64_t)u * 16), u * U + head, 0);
    }
    ends(one);
  }
};

// For `between`: f(value, index) element by element, which is the faster where units hold few
template <class F>
__device__ inline auto each(F&& f) {
  return [f](const auto& x, const auto& in, int e0) {
    constexpr int U = sizeof(in) / sizeof(in[0]);
#pragma unroll
    for (int q = 0; q < U; ++q)
      if (in[q]) f(x[q], e0 + q);
  };
}

// ... and a unit's elements into list[], past which sh.n only counts: one addition per wave, not
// one per element, where many come at once (16 rows x 1000: 12.6 -> 9.7 us with the bound below)
template <int DT, int NT, int U>
__device__ inline void append(Shared<DT, NT>& sh, const float (&x)[U], const bool (&in)[U], int e0) {
  uint64_t m[U];
  uint32_t num = 0;
#pragma unroll
  for (int q = 0; q < U; ++q) {
    m[q] = __ballot(in[q]);
    num += (uint32_t)__popcll(m[q]);
  }
  const uint64_t active = __ballot(true);
  uint32_t at = 0;
  if ((threadIdx.x & (kWave - 1)) == (uint32_t)__ffsll((long long)active) - 1u)
    at = atomicAdd(&sh.n, num);
  at = __builtin_amdgcn_readfirstlane(at);
#pragma unroll
  for (int q = 0; q < U; ++q) {
    if (!m[q]) continue;   // uniform
    const uint32_t i = at + __builtin_amdgcn_mbcnt_hi(
                                (uint32_t)(m[q] >> 32), __builtin_amdgcn_mbcnt_lo((uint32_t)m[q], 0u));
    if (in[q] && i < (uint32_t)kList)
      sh.u.l.list[i] = cand_key(value_key(__float_as_uint(x[q])), (uint32_t)(e0 + q));
    at += (uint32_t)__popcll(m[q]);
  }
}

// A key that at least k elements reach: the k-th largest of the maxima of kGroups groups of
// threads (0 where fewer groups hold a value).  k <= kFewTopK.
template <int DT, int NT>
__device__ inline uint32_t top_k_bound(float mx, int k, Shared<DT, NT>& sh) {
  constexpr int kPer = NT / kGroups;
  const int tid = threadIdx.x, lane = tid & (kWave - 1);
  uint32_t key = mx > -INFINITY ? value_key(__float_as_uint(mx)) : 0u;
#pragma unroll
  for (int d = 1; d < kPer; d <<= 1) key = max(key, (uint32_t)__shfl_xor(key, d));
  if (tid % kPer == 0) sh.group[tid / kPer] = key;
  __syncthreads();
  uint32_t g[kGroups / kWave];
#pragma unroll
  for (int i = 0; i < kGroups / kWave; ++i) g[i] = sh.group[i * kWave + lane];
  // the key's upper 16 bits, a wave for each candidate of the next 3 or 4 (for fp32 rows the bound
  // comes out a little low)
  constexpr int kWaves = NT / kWave, kBits = kWaves == 16 ? 4 : 3;
  static_assert(kWaves == 1 << kBits, "a wave per candidate");
  const int wave = __builtin_amdgcn_readfirstlane(tid / kWave);
  uint32_t T = 0;
#pragma unroll
  for (int s = 0; s * kBits < 16; ++s) {
    const int bits = min(kBits, 16 - s * kBits), bit = 32 - s * kBits - bits;
    const uint32_t c = T | ((uint32_t)wave << bit);
    uint32_t n = 0;
#pragma unroll
    for (int i = 0; i < kGroups / kWave; ++i) n += (uint32_t)__popcll(__ballot(g[i] >= c));
    uint32_t* const num = (s & 1) ? sh.other32 : sh.red32;   // the last step's may still be read
    if (lane == 0) num[wave] = n;
    __syncthreads();
    const uint64_t hit = __ballot(lane < (1 << bits) && num[lane & (kWaves - 1)] >= (uint32_t)k);
    // 0 reaches all groups, of which there are more than k
    T |= (uint32_t)(63 - __clzll((long long)hit)) << bit;
  }
  return T;
}

// ----------------------------------------------------------------------------------
// Elements ranked one by one: list[0 .. n) into sorted[]
template <int DT, int NT>
__device__ inline void sort_list(uint32_t n, Shared<DT, NT>& sh) {
  ListScratch& ls = sh.u.l;
  const uint32_t whole = n & ~7u;
  for (uint32_t i = threadIdx.x; i < n; i += NT) {
    const uint64_t mine = ls.list[i];
    uint32_t rank = 0, j = 0;
    ulonglong2 v[4];   // eight at a time, every lane the same ones
    auto read = [&]() {
#pragma unroll
      for (int t = 0; t < 4; ++t) v[t] = *(const ulonglong2*)&ls.list[j + 2 * t];
    };
    for (; j < whole; j += 8) {
      read();
#pragma unroll
      for (int t = 0; t < 4; ++t) rank += (v[t].x > mine ? 1u : 0u) + (v[t].y > mine ? 1u : 0u);
    }
    if (j < n) {   // (the list has room for eight; what lies past n is not counted)
      read();
#pragma unroll
      for (int t = 0; t < 4; ++t) {
        rank += j + 2 * t < n && v[t].x > mine ? 1u : 0u;
        rank += j + 2 * t + 1 < n && v[t].y > mine ? 1u : 0u;
      }
    }
    ls.sorted[rank] = mine;
  }
  __syncthreads();
}

// cum[i] = f(sum of w(key of sorted[0]) .. w(key of sorted[i])); returns the whole sum
template <int DT, int NT, class W, class F>
__device__ inline uint64_t sum_list(uint32_t n, Shared<DT, NT>& sh, W&& w, F&& f) {
  constexpr int E = kList / NT;
  ListScratch& ls = sh.u.l;
  const uint32_t i0 = threadIdx.x * E;
  uint64_t m[E], sum = 0, all;
#pragma unroll
  for (int e = 0; e < E; ++e) {
    m[e] = i0 + e < n ? w((uint32_t)(ls.sorted[i0 + e] >> 32)) : 0ull;
    sum += m[e];
  }
  uint64_t run = block_scan_u64<Shared<DT, NT>, NT>(sum, sh, &all) - sum;
#pragma unroll
  for (int e = 0; e < E; ++e) {
    run += m[e];
    if (i0 + e < n) ls.cum[i0 + e] = f(run);
  }
  __syncthreads();
  return all;
}

// The first i < n whose value(i) exceeds target, n if none does (values do not fall; n at most
// 64 B).  Two reads, by every wave for itself: no barrier.
template <int B, class F>
__device__ inline int first_above(uint64_t target, int n, F&& value) {
  static_assert(B <= kWave, "a block per lane, then a lane per element of one");
  const int lane = threadIdx.x & (kWave - 1);
  const int end = lane * B + B - 1;
  const uint64_t blocks = __ballot(end >= n || value(end) > target);
  const int i = (blocks ? (int)__ffsll((long long)blocks) - 1 : kWave - 1) * B + lane;
  const uint64_t hit = __ballot(lane < B && (i >= n || value(i) > target));
  return min(i - lane + (hit ? (int)__ffsll((long long)hit) - 1 : B), n);
}
// ... in cum[0 .. n), where one does
template <int DT, int NT>
__device__ inline uint32_t first_in_list(uint64_t target, uint32_t n, Shared<DT, NT>& sh) {
  return (uint32_t)first_above<kList / kWave>(target, (int)n,
                                             [&](int i) { return sh.u.l.cum[i]; });
}

// how many of the list's first elements satisfy `in` (those that do come first)
template <int DT, int NT, class F>
__device__ inline uint32_t count_list(uint32_t n, Shared<DT, NT>& sh, F&& in) {
  uint64_t c = 0;
  for (uint32_t i = threadIdx.x; i < n; i += NT)
    c += in((uint32_t)(sh.u.l.sorted[i] >> 32)) ? 1 : 0;
  return (uint32_t)block_sum_u64<Shared<DT, NT>, NT>(c, sh);
}

// A float bound rounded down by more than the arithmetic can be off
__device__ inline float bound_below(double x, float M) {
  return (float)(x - 1e-6 * (fabs(x) + fabs((double)M)));
}

// A small top_k, or min_p: the elements above a bound, ranked.  False: more than kList of them.
template <int DT, int NT>
__device__ __attribute__((always_inline)) inline bool sample_listed(
    const Passes<DT, NT>& passes, const Maxima& mx, const Weights& w, const RowSettings& st,
    Shared<DT, NT>& sh, Drawn* out) {
  const double least = st.least();
  float thr = -INFINITY;
  if (st.cut_by_min_p() && w.scale > 0.0)   // (an infinite temperature: all weights are equal)
    thr = w.top == INFINITY ? w.top : bound_below((double)w.top + least / w.scale, w.top);
  if (st.few()) {
    const uint32_t key = top_k_bound<DT, NT>(mx.all, st.k, sh);
    if (key) thr = fmaxf(thr, key_value(key));
  }
  ListScratch& ls = sh.u.l;
  if (threadIdx.x == 0) sh.n = 0u;
  __syncthreads();
  passes.between(mx, thr, INFINITY, sh,
                 [&](const auto& x, const auto& in, int e0) { append<DT, NT>(sh, x, in, e0); });
  __syncthreads();
  const uint32_t n = sh.n;
  if (n > (uint32_t)kList) return false;
  sort_list<DT, NT>(n, sh);
  uint64_t S = sum_list<DT, NT>(n, sh, w, [](uint64_t c) { return c; });
  if (st.k > 0 && (uint32_t)st.k < n) S = ls.cum[st.k - 1];
  if (st.p < 1.f) S = ls.cum[first_in_list<DT, NT>(top_p_sum(st.p, S) - 1, n, sh)];
  if (st.mp > 0.f) {
    const uint32_t in =
        count_list<DT, NT>(n, sh, [&](uint32_t key) { return w.log2w(key) >= least; });
    S = min(S, ls.cum[in - 1]);
  }
  const uint32_t r = first_in_list<DT, NT>(draw_target(st.u, S), n, sh);
  out->token = (int)cand_index(ls.sorted[r]);
  out->prob = (float)((double)(ls.cum[r] - (r ? ls.cum[r - 1] : 0ull)) / (double)S);
  return true;
}

// ----------------------------------------------------------------------------------
// bf16: a row holds few distinct values, so the elements are counted by value (16-bit keys from
// the largest down, as far as weights reach) and every sum is over values: one exponential per
// value that occurs, none per element, and a crossing is exact at once.
// Without a known maximum the row is read once: the window's upper end lies above the largest of
// the first values by a factor of 256 (1024 keys), or by 64, and the pass finds the maximum as it
// counts.
// Returns false where the window is too wide, a value lies above it or occurs 65536 times, or a
// positive NaN takes part.  16 bits per count let two workgroups share a CU's LDS.
template <int DT, int NT>
__device__ __attribute__((always_inline)) inline bool sample_counted(
    const Passes<DT, NT>& passes, Maxima& mx, bool known, float M, const RowSettings& st,
    Shared<DT, NT>& sh, Drawn* out) {
  constexpr int kWaves = NT / kWave;
  const int tid = threadIdx.x, lane = tid & (kWave - 1), wave = tid / kWave;
  Weights w{M, 0u, 1.4426950408889634074 / (double)st.T};
  CountScratch& cs = sh.u.c;
  if (!known) {
    if (passes.full == 0) return false;
    M = passes.first_max(sh);
    if (!(M > -INFINITY)) return false;
  }
  // down to the values whose weight rounds to 0 (two more: the bound is rounded to bf16)
  const float low = (float)((double)M - 44.5 / w.scale);
  uint32_t klow = low > -INFINITY ? key16(low) : 0u;
  klow = klow > kLowest16 + 2u ? klow - 2u : kLowest16;
  if (klow == 0x8000u) klow = 0x7FFFu;   // +0 and -0 are equal
  klow = min(klow, key16(M));
  uint32_t kM = key16(M);   // the window's upper end
  if (!known) {
    kM = min(max(kM + 1024u, key16(M + 64.f)), 0xFF80u);   // +inf's key
  }
  const uint32_t Wn = kM - klow + 1u;
  if (Wn > (uint32_t)kWindow) return false;
  const int runs = (int)((Wn + kRun - 1) / kRun);
  for (int i = tid; i < runs * (kRun / 8); i += NT)
    ((uint4*)cs.count)[i] = make_uint4(0u, 0u, 0u, 0u);
  __syncthreads();
  uint32_t in_window = 0;   // of the wave
  u16x2 mk[kParts] = {};
  passes.template units<4>([&](const uint4& v, int, int s) {
    const uint32_t ww[4] = {v.x, v.y, v.z, v.w};
    const u16x2 top = {(unsigned short)kM, (unsigned short)kM};
#pragma unroll
    for (int q = 0; q < 4; ++q) {
      // NaN keys fall outside the window
      const u16x2 k = keys16(ww[q]);
      mk[s] = __builtin_elementwise_max(mk[s], k);
      const uint32_t idx = __builtin_bit_cast(uint32_t, (u16x2)(top - k));
      const uint32_t i0 = idx & 0xFFFFu, i1 = idx >> 16;
      in_window += __popcll(__ballot(i0 < Wn)) + __popcll(__ballot(i1 < Wn));
      // a shift counts its amount's low five bits only: 16 (i & 1)
      atomicAdd(&cs.count[i0 < Wn ? i0 >> 1 : kWindow / 2 + lane], 1u << ((i0 << 4) & 31u));
      atomicAdd(&cs.count[i1 < Wn ? i1 >> 1 : kWindow / 2 + lane], 1u << ((i1 << 4) & 31u));
    }
  });
  if (!known) {
    if (!passes.from_keys(mk, &mx)) return false;
    M = block_max_f32<Shared<DT, NT>, NT>(mx.all, sh);
    if (key16(M) > kM) return false;
  }
  if (M == 0.f) M = 0.f;   // not -0
  w.top = M;
  w.key = value_key(__float_as_uint(M));
  __syncthreads();
  auto count_at = [&](uint32_t i) -> uint32_t {
    return (cs.count[i >> 1] >> (16 * (i & 1u))) & 0xFFFFu;
  };
  if (tid == 0 && kM >= 0x8000u && kM - 0x8000u + 1u < Wn) {   // -0 counts as +0
    const uint32_t z = kM - 0x8000u;
    const uint32_t a = count_at(z), b = count_at(z + 1u);
    cs.count[z >> 1] += ((a + b) & 0xFFFFu) << (16 * (z & 1u));
    cs.count[z >> 1] -= a << (16 * (z & 1u));
    cs.count[(z + 1u) >> 1] -= b << (16 * ((z + 1u) & 1u));
  }
  __syncthreads();

  // four values per lane of run r: their counts and weights
  struct Four {
    uint32_t c[4];
    uint64_t W[4], m[4];
  };
  auto four = [&](int r) -> Four {
    const uint2 p = ((const uint2*)cs.count)[r * kWave + lane];
    Four f;
    f.c[0] = p.x & 0xFFFFu;
    f.c[1] = p.x >> 16;
    f.c[2] = p.y & 0xFFFFu;
    f.c[3] = p.y >> 16;
#pragma unroll
    for (int j = 0; j < 4; ++j) {
      f.W[j] = w(key32(kM - (uint32_t)(r * kRun + 4 * lane + j)));
      f.m[j] = f.W[j] * f.c[j];
    }
    return f;
  };
  for (int r = wave; r < runs; r += kWaves) {
    const uint2 p = ((const uint2*)cs.count)[r * kWave + lane];
    uint64_t m = 0;
    uint32_t n = 0;
    if (__ballot((p.x | p.y) != 0u)) {
      const Four f = four(r);
      m = wave_sum_u64(f.m[0] + f.m[1] + f.m[2] + f.m[3]);
      n = __builtin_amdgcn_readlane(wave_scan_u32(f.c[0] + f.c[1] + f.c[2] + f.c[3]), kWave - 1);
    }
    if (lane == 0) cs.mass[r] = m, cs.num[r] = n;
  }
  __syncthreads();
  uint64_t S, have;
  {
    // the runs' counts, and above them the elements that the waves have seen in the window
    const uint64_t m = tid < runs ? cs.mass[tid] : 0ull, n = tid < runs ? cs.num[tid] : 0ull;
    const uint64_t seen = lane == 0 ? (uint64_t)in_window << 32 : 0ull;
    const uint64_t pm = block_scan_u64<Shared<DT, NT>, NT>(m, sh, &S) - m;
    const uint64_t pn = block_scan_u64<Shared<DT, NT>, NT>(n + seen, sh, &have) - n;
    if (tid < runs) cs.mass[tid] = pm, cs.num[tid] = (uint32_t)pn;
  }
  __syncthreads();
  // a count past 16 bits loses 65536, or turns them into one of its neighbour's
  if ((have >> 32) != (have & 0xFFFFFFFFull)) return false;
  have &= 0xFFFFFFFFull;

  struct Cross {
    uint32_t pos, ties, nth;     // window position, elements there, the crossing one among them
    uint64_t through, W;         // sum with the crossing one, weight of each
  };
  // Where the running sum (count) first exceeds target.  One wave looks into the run (all of
  // them would share its evaluation of 256 weights' worth of vector time).
  auto crossing = [&](uint64_t target, bool by_count) -> Cross {
    if (wave == 0) {
      // the last run before which the sum does not exceed it
      constexpr int kBlock = (kRuns + kWave - 1) / kWave;
      const int r =
          (by_count ? first_above<kBlock>(target, runs, [&](int i) { return (uint64_t)cs.num[i]; })
                    : first_above<kBlock>(target, runs, [&](int i) { return cs.mass[i]; })) - 1;
      const Four f = four(r);
      uint64_t m[4];   // what is counted
#pragma unroll
      for (int j = 0; j < 4; ++j) m[j] = by_count ? (uint64_t)f.c[j] : f.m[j];
      const uint64_t mine = m[0] + m[1] + m[2] + m[3];
      const uint64_t incl = (by_count ? (uint64_t)cs.num[r] : cs.mass[r]) + wave_scan_u64(mine);
      const uint64_t sums = by_count ? wave_scan_u64(f.m[0] + f.m[1] + f.m[2] + f.m[3]) : 0ull;
      const int l = __ffsll((long long)__ballot(incl > target)) - 1;
      if (lane == l) {
        uint64_t above = incl - mine, sum = cs.mass[r] + sums - (f.m[0] + f.m[1] + f.m[2] + f.m[3]);
        uint64_t W = f.W[0];
        uint32_t j = 0, ties = f.c[0];
#pragma unroll
        for (int t = 0; t < 3; ++t)
          if (j == (uint32_t)t && above + m[t] <= target) {
            above += m[t];
            sum += f.m[t];
            j = t + 1;
            W = f.W[t + 1];
            ties = f.c[t + 1];
          }
        const uint32_t nth = by_count ? (uint32_t)(target - above) : quotient(target - above, W);
        sh.out32[1] = (uint32_t)(r * kRun + 4 * lane) + j;
        sh.out32[2] = ties;
        sh.out32[3] = nth;
        sh.out64[0] = (by_count ? sum : above) + (nth + 1ull) * W;
        sh.out64[1] = W;
      }
    }
    __syncthreads();
    const Cross x{sh.out32[1], sh.out32[2], sh.out32[3], sh.out64[0], sh.out64[1]};
    __syncthreads();
    return x;
  };
  // sum of the weights before window position i
  auto sum_before = [&](uint32_t i) -> uint64_t {
    const int r = (int)(i / kRun);
    const Four f = four(r);
    uint64_t m = 0;
#pragma unroll
    for (int j = 0; j < 4; ++j) m += (uint32_t)(r * kRun + 4 * lane + j) < i ? f.m[j] : 0ull;
    return cs.mass[r] + wave_sum_u64(m);
  };

  uint64_t kept = S;
  if (st.k > 0 && (uint64_t)st.k < have) {
    kept = crossing((uint64_t)(st.k - 1), true).through;
  }
  if (st.p < 1.f) {
    kept = crossing(top_p_sum(st.p, kept) - 1, false).through;
  }
  if (st.mp > 0.f) {
    const double least = st.least();
    uint32_t lo = 0, hi = Wn;   // positions to lo are kept, those from hi on are not
    while (hi - lo > 1u) {
      const uint32_t mid = (lo + hi) / 2u;
      if (w.log2w(key32(kM - mid)) >= least) lo = mid;
      else hi = mid;
    }
    if (hi < Wn) kept = min(kept, sum_before(hi));
  }
  const Cross c = crossing(draw_target(st.u, kept), false);
  const uint32_t key = key32(kM - c.pos);
  out->prob = (float)((double)c.W / (double)kept);
  if (c.ties > (uint32_t)kList) {
    out->token = nth_index<DT, NT>(passes.row, key, c.nth, sh);
    return true;
  }
  // the nth of the value's elements in index order
  if (tid == 0) sh.n = 0u;
  __syncthreads();   // the counts are read: the list may take their place
  const float value = key_value(key);
  passes.between(mx, value, value, sh, each([&](float, int e) {
    sh.u.l.list[atomicAdd(&sh.n, 1u)] = (uint64_t)(0xFFFFFFFFu - (uint32_t)e);
  }));
  __syncthreads();
  sort_list<DT, NT>(c.ties, sh);
  out->token = (int)(0xFFFFFFFFu - (uint32_t)sh.u.l.sorted[c.nth]);
  return true;
}

// ----------------------------------------------------------------------------------
// fp32, the whole vocabulary's sum (a larger top_k, top_p or no filter): weights are added up by
// bins of 1/32 octave.  Weight 2^-(z / 32), z = 32 log2(e) (M - x) / T, is the bin's 2^-(b / 32),
// b = z rounded to an integer, times a factor 2^-(t / 32), t = z - b, from a short series; a bin
// adds up its factors (integers of 2^-43), and its sum is that times 2^-(b / 32), rounded down.
// The bin where a running sum or count passes its target is then ranked one by one; of one that
// the list does not hold, 1/1024 is, found the same way, or that has one value only (logits that
// were bf16 once).  b comes from adding 1.5 * 2^52: its low word is the integer.  (Conversions and
// the fraction of a double run at a quarter of the rate of products: with them, and bins from b to
// b + 1, the pass over 50257 values took 8.3 us.)
// False: anything denser, or an infinite maximum or temperature.
template <int DT, int NT>
__device__ __attribute__((always_inline)) inline bool sample_binned(
    const Passes<DT, NT>& passes, const Maxima& mx, const Weights& w, const RowSettings& st,
    Shared<DT, NT>& sh, Drawn* out) {
  const int tid = threadIdx.x, lane = tid & (kWave - 1);
  BinScratch& bs = sh.u.b;
  const float M = w.top;
  // differences to an infinite maximum are not 0 even for its equals, and at an infinite
  // temperature all weights are equal
  if (M == INFINITY || !(w.scale > 0.0)) return false;
  const double scale = kPerOctave * w.scale, inverse = 1.0 / scale;
  for (int i = tid; i < kWeightBins; i += NT) bs.mass[i] = 0ull, bs.num[i] = 0u;
  __syncthreads();
  constexpr double kInt = 6755399441055744.0;   // 1.5 * 2^52
  // depths from here on add nothing (a million of them would add up to more than their weights,
  // each of which is 0)
  constexpr double kDeepest = kOctaves * kPerOctave;
  auto depth = [&](float x) -> double { return ((double)M - (double)x) * scale; };
  auto offset = [&](double z) -> double { return z - ((z + kInt) - kInt); };
  auto bin_at = [&](double z) -> int { return (int)__double_as_longlong(z + kInt); };
  // 2^-(t / 32) to 2^-48 for |t| <= 1/2
  auto factor = [&](double t) -> uint64_t {
    constexpr double c = -0.69314718055994530942 / kPerOctave;
    double p = scalar(c * c * c * c * c / 120.0);
    p = fma(p, t, scalar(c * c * c * c / 24.0));
    p = fma(p, t, scalar(c * c * c / 6.0));
    p = fma(p, t, scalar(c * c * 0.5));
    p = fma(p, t, scalar(c));
    return fixed43(fma(p, t, scalar(513.0)));
  };
  const bool counts = st.k > 0;
  passes.template units<4>([&](const uint4& v, int, int) {
    const uint32_t ww[4] = {v.x, v.y, v.z, v.w};
    double z[4];
    uint64_t f[4];
    // the four series side by side; elements past the last bin (or NaN) add nothing
#pragma unroll
    for (int q = 0; q < 4; ++q) {
      z[q] = depth(__uint_as_float(ww[q]));
      f[q] = factor(offset(z[q]));
    }
    // (kept out of the branches, where each would wait for its own chain of products)
    asm volatile("" : "+v"(f[0]), "+v"(f[1]), "+v"(f[2]), "+v"(f[3]));
    int at[4];
#pragma unroll
    for (int q = 0; q < 4; ++q) {
      at[q] = z[q] < kDeepest ? bin_at(z[q]) : kWeightBins + lane;
      atomicAdd((unsigned long long*)&bs.mass[at[q]], (unsigned long long)f[q]);
    }
    if (counts) {   // uniform
#pragma unroll
      for (int q = 0; q < 4; ++q) atomicAdd(&bs.num[at[q]], 1u);
    }
  });
  __syncthreads();
  auto bin_scale = [&](int b) -> double { return exp2_neg(-(double)b / kPerOctave); };
  uint64_t S, have = 0;
  {
    constexpr int E = (kWeightBins + NT - 1) / NT;
    uint64_t m[E], n[E], sum = 0, num = 0;
#pragma unroll
    for (int e = 0; e < E; ++e) {
      const int b = tid * E + e;
      m[e] = b < kWeightBins ? (uint64_t)(bin_scale(b) * (double)bs.mass[b]) : 0ull;
      n[e] = b < kWeightBins ? bs.num[b] : 0u;
      sum += m[e];
      num += n[e];
    }
    uint64_t run = block_scan_u64<Shared<DT, NT>, NT>(sum, sh, &S) - sum;
    uint64_t nrun = counts ? block_scan_u64<Shared<DT, NT>, NT>(num, sh, &have) - num : 0ull;
#pragma unroll
    for (int e = 0; e < E; ++e) {
      const int b = tid * E + e;
      if (b < kWeightBins) bs.mass[b] = run, bs.num[b] = (uint32_t)nrun;
      run += m[e];
      nrun += n[e];
    }
  }
  __syncthreads();

  // the part of its bin that an element with offset t is in
  auto sub_at = [&](double t) -> int { return min((int)((t + 0.5) * kSub), kSub - 1); };
  // f(x, z, t, index) for the elements of a bin's parts lo .. hi
  auto within = [&](int bin, int lo, int hi, auto&& f) {
    const double z0 = (double)bin - 0.5;
    passes.between(mx, bound_below((double)M - (z0 + (double)(hi + 1) / kSub) * inverse, M),
                   -bound_below((z0 + (double)lo / kSub) * inverse - (double)M, M), sh,
                   each([&](float x, int e) {
                     const double z = depth(x), t = offset(z);
                     if (!(z < kDeepest) || bin_at(z) != bin) return;
                     const int i = sub_at(t);
                     if (i >= lo && i <= hi) f(x, z, t, e);
                   }));
    __syncthreads();
  };
  // list[] from the elements of a bin's parts lo .. hi; their number
  auto collect = [&](int bin, int lo, int hi) -> uint32_t {
    __syncthreads();
    if (tid == 0) sh.n = 0u;
    within(bin, lo, hi, [&](float x, double, double, int e) {
      const uint32_t i = atomicAdd(&sh.n, 1u);
      if (i < (uint32_t)kList)
        bs.l.list[i] = cand_key(value_key(__float_as_uint(x)), (uint32_t)e);
    });
    return sh.n;
  };
  struct Found {
    uint32_t key, nth;   // the element's key; its place among its equals where token is -1
    int token, bin;
    uint64_t through;    // the running sum with it
  };
  // The element where the running sum (count) in rank order first exceeds target
  auto locate = [&](uint64_t target, bool by_count, Found& f) -> bool {
    // the last bin before which the sum does not exceed it
    constexpr int kBlock = (kWeightBins + kWave - 1) / kWave;
    const int bin =
        (by_count ? first_above<kBlock>(target, kWeightBins, [&](int b) { return (uint64_t)bs.num[b]; })
                  : first_above<kBlock>(target, kWeightBins, [&](int b) { return bs.mass[b]; })) - 1;
    f.bin = bin;
    const double bsc = bin_scale(bin);
    const uint64_t before = bs.mass[bin];
    // the running sum after the bin's factors c
    auto through = [&](uint64_t c) -> uint64_t { return before + (uint64_t)(bsc * (double)c); };
    int sub0 = 0, sub1 = kSub - 1;
    uint64_t c0 = 0;                      // factors of the bin, elements, before the list
    uint32_t n0 = bs.num[bin];
    uint32_t n = collect(bin, sub0, sub1);
    if (n > (uint32_t)kList) {
      __syncthreads();
      for (int i = tid; i < kSub; i += NT) bs.sub[i] = 0ull, bs.sub_num[i] = 0u;
      __syncthreads();
      within(bin, sub0, sub1, [&](float, double, double t, int) {
        const int i = sub_at(t);
        atomicAdd((unsigned long long*)&bs.sub[i], (unsigned long long)factor(t));
        atomicAdd(&bs.sub_num[i], 1u);
      });
      constexpr int E = kSub / NT;
      uint64_t m[E], k[E], sum = 0, num = 0, all;
#pragma unroll
      for (int e = 0; e < E; ++e) {
        m[e] = bs.sub[tid * E + e];
        k[e] = bs.sub_num[tid * E + e];
        sum += m[e];
        num += k[e];
      }
      uint64_t run = block_scan_u64<Shared<DT, NT>, NT>(sum, sh, &all) - sum;
      uint64_t nrun = n0 + block_scan_u64<Shared<DT, NT>, NT>(num, sh, &all) - num;
#pragma unroll
      for (int e = 0; e < E; ++e) {
        const uint64_t lo = by_count ? nrun : through(run);
        const uint64_t hi = by_count ? nrun + k[e] : through(run + m[e]);
        if (lo <= target && target < hi) {
          sh.out32[1] = (uint32_t)(tid * E + e);
          sh.out32[2] = (uint32_t)nrun;
          sh.out64[0] = run;
        }
        run += m[e];
        nrun += k[e];
      }
      __syncthreads();
      sub0 = sub1 = (int)sh.out32[1];
      n0 = sh.out32[2];
      c0 = sh.out64[0];
      n = collect(bin, sub0, sub1);
    }
    if (n > (uint32_t)kList) {   // more than the list holds: equals?
      const uint32_t key = (uint32_t)(bs.l.list[0] >> 32);
      if (tid == 0) sh.out32[3] = 0u;
      within(bin, sub0, sub1, [&](float x, double, double, int) {
        if (value_key(__float_as_uint(x)) != key) sh.out32[3] = 1u;
      });
      if (sh.out32[3]) return false;
      const uint64_t W = factor(offset(depth(key_value(key))));
      uint32_t nth = (uint32_t)(target - n0);
      if (!by_count) {
        uint32_t hi = n - 1;   // the crossing one is in [nth, hi]
        nth = 0;
        while (nth < hi) {
          const uint32_t mid = (nth + hi) / 2;
          if (through(c0 + (mid + 1ull) * W) > target) hi = mid;
          else nth = mid + 1;
        }
      }
      f.key = key;
      f.nth = nth;
      f.token = -1;
      f.through = through(c0 + (nth + 1ull) * W);
      return true;
    }
    sort_list<DT, NT>(n, sh);
    sum_list<DT, NT>(
        n, sh, [&](uint32_t key) { return factor(offset(depth(key_value(key)))); },
        [&](uint64_t c) { return through(c0 + c); });
    const uint32_t i = by_count ? (uint32_t)(target - n0) : first_in_list<DT, NT>(target, n, sh);
    const uint64_t e = bs.l.sorted[i];
    f.key = (uint32_t)(e >> 32);
    f.token = (int)cand_index(e);
    f.through = bs.l.cum[i];
    return true;
  };

  // what min_p keeps (before the loop: inside, the compiler evaluates its logarithm and bounds
  // for every row, 1 us)
  uint64_t Sm = S;
  if (st.mp > 0.f) {
    const double last = -kPerOctave * st.least();   // the depth of the last one kept
    if (last < kDeepest) {
      const int bin = bin_at(last);
      uint64_t c = 0;   // of the bin, what is kept
      within(bin, 0, kSub - 1, [&](float, double z, double t, int) {
        if (z <= last) c += factor(t);
      });
      c = block_sum_u64<Shared<DT, NT>, NT>(c, sh);
      Sm = bs.mass[bin] + (uint64_t)(bin_scale(bin) * (double)c);
    }
  }
  uint64_t kept = S;
  Found f;
#pragma unroll 1
  for (int step = 0; step < 3; ++step) {   // top_k, top_p, the drawn one
    uint64_t target;
    if (step == 0) {
      if (!counts || (uint64_t)st.k >= have) continue;
      target = (uint64_t)(st.k - 1);
    } else if (step == 1) {
      if (!(st.p < 1.f)) continue;
      target = top_p_sum(st.p, kept) - 1;
    } else {
      kept = min(kept, Sm);
      target = draw_target(st.u, kept);
    }
    if (!locate(target, step == 0, f)) return false;
    if (step < 2) kept = f.through;
  }
  out->token = f.token >= 0 ? f.token : nth_index<DT, NT>(passes.row, f.key, f.nth, sh);
  out->prob = (float)(bin_scale(f.bin) * (double)factor(offset(depth(key_value(f.key)))) /
                      (double)kept);
  return true;
}

template <int DT, int NT>
__global__ __launch_bounds__(NT, 4) void sample_kernel(
    const void* __restrict__ logits, int64_t row_bytes, int budget, int vocab,
    const int32_t* __restrict__ n_nodes, const Settings s, const float* __restrict__ u,
    int32_t* __restrict__ tokens, float* __restrict__ probs) {
  __shared__ Shared<DT, NT> sh;
  const int r = blockIdx.x, b = r / budget, tid = threadIdx.x;
  if (n_nodes && r - b * budget >= n_nodes[b]) {
    if (tid == 0) {
      tokens[r] = -1;
      if (probs) probs[r] = 0.f;
    }
    return;
  }
  const Row<DT> row((const char*)logits + (size_t)r * row_bytes, vocab);
  const Passes<DT, NT> passes(row);
  RowSettings st;
  auto uniform = [](float x) {
    return __uint_as_float(__builtin_amdgcn_readfirstlane(__float_as_uint(x)));
  };
  st.T = uniform(s.temperature ? s.temperature[b] : 1.f);
  st.k = __builtin_amdgcn_readfirstlane(s.top_k ? s.top_k[b] : 0);
  st.p = uniform(s.top_p ? s.top_p[b] : 1.f);
  st.mp = uniform(s.min_p ? s.min_p[b] : 0.f);
  st.u = uniform(u[r]);
  Drawn d;
  bool done = false;
  const bool listed = st.few() || st.cut_by_min_p();
  Maxima mx;
  float M = 0.f;
  // The largest value, and with it greedy rows and the ranked few; false: nothing is left to do
  // here
  auto with_max = [&]() -> bool {
    mx = passes.max_value();
    M = block_max_f32<Shared<DT, NT>, NT>(mx.all, sh);
    if (M == 0.f) M = 0.f;   // not -0
    if (!(M > -INFINITY)) return false;
    if (!(st.T > 0.f)) {
      if (tid == 0) sh.n = 0xFFFFFFFFu;
      __syncthreads();
      passes.between(mx, M, INFINITY, sh, [&](const auto&, const auto& in, int e0) {
        int least = 0x7FFFFFFF;
#pragma unroll
        for (int q = Row<DT>::U - 1; q >= 0; --q) least = in[q] ? e0 + q : least;
        atomicMin(&sh.n, (uint32_t)least);
      });
      __syncthreads();
      d = {(int)sh.n, 1.f};
      done = true;
    } else if (listed) {
      const Weights w{M, value_key(__float_as_uint(M)), 1.4426950408889634074 / (double)st.T};
      done = sample_listed<DT, NT>(passes, mx, w, st, sh, &d);
      __syncthreads();
    }
    return !done;
  };
  if constexpr (DT == TAPS_BF16) {
    // rows whose whole sum counts are read once, and again only where that fails
    for (int known = __builtin_amdgcn_readfirstlane(st.T > 0.f && !listed ? 0 : 1);; known = 1) {
      // (or the compiler lays the loop out twice, and evaluates before it all that any path
      // makes of the settings)
      asm volatile("" : "+s"(known), "+s"(st.T), "+s"(st.p), "+s"(st.mp), "+s"(st.u), "+s"(st.k));
      if (known && !with_max()) break;
      done = sample_counted<DT, NT>(passes, mx, known != 0, M, st, sh, &d);
      if (done || known) break;
      __syncthreads();
    }
  } else if (with_max()) {
    const Weights w{M, value_key(__float_as_uint(M)), 1.4426950408889634074 / (double)st.T};
    done = sample_binned<DT, NT>(passes, mx, w, st, sh, &d);
  }
  if (!done) {   // uniform
    __syncthreads();
    d = sample_general<DT, NT>(row, st, sh);
  }
  if (tid == 0) {
    tokens[r] = d.token;
    if (probs) probs[r] = d.prob;
  }
}

template <int DT>
hipError_t launch_dt(const void* logits, int64_t row_bytes, int budget, int vocab, int rows,
                     const int32_t* n_nodes, const Settings& st, const float* u, int32_t* tokens,
                     float* probs, hipStream_t stream) {
  // one row per CU: all its waves; more rows: two workgroups share a CU, one's passes over
  // memory beside the other's work in LDS.  us with 1024 / 512 threads, 151,936 values in bf16 with
  // top_p, with top_k + top_p, in fp32 with top_p, 50,257 in fp32 with top_k: 256 rows 35 / 40, 25 /
  // 24, 97 / 104, 18 / 17; 257 rows 57 / 48, 37 / 28, 136 / 120, 26 / 19; 500 rows 71 / 60, 49 / 40,
  // 171 / 172, 37 / 28; 768 rows 102 / 93, 71 / 56, 244 / 264, 55 / 43.
  if (rows <= 256)
    sample_kernel<DT, 1024><<<(unsigned)rows, 1024, 0, stream>>>(logits, row_bytes, budget, vocab,
                                                                 n_nodes, st, u, tokens, probs);
  else
    sample_kernel<DT, 512><<<(unsigned)rows, 512, 0, stream>>>(logits, row_bytes, budget, vocab,
                                                               n_nodes, st, u, tokens, probs);
  return hipGetLastError();
}

}  // namespace

hipError_t launch_sample(const void* logits, int64_t row_bytes, int batch, int budget, int vocab,
                         int dtype, const int32_t* n_nodes, const taps_sampling& s,
                         const float* u, int32_t* tokens, float* probs, hipStream_t stream) {
  if (batch <= 0) return hipSuccess;
  const Settings st{s.temperature, s.top_p, s.min_p, s.top_k};
  const int rows = batch * budget;
  return dtype == TAPS_BF16 ? launch_dt<TAPS_BF16>(logits, row_bytes, budget, vocab, rows, n_nodes,
                                                   st, u, tokens, probs, stream)
                            : launch_dt<TAPS_FP32>(logits, row_bytes, budget, vocab, rows, n_nodes,
                                                   st, u, tokens, probs, stream);
}

}  // namespace taps

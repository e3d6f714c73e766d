// Per-head RMSNorm of new queries and keys, rotary positions and the cache write in one pass
// (qk_rope_paged).
//
// x' = x * rsqrt(mean x^2 + eps) * w per head; pair j of a head turns by pos * f_j:
// (a, b) -> m (a cos - b sin), m (b cos + a sin).  Pairs are (j, j + rot / 2) or (2j, 2j + 1); the
// head's dims from rot on are not turned.  V is copied.
//
// A head is HD / 8 lanes of 8 values each, two runs of four: (half layout) the runs 4j.. and
// rot / 2 + 4j.. of the four pairs 4j..4j+3, or eight neighbours, so that both values of a pair sit
// in one lane and the lane's four angles are the same for every head.  A wave takes 64 / (HD / 8)
// heads at a time, all heads (Q, K and V) of its row with one set of angles.
//
// Angles are formed in 64 bits, in turns: a position of 2^20 times a frequency leaves an fp32
// product no better than 2^-4 of a radian.  The reduced angle (|x| <= pi / 4, off by 2^-25) goes
// through the Taylor series of sine and cosine to x^11 and x^10 (remainders below 2^-33).
//
// Bound: HBM, everything is read and written once.
#include <algorithm>

#include "common.h"

namespace taps {
namespace {

typedef float f32x4 __attribute__((ext_vector_type(4)));
typedef uint32_t u32x4 __attribute__((ext_vector_type(4)));
typedef uint32_t u32x2 __attribute__((ext_vector_type(2)));

constexpr int kThreads = 256;
constexpr int kWaves = kThreads / kWave;

struct RopeArgs {
  const unsigned char *Q, *K, *V;
  int64_t qs, ks, vs;   // row strides in bytes
  const int32_t* pos;
  const int64_t* slots;
  const double* freq;
  const void *qw, *kw;
  unsigned char *Qo, *Kp, *Vp;
  int64_t pool_rows;
  float eps, mscale;
  int rows, Hq, Hkv, rot;
};

// four values in memory: raw words
template <typename T>
struct Quad;
template <>
struct Quad<__bf16> {
  typedef u32x2 raw;
  static __device__ inline void widen(const raw& r, float* x) {
    x[0] = __uint_as_float(r[0] << 16);
    x[1] = __uint_as_float(r[0] & 0xFFFF0000u);
    x[2] = __uint_as_float(r[1] << 16);
    x[3] = __uint_as_float(r[1] & 0xFFFF0000u);
  }
  static __device__ inline raw narrow(const float* x) {   // to nearest, ties to even
    typedef __bf16 bf16x4 __attribute__((ext_vector_type(4)));
    bf16x4 b;
#pragma unroll
    for (int t = 0; t < 4; ++t) b[t] = (__bf16)x[t];
    return __builtin_bit_cast(raw, b);
  }
};
template <>
struct Quad<float> {
  typedef u32x4 raw;
  static __device__ inline void widen(const raw& r, float* x) {
#pragma unroll
    for (int t = 0; t < 4; ++t) x[t] = __uint_as_float(r[t]);
  }
  static __device__ inline raw narrow(const float* x) {
    return raw{__float_as_uint(x[0]), __float_as_uint(x[1]), __float_as_uint(x[2]),
               __float_as_uint(x[3])};
  }
};

template <int CTRL>
__device__ inline float dpp_add(float x) {
  return x + __uint_as_float(__builtin_amdgcn_update_dpp(0u, __float_as_uint(x), CTRL, 0xf, 0xf,
                                                         true));
}
// sum over the LPH (8 or 16) lanes of a head, in each of them
template <int LPH>
__device__ inline float head_sum(float x) {
  x = dpp_add<0xB1>(x);    // lane ^ 1
  x = dpp_add<0x4E>(x);    // lane ^ 2
  x = dpp_add<0x141>(x);   // the other four of eight
  if constexpr (LPH == 16) x = dpp_add<0x140>(x);   // the other eight of sixteen
  return x;
}

// m cos and m sin of pos * f, f in turns per position
__device__ inline void turn(double pos, double f, float m, float& c, float& s) {
  const double r = pos * f;
  const double q = (r - __builtin_rint(r)) * 4.0;   // quarter turns, |q| <= 2
  const double k = __builtin_rint(q);
  const float x = (float)((q - k) * 1.5707963267948966);
  const float z = x * x;
  // x^(2i+1) / (2i+1)! and x^(2i) / (2i)!
  float sn = fmaf(z, -1.f / 39916800.f, 1.f / 362880.f);
  sn = fmaf(z, sn, -1.f / 5040.f);
  sn = fmaf(z, sn, 1.f / 120.f);
  sn = fmaf(z, sn, -1.f / 6.f);
  sn = fmaf(x * z, sn, x);
  float cs = fmaf(z, -1.f / 3628800.f, 1.f / 40320.f);
  cs = fmaf(z, cs, -1.f / 720.f);
  cs = fmaf(z, cs, 1.f / 24.f);
  cs = fmaf(z, cs, -0.5f);
  cs = fmaf(z, cs, 1.f);
  const int n = (int)k;
  const float a = (n & 1) ? cs : sn, b = (n & 1) ? sn : cs;
  s = m * ((n & 2) ? -a : a);
  c = m * (((n + 1) & 2) ? -b : b);
}

template <typename T, int HD, bool INTERLEAVED>
__global__ __launch_bounds__(kThreads) void rope_kernel(const RopeArgs A, int per_row) {
  using Qd = Quad<T>;
  typedef typename Qd::raw raw;
  constexpr int LPH = HD / 8, HPW = kWave / LPH;
  constexpr int CH = 4;   // heads of a lane whose loads are in flight together
  const int lane = threadIdx.x & (kWave - 1), j = lane % LPH, hl = lane / LPH;
  const int rq = A.rot / 4;
  const bool turned = j < rq / 2;
  // first dims of the lane's two runs
  const int d0 = INTERLEAVED ? 8 * j : turned ? 4 * j : A.rot + 8 * (j - rq / 2);
  const int d1 = !INTERLEAVED && turned ? A.rot / 2 + 4 * j : d0 + 4;
  const int heads = A.Hq + 2 * A.Hkv, passes = (heads + HPW - 1) / HPW;

  double f[4];
#pragma unroll
  for (int t = 0; t < 4; ++t)
    f[t] = turned ? A.freq[4 * j + t] * 0.15915494309189535 : 0.0;   // 1 / (2 pi)
  float qw[8], kw[8];
  auto weights = [&](const void* w, float* x) {
    if (!w) return;
    Qd::widen(*(const raw*)((const T*)w + d0), x);
    Qd::widen(*(const raw*)((const T*)w + d1), x + 4);
  };
  weights(A.qw, qw);
  weights(A.kw, kw);

  // a row's passes are dealt to per_row waves
  const int wave = __builtin_amdgcn_readfirstlane((int)threadIdx.x / kWave);
  const int64_t units = (int64_t)A.rows * per_row, step = (int64_t)gridDim.x * kWaves;
  for (int64_t u = (int64_t)blockIdx.x * kWaves + wave; u < units; u += step) {
    const int row = (int)(u / per_row), part = (int)(u - (int64_t)row * per_row);
    const int p0 = (int)((int64_t)passes * part / per_row);
    const int p1 = (int)((int64_t)passes * (part + 1) / per_row);
    const int64_t slot = A.slots[row];
    const bool keep = slot >= 0 && slot < A.pool_rows;
    const double pos = (double)A.pos[row];
    const unsigned char* const q = A.Q + (size_t)row * A.qs;
    const unsigned char* const k = A.K + (size_t)row * A.ks;
    const unsigned char* const v = A.V + (size_t)row * A.vs;
    float c[4], s[4];
    bool first = true;
    for (int p = p0; p < p1; p += CH) {
      raw x0[CH] = {}, x1[CH] = {};
#pragma unroll
      for (int i = 0; i < CH; ++i) {
        const int h = (p + i) * HPW + hl;
        if (p + i < p1 && h < heads) {
          const int kind = h < A.Hq ? 0 : h < A.Hq + A.Hkv ? 1 : 2;
          const int hh = kind == 0 ? h : kind == 1 ? h - A.Hq : h - A.Hq - A.Hkv;
          const T* const src = (const T*)(kind == 0 ? q : kind == 1 ? k : v) + (size_t)hh * HD;
          x0[i] = *(const raw*)(src + d0);
          x1[i] = *(const raw*)(src + d1);
        }
      }
      if (first) {   // under the first loads
        first = false;
#pragma unroll
        for (int t = 0; t < 4; ++t) turn(pos, f[t], A.mscale, c[t], s[t]);
      }
#pragma unroll
      for (int i = 0; i < CH; ++i) {
        const int h = (p + i) * HPW + hl;
        const bool in = p + i < p1 && h < heads;
        const int kind = h < A.Hq ? 0 : h < A.Hq + A.Hkv ? 1 : 2;
        const int hh = kind == 0 ? h : kind == 1 ? h - A.Hq : h - A.Hq - A.Hkv;
        float x[8];
        Qd::widen(x0[i], x);
        Qd::widen(x1[i], x + 4);
        float sq = 0.f;
#pragma unroll
        for (int t = 0; t < 8; ++t) sq = fmaf(x[t], x[t], sq);
        const float ms = fmaf(head_sum<LPH>(sq), 1.f / HD, A.eps);
        float rs = __builtin_amdgcn_rsqf(ms);
        // one Newton step: the instruction alone is off by a unit in the last place
        const float e = fmaf(-ms * rs, rs, 1.f);
        rs = e == e && e < 1.f ? fmaf(0.5f * rs, e, rs) : rs;   // (not of 0 and infinity)
        const bool norm = kind == 0 ? A.qw != nullptr : A.kw != nullptr;
        if (norm) {
#pragma unroll
          for (int t = 0; t < 8; ++t) x[t] = x[t] * rs * (kind == 0 ? qw[t] : kw[t]);
        }
        if (turned) {
#pragma unroll
          for (int t = 0; t < 4; ++t) {
            const int a = INTERLEAVED ? 2 * t : t, b = INTERLEAVED ? 2 * t + 1 : 4 + t;
            const float xa = x[a], xb = x[b];
            x[a] = fmaf(xa, c[t], -xb * s[t]);
            x[b] = fmaf(xb, c[t], xa * s[t]);
          }
        }
        T* dst;
        if (kind == 0) dst = (T*)A.Qo + ((size_t)row * A.Hq + hh) * HD;
        else dst = (T*)(kind == 1 ? A.Kp : A.Vp) + ((size_t)slot * A.Hkv + hh) * HD;
        if (in && (kind == 0 || keep)) {
          *(raw*)(dst + d0) = kind == 2 ? x0[i] : Qd::narrow(x);
          *(raw*)(dst + d1) = kind == 2 ? x1[i] : Qd::narrow(x + 4);
        }
      }
    }
  }
}

template <typename T, int HD>
hipError_t launch_t(const RopeArgs& A, int interleaved, hipStream_t s) {
  const int passes = (A.Hq + 2 * A.Hkv + kWave / (HD / 8) - 1) / (kWave / (HD / 8));
  // few rows: a row's heads over several waves
  const int per_row = std::min(passes, std::max(1, 2048 / A.rows));
  const int64_t units = (int64_t)A.rows * per_row;
  const unsigned grid = (unsigned)std::min<int64_t>((units + kWaves - 1) / kWaves, 2048);
  if (interleaved) rope_kernel<T, HD, true><<<grid, kThreads, 0, s>>>(A, per_row);
  else rope_kernel<T, HD, false><<<grid, kThreads, 0, s>>>(A, per_row);
  return hipGetLastError();
}

}  // namespace

hipError_t launch_rope(const void* Q, const void* K, const void* V, int64_t q_stride_bytes,
                       int64_t k_stride_bytes, int64_t v_stride_bytes, const int32_t* pos,
                       const int64_t* slots, int rows, int Hq, int Hkv, int head_dim, int dtype,
                       const taps_rope& r, void* Qo, void* Kp, void* Vp, int64_t pool_rows,
                       hipStream_t s) {
  if (rows <= 0) return hipSuccess;
  RopeArgs A;
  A.Q = (const unsigned char*)Q, A.K = (const unsigned char*)K, A.V = (const unsigned char*)V;
  A.qs = q_stride_bytes, A.ks = k_stride_bytes, A.vs = v_stride_bytes;
  A.pos = pos, A.slots = slots, A.freq = r.inv_freq, A.qw = r.q_norm, A.kw = r.k_norm;
  A.Qo = (unsigned char*)Qo, A.Kp = (unsigned char*)Kp, A.Vp = (unsigned char*)Vp;
  A.pool_rows = pool_rows, A.eps = r.norm_eps, A.mscale = r.mscale;
  A.rows = rows, A.Hq = Hq, A.Hkv = Hkv, A.rot = r.rot_dim;
  if (dtype == TAPS_BF16)
    return head_dim == 128 ? launch_t<__bf16, 128>(A, r.interleaved, s)
                           : launch_t<__bf16, 64>(A, r.interleaved, s);
  return head_dim == 128 ? launch_t<float, 128>(A, r.interleaved, s)
                         : launch_t<float, 64>(A, r.interleaved, s);
}

}  // namespace taps

// Per-head RMSNorm of new queries and keys, rotary positions and the cache write in one pass
// (qk_rope_paged).
//
// x' = x * rsqrt(mean x^2 + eps) * w per head; pair j of a head turns by pos * f_j:
// (a, b) -> m (a cos - b sin), m (b cos + a sin).  Pairs are (j, j + rot / 2) or (2j, 2j + 1); the
// head's dims from rot on are not turned.  V is copied.
//
// A lane holds 2 RUN values of a head in two runs: (half layout) RUN * j.. and rot / 2 + RUN * j..
// of the pairs RUN * j.., or neighbours, so that both values of a pair sit in one lane and the
// lane's RUN angles are the same for every head.  A run is 16 bytes where the rotated part is whole
// runs of them, else (bf16, rot_dim not a multiple of 16) 8.  A wave takes as many heads of one
// kind (Q, K or V) at a time as fit, all heads of its row with one set of angles.
//
// Angles are formed in 64 bits, in turns: a position of 2^20 times a frequency leaves an fp32
// product no better than 2^-4 of a radian.  The reduced angle (|x| <= pi / 4, off by 2^-25) goes
// through the Taylor series of sine and cosine to x^11 and x^10 (remainders below 2^-33).
//
// The norm takes heads of any size: where the mean square leaves 2^-100 .. 2^100 (values near the
// ends of the type's range, an eps of almost nothing) the head is scaled by a power of two first.
//
// Bound: HBM, everything is read and written once.  16,384 rows of 32/8 heads of 128 in bf16 (403
// MB) take 83 us, 4.8 TB/s (a copy of 2 GB: 5.0); 2047 rows of 16/2 heads of 64 in fp32 (21 MB) 7.7
// us.
// Single tokens: latency, 5 us.
#include <algorithm>

#include "common.h"

namespace taps {
namespace {

typedef uint32_t u32x4 __attribute__((ext_vector_type(4)));

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

// a run in memory: raw words
template <typename T, int RUN>
struct Run;
template <int RUN>
struct Run<__bf16, RUN> {
  typedef uint32_t raw __attribute__((ext_vector_type(RUN / 2)));
  static __device__ inline void widen(const raw& r, float* x) {
#pragma unroll
    for (int t = 0; t < RUN / 2; ++t) {
      x[2 * t] = __uint_as_float(r[t] << 16);
      x[2 * t + 1] = __uint_as_float(r[t] & 0xFFFF0000u);
    }
  }
  static __device__ inline raw narrow(const float* x) {   // to nearest, ties to even
    typedef __bf16 bf16xn __attribute__((ext_vector_type(RUN)));
    bf16xn b;
#pragma unroll
    for (int t = 0; t < RUN; ++t) b[t] = (__bf16)x[t];
    return __builtin_bit_cast(raw, b);
  }
};
template <>
struct Run<float, 4> {
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
__device__ inline float dpp(float x) {
  return __uint_as_float(__builtin_amdgcn_update_dpp(0u, __float_as_uint(x), CTRL, 0xf, 0xf, true));
}
// f over the LPH (4, 8 or 16) lanes of a head, the same in each of them
template <int LPH, typename F>
__device__ inline float over_head(float x, F f) {
  x = f(x, dpp<0xB1>(x));    // lane ^ 1
  x = f(x, dpp<0x4E>(x));    // lane ^ 2
  if constexpr (LPH >= 8) x = f(x, dpp<0x141>(x));    // the other four of eight
  if constexpr (LPH == 16) x = f(x, dpp<0x140>(x));   // the other eight of sixteen
  return x;
}
// eps + the mean of a head's squares, EPL values a lane
template <int HD, int EPL>
__device__ inline float mean_square(const float* x, float eps) {
  float sq = 0.f;
#pragma unroll
  for (int t = 0; t < EPL; ++t) sq = fmaf(x[t], x[t], sq);
  sq = over_head<HD / EPL>(sq, [](float a, float b) { return a + b; });
  return fmaf(sq, 1.f / HD, eps);
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

template <typename T, int HD, bool INTERLEAVED, int RUN>
__global__ __launch_bounds__(kThreads) void rope_kernel(const RopeArgs A, int per_row) {
  using Rn = Run<T, RUN>;
  typedef typename Rn::raw raw;
  constexpr int EPL = 2 * RUN, LPH = HD / EPL, HPW = kWave / LPH;
  constexpr int CH = 3;   // passes whose loads are in flight together
  const int lane = threadIdx.x & (kWave - 1), j = lane % LPH, hl = lane / LPH;
  const bool turned = j < A.rot / EPL;
  // first dims of the lane's two runs
  const int d0 = INTERLEAVED ? EPL * j : turned ? RUN * j : A.rot + EPL * (j - A.rot / EPL);
  const int d1 = !INTERLEAVED && turned ? A.rot / 2 + RUN * j : d0 + RUN;
  // passes over the heads of Q, K and V
  const int nq = (A.Hq + HPW - 1) / HPW, nk = (A.Hkv + HPW - 1) / HPW, passes = nq + 2 * nk;

  double f[RUN];
#pragma unroll
  for (int t = 0; t < RUN; ++t)
    f[t] = turned ? A.freq[RUN * j + t] * 0.15915494309189535 : 0.0;   // 1 / (2 pi)
  raw w[2][2] = {};
#pragma unroll
  for (int i = 0; i < 2; ++i) {
    const T* const nw = (const T*)(i == 0 ? A.qw : A.kw);
    if (nw) w[i][0] = *(const raw*)(nw + d0), w[i][1] = *(const raw*)(nw + d1);
  }

  // a row's passes are dealt to per_row waves
  const int wave = __builtin_amdgcn_readfirstlane((int)threadIdx.x / kWave);
  const int64_t units = (int64_t)A.rows * per_row, step = (int64_t)gridDim.x * kWaves;
  for (int64_t u = (int64_t)blockIdx.x * kWaves + wave; u < units; u += step) {
    int row = (int)u, p0 = 0, p1 = passes;
    if (per_row > 1) {
      row = (int)u / per_row;   // (few rows)
      const int part = (int)u - row * per_row;
      p0 = passes * part / per_row, p1 = passes * (part + 1) / per_row;
    }
    const int64_t slot = A.slots[row];
    const bool keep = slot >= 0 && slot < A.pool_rows;
    const double pos = (double)A.pos[row];
    float c[RUN], s[RUN];
    bool first = true;
    for (int p = p0; p < p1; p += CH) {
      raw x0[CH], x1[CH];
#pragma unroll
      for (int i = 0; i < CH; ++i) {
        const int q = min(p + i, p1 - 1);   // (past the last: the same again, not stored)
        const int kind = q < nq ? 0 : q < nq + nk ? 1 : 2;
        const unsigned char* const base = kind == 0   ? A.Q + (size_t)row * A.qs
                                          : kind == 1 ? A.K + (size_t)row * A.ks
                                                      : A.V + (size_t)row * A.vs;
        const int h = (kind == 0 ? q : kind == 1 ? q - nq : q - nq - nk) * HPW + hl;
        const uint32_t at = (uint32_t)min(h, (kind == 0 ? A.Hq : A.Hkv) - 1) * HD;
        x0[i] = *(const raw*)((const T*)base + (at + d0));
        x1[i] = *(const raw*)((const T*)base + (at + d1));
      }
      if (first) {   // under the first loads
        first = false;
#pragma unroll
        for (int t = 0; t < RUN; ++t) turn(pos, f[t], A.mscale, c[t], s[t]);
      }
#pragma unroll
      for (int i = 0; i < CH; ++i) {
        if (p + i >= p1) break;
        const int q = p + i, kind = q < nq ? 0 : q < nq + nk ? 1 : 2;
        const int h = (kind == 0 ? q : kind == 1 ? q - nq : q - nq - nk) * HPW + hl;
        const bool in = h < (kind == 0 ? A.Hq : A.Hkv) && (kind == 0 || keep);
        if (kind != 2) {
          float x[EPL];
          Rn::widen(x0[i], x);
          Rn::widen(x1[i], x + RUN);
          if (kind == 0 ? A.qw != nullptr : A.kw != nullptr) {
            float ms = mean_square<HD, EPL>(x, A.eps);
            // squares beyond 32 bits, or so small that they lose theirs: the head and the root of
            // eps by a power of two near 1 (the norm does not depend on it)
            const bool far = !(ms > 0x1p-100f && ms < 0x1p100f);
            if (__ballot(far)) {
              float mx = 0.f;
#pragma unroll
              for (int t = 0; t < EPL; ++t) mx = fmaxf(mx, fabsf(x[t]));
              mx = over_head<LPH>(mx, [](float a, float b) { return fmaxf(a, b); });
              int e = __builtin_amdgcn_frexp_expf(mx);   // (0 of 0, infinity and NaN)
              if (A.eps > 0.f) {
                const int half = (__builtin_amdgcn_frexp_expf(A.eps) + 1) >> 1;
                e = mx > 0.f ? max(e, half) : half;
              }
              e = far ? e : 0;
#pragma unroll
              for (int t = 0; t < EPL; ++t) x[t] = __builtin_ldexpf(x[t], -e);
              ms = mean_square<HD, EPL>(x, __builtin_ldexpf(A.eps, -2 * e));
            }
            float rs = __builtin_amdgcn_rsqf(ms);
            // one Newton step: the instruction alone is off by a unit in the last place
            const float e = fmaf(-ms * rs, rs, 1.f);
            rs = e == e && e < 1.f ? fmaf(0.5f * rs, e, rs) : rs;   // (not of 0 and infinity)
            float g[EPL];
            Rn::widen(kind == 0 ? w[0][0] : w[1][0], g);
            Rn::widen(kind == 0 ? w[0][1] : w[1][1], g + RUN);
#pragma unroll
            for (int t = 0; t < EPL; ++t) x[t] = x[t] * rs * g[t];
          }
          if (turned) {
#pragma unroll
            for (int t = 0; t < RUN; ++t) {
              const int a = INTERLEAVED ? 2 * t : t, b = INTERLEAVED ? 2 * t + 1 : RUN + t;
              const float xa = x[a], xb = x[b];
              x[a] = fmaf(xa, c[t], -xb * s[t]);
              x[b] = fmaf(xb, c[t], xa * s[t]);
            }
          }
          x0[i] = Rn::narrow(x);
          x1[i] = Rn::narrow(x + RUN);
        }
        unsigned char* const base =
            kind == 0 ? A.Qo + (size_t)row * A.Hq * (HD * sizeof(T))
                      : (kind == 1 ? A.Kp : A.Vp) + (size_t)slot * A.Hkv * (HD * sizeof(T));
        if (in) {
          const uint32_t at = (uint32_t)h * HD;
          *(raw*)((T*)base + (at + d0)) = x0[i];
          *(raw*)((T*)base + (at + d1)) = x1[i];
        }
      }
    }
  }
}

template <typename T, int HD, int RUN>
hipError_t launch_t(const RopeArgs& A, int interleaved, hipStream_t s) {
  constexpr int HPW = kWave / (HD / (2 * RUN));
  const int passes = (A.Hq + HPW - 1) / HPW + 2 * ((A.Hkv + HPW - 1) / HPW);
  // few rows: a row's passes over several waves, each of which forms the row's angles (us of 600,
  // 1024 and 2047 rows of 32/8 heads of 128 with up to 2048 / 4096 / 8192 waves: 6.5 / 8.2 / 8.2,
  // 8.3 / 9.7 / 11.9, 11.8 / 12.3 / 15.6; of 64 rows 4.2)
  const int per_row = std::min(passes, std::max(1, 2048 / A.rows));
  const int64_t units = (int64_t)A.rows * per_row;
  const unsigned grid = (unsigned)std::min<int64_t>((units + kWaves - 1) / kWaves, 2048);
  if (interleaved) rope_kernel<T, HD, true, RUN><<<grid, kThreads, 0, s>>>(A, per_row);
  else rope_kernel<T, HD, false, RUN><<<grid, kThreads, 0, s>>>(A, per_row);
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
  const int il = r.interleaved;
  if (dtype == TAPS_FP32)
    return head_dim == 128 ? launch_t<float, 128, 4>(A, il, s) : launch_t<float, 64, 4>(A, il, s);
  if (r.rot_dim % 16 == 0)
    return head_dim == 128 ? launch_t<__bf16, 128, 8>(A, il, s) : launch_t<__bf16, 64, 8>(A, il, s);
  return head_dim == 128 ? launch_t<__bf16, 128, 4>(A, il, s) : launch_t<__bf16, 64, 4>(A, il, s);
}

}  // namespace taps

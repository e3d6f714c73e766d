// Attention of one new token per request over a paged KV cache (decode_attn_paged).
//
// O[b,h] = softmax_j(scale * q_bh . k_jg) v_jg over the request's rows j < kv_len[b], g = h / G,
// G = Hq / Hkv.  One pass with the running maximum and sum of the softmax.  The requests' rows,
// one after the other in units of 128 keys, are cut into equal parts, one per workgroup that
// the chip holds at once (for each KV head and group of 16 of its query heads): every workgroup
// has the same work whatever the lengths are, and reads it to the end without a pause.  A part
// may end inside a request; such pieces leave (O, max, sum), which a second kernel adds.  The
// four waves of a workgroup deal a unit's 32-key tiles among themselves.
//
// A wave's tile, in registers only (bf16):
//   * S^T = K Q^T on v_mfma_f32_16x16x32_bf16, two blocks of 16 keys: lane (g = l / 16, c =
//     l % 16) holds 8 dims of key c and of query head c, and ends with the scores of head c
//     for the keys 16 i + 4 g + 0..3;
//   * O^T += V^T P^T: the lane's eight probabilities are the eight k-values of its lane in the
//     B operand if k-value j of group g is key 16 (j / 4) + 4 g + j % 4.  The A operand then
//     wants those eight keys of one dim: the lane loads HD / 16 consecutive dims (from
//     c * HD / 16) of each of the eight rows, whole rows per 16 lanes, and transposes the
//     block in registers (one v_perm_b32 for two values).  Row m of block t is dim
//     m * HD / 16 + t.
// fp32: the same layout on v_mfma_f32_16x16x4_f32, a score or probability a k-value.
// P enters the second product as two bf16 values, the rounded weight and what the rounding
// left: the matrix instructions have room, and one bf16 (an error of 2^-9 of each weight)
// made up most of the outputs' error.
//
// Bound: HBM (K and V are read once; a group of more than 16 query heads reads them once per 16):
// 128 requests of 512-32K keys (64/8 heads of 128, bf16) 742 us, 5.5 TB/s (of 64: 405, 5.0); 16 of
// 512-16K (32/8) 67 us, 4.5 TB/s, 59 where the last-level cache keeps what it holds of them; fp32,
// 64 of 512-8K (32/8 of 128) 249 us, 5.8 TB/s.  Short batches: latency, two launches and the dependent reads of lengths, page
// ids, keys and pieces (one request of 8192 keys 12.7 us; its bytes take 6.3).
#include <algorithm>

#include "common.h"
#include "scan.h"

namespace taps {
namespace {

typedef float f32x4 __attribute__((ext_vector_type(4)));
typedef uint32_t u32x4 __attribute__((ext_vector_type(4)));
typedef uint32_t u32x2 __attribute__((ext_vector_type(2)));
typedef __bf16 bf16x8 __attribute__((ext_vector_type(8)));

constexpr int kWaves = 4;
constexpr int kThreads = kWaves * kWave;
constexpr int kHeads = 16;   // query heads per workgroup
constexpr int kTile = 32;    // keys per tile: a divisor of every page

// max and sum over the four lanes that share l % 16, in each of them
__device__ inline float quad_max(float x) {
  auto a = __builtin_amdgcn_permlane16_swap(__float_as_uint(x), __float_as_uint(x), false, false);
  x = fmaxf(__uint_as_float(a[0]), __uint_as_float(a[1]));
  a = __builtin_amdgcn_permlane32_swap(__float_as_uint(x), __float_as_uint(x), false, false);
  return fmaxf(__uint_as_float(a[0]), __uint_as_float(a[1]));
}
__device__ inline float quad_sum(float x) {
  auto a = __builtin_amdgcn_permlane16_swap(__float_as_uint(x), __float_as_uint(x), false, false);
  x = __uint_as_float(a[0]) + __uint_as_float(a[1]);
  a = __builtin_amdgcn_permlane32_swap(__float_as_uint(x), __float_as_uint(x), false, false);
  return __uint_as_float(a[0]) + __uint_as_float(a[1]);
}

// weight 2^((m - M) * scale) of a part whose reference score is m (none: 0)
__device__ inline float part_weight(float m, float M, float scale_log2) {
  return m == -INFINITY ? 0.f : __builtin_amdgcn_exp2f((m - M) * scale_log2);
}

// The operands of one tile and its two products.  load_k / load_v: p is the tile's first row
// of this KV head (uniform), rs the row stride in elements.
template <typename T, int HD>
struct Tile;

template <int HD>
struct Tile<__bf16, HD> {
  static constexpr int NKK = HD / 32;
  static constexpr int DPL = HD / 16;   // V dims per lane and key
  bf16x8 q[NKK];
  bf16x8 k[2][NKK];
  uint32_t v[8][DPL / 2];

  __device__ inline void load_q(const __bf16* p, bool in) {
    const int g = (threadIdx.x & (kWave - 1)) >> 4;
#pragma unroll
    for (int kk = 0; kk < NKK; ++kk) {
      const u32x4 z = {0u, 0u, 0u, 0u};
      const u32x4 x = in ? *(const u32x4*)(p + 32 * kk + 8 * g) : z;
      q[kk] = __builtin_bit_cast(bf16x8, x);
    }
  }
  __device__ inline void load_k(const __bf16* p, uint32_t rs) {
    const int lane = threadIdx.x & (kWave - 1), c = lane & 15, g = lane >> 4;
#pragma unroll
    for (int i = 0; i < 2; ++i)
#pragma unroll
      for (int kk = 0; kk < NKK; ++kk)
        k[i][kk] = *(const bf16x8*)(p + (uint32_t)((16 * i + c) * rs + 32 * kk + 8 * g));
  }
  __device__ inline void load_v(const __bf16* p, uint32_t rs) {
    const int lane = threadIdx.x & (kWave - 1), c = lane & 15, g = lane >> 4;
#pragma unroll
    for (int j = 0; j < 8; ++j) {
      const __bf16* r = p + (uint32_t)((16 * (j >> 2) + 4 * g + (j & 3)) * rs + DPL * c);
      if constexpr (DPL == 8) {
        const u32x4 x = *(const u32x4*)r;
#pragma unroll
        for (int t = 0; t < 4; ++t) v[j][t] = x[t];
      } else {
        const u32x2 x = *(const u32x2*)r;
        v[j][0] = x[0];
        v[j][1] = x[1];
      }
    }
  }
  // keys from `have` on hold nothing of the request
  __device__ inline void clear_v(int have) {
    const int g = (threadIdx.x & (kWave - 1)) >> 4;
#pragma unroll
    for (int j = 0; j < 8; ++j)
#pragma unroll
      for (int t = 0; t < DPL / 2; ++t)
        v[j][t] = 16 * (j >> 2) + 4 * g + (j & 3) < have ? v[j][t] : 0u;
  }
  __device__ inline void scores(f32x4 (&s)[2]) const {
#pragma unroll
    for (int i = 0; i < 2; ++i) {
      s[i] = f32x4{0.f, 0.f, 0.f, 0.f};
#pragma unroll
      for (int kk = 0; kk < NKK; ++kk)
        s[i] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(k[i][kk], q[kk], s[i], 0, 0, 0);
    }
  }
  __device__ inline void accumulate(const float (&p)[8], f32x4 (&o)[DPL]) const {
    bf16x8 hi, lo;
#pragma unroll
    for (int j = 0; j < 8; ++j) {
      hi[j] = (__bf16)p[j];
      lo[j] = (__bf16)(p[j] - (float)hi[j]);
    }
#pragma unroll
    for (int t = 0; t < DPL; ++t) {
      u32x4 a;
#pragma unroll
      for (int w = 0; w < 4; ++w)   // (key 2w, key 2w + 1) of dim t
        a[w] = __builtin_amdgcn_perm(v[2 * w + 1][t >> 1], v[2 * w][t >> 1],
                                     (t & 1) ? 0x07060302u : 0x05040100u);
      const bf16x8 av = __builtin_bit_cast(bf16x8, a);
      o[t] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(av, hi, o[t], 0, 0, 0);
      o[t] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(av, lo, o[t], 0, 0, 0);
    }
  }
};

template <int HD>
struct Tile<float, HD> {
  static constexpr int J = HD / 16;
  static constexpr int DPL = HD / 16;
  f32x4 q[J];
  f32x4 k[2][J];
  f32x4 v[8][DPL / 4];

  __device__ inline void load_q(const float* p, bool in) {
    const int g = (threadIdx.x & (kWave - 1)) >> 4;
#pragma unroll
    for (int j = 0; j < J; ++j) {
      const f32x4 z = {0.f, 0.f, 0.f, 0.f};
      q[j] = in ? *(const f32x4*)(p + 16 * j + 4 * g) : z;
    }
  }
  __device__ inline void load_k(const float* p, uint32_t rs) {
    const int lane = threadIdx.x & (kWave - 1), c = lane & 15, g = lane >> 4;
#pragma unroll
    for (int i = 0; i < 2; ++i)
#pragma unroll
      for (int j = 0; j < J; ++j)
        k[i][j] = *(const f32x4*)(p + (uint32_t)((16 * i + c) * rs + 16 * j + 4 * g));
  }
  __device__ inline void load_v(const float* p, uint32_t rs) {
    const int lane = threadIdx.x & (kWave - 1), c = lane & 15, g = lane >> 4;
#pragma unroll
    for (int j = 0; j < 8; ++j)
#pragma unroll
      for (int u = 0; u < DPL / 4; ++u)
        v[j][u] = *(const f32x4*)(p + (uint32_t)((16 * (j >> 2) + 4 * g + (j & 3)) * rs +
                                                 DPL * c + 4 * u));
  }
  __device__ inline void clear_v(int have) {
    const int g = (threadIdx.x & (kWave - 1)) >> 4;
#pragma unroll
    for (int j = 0; j < 8; ++j)
#pragma unroll
      for (int u = 0; u < DPL / 4; ++u)
#pragma unroll
        for (int t = 0; t < 4; ++t)
          v[j][u][t] = 16 * (j >> 2) + 4 * g + (j & 3) < have ? v[j][u][t] : 0.f;
  }
  // four partial sums per score: chains a quarter as long round less
  __device__ inline void scores(f32x4 (&s)[2]) const {
#pragma unroll
    for (int i = 0; i < 2; ++i) {
      f32x4 sp[4];
#pragma unroll
      for (int e = 0; e < 4; ++e) sp[e] = f32x4{0.f, 0.f, 0.f, 0.f};
#pragma unroll
      for (int j = 0; j < J; ++j)
#pragma unroll
        for (int e = 0; e < 4; ++e)
          sp[e] = __builtin_amdgcn_mfma_f32_16x16x4f32(k[i][j][e], q[j][e], sp[e], 0, 0, 0);
      s[i] = (sp[0] + sp[1]) + (sp[2] + sp[3]);
    }
  }
  __device__ inline void accumulate(const float (&p)[8], f32x4 (&o)[DPL]) const {
#pragma unroll
    for (int j = 0; j < 8; ++j)
#pragma unroll
      for (int t = 0; t < DPL; ++t)
        o[t] = __builtin_amdgcn_mfma_f32_16x16x4f32(v[j][t / 4][t % 4], p[j], o[t], 0, 0, 0);
  }
};

__device__ inline void store4(float* p, const f32x4& x) { *(f32x4*)p = x; }
__device__ inline void store4(__bf16* p, const f32x4& x) {
  typedef __bf16 bf16x4 __attribute__((ext_vector_type(4)));
  bf16x4 r;
#pragma unroll
  for (int t = 0; t < 4; ++t) r[t] = (__bf16)x[t];
  *(bf16x4*)p = r;
}

constexpr int kUnit = kWaves * kTile;   // keys: a tile per wave

__device__ inline int len_of(const int32_t* lenp, int b, int max_len) {
  return min(max(lenp[b], 0), max_len);
}
__device__ inline int units_of(int len) { return (len + kUnit - 1) / kUnit; }

__device__ inline int wave_scan(int v) { return (int)wave_scan_u32((uint32_t)v); }

// first unit of part j when `total` units are cut into `parts`
__device__ inline int part_begin(int j, int total, int parts) {
  return (int)((int64_t)j * total / parts);
}

// Scratch of a call whose requests are cut: first unit of each request ([batch + 1]), then two
// pieces per workgroup (the one that begins inside a request, the one that begins a request
// and does not end it): O [kHeads][HD], (max, sum) [kHeads]
struct DecodeWs {
  int32_t* first;
  float* O;
  float2* ML;
};

// Workgroup (part j, KV head, head tile); parts 0: one workgroup per (request, KV head, tile).
template <typename T, int HD>
__global__ __launch_bounds__(kThreads) void decode_kernel(
    const T* __restrict__ Q, int64_t q_stride, const T* __restrict__ Kp, const T* __restrict__ Vp,
    const PagedKV pk, const int32_t* __restrict__ lenp, int batch, int Hq, int Hkv, int max_len,
    float scale_log2, int parts, int htiles, int groups, T* __restrict__ O, const DecodeWs ws) {
  constexpr int DPL = HD / 16;
  constexpr int OROW = HD + 4;   // LDS row stride of the waves' outputs
  __shared__ float s_o[kWaves][kHeads][OROW];
  __shared__ float s_m[kWaves][kHeads], s_l[kWaves][kHeads];

  // the head tiles of a (part, KV head) are 8 block ids apart: one XCD, whose L2 then holds its
  // keys; the KV heads of a part run side by side and read the same rows
  const int xcd = blockIdx.x & 7, slot = (int)((blockIdx.y * gridDim.x + blockIdx.x) >> 3);
  const int group = (slot / htiles) * 8 + xcd, ht = slot % htiles;
  if (group >= groups) return;
  const int kvh = group % Hkv, part = group / Hkv;
  const int G = Hq / Hkv, h0 = ht * kHeads, heads = min(G - h0, kHeads);
  const int tid = threadIdx.x, lane = tid & (kWave - 1), c = lane & 15, g = lane >> 4;
  const int wave = __builtin_amdgcn_readfirstlane(tid / kWave);
  const uint32_t rs = (uint32_t)Hkv * HD;
  const int slot_mask = (1 << pk.page_shift) - 1;
  const int head = kvh * G + h0 + min(c, heads - 1);
  Tile<T, HD> tile;

  // this workgroup's units: from unit u of request b on, `left` of them
  int b = part, u = 0, left = 0;
  if (parts == 0) {
    left = units_of(len_of(lenp, b, max_len));
    if (left == 0) {   // an empty request: zeros
      for (int i = tid; i < heads * (HD / 4); i += kThreads)
        store4(O + ((size_t)b * Hq + kvh * G + h0) * HD + 4 * i, f32x4{0.f, 0.f, 0.f, 0.f});
      return;
    }
  } else {
    // the units of 64 requests at a time; the first 64 are read once
    auto units_at = [&](int b0) {
      return b0 + lane < batch ? units_of(len_of(lenp, b0 + lane, max_len)) : 0;
    };
    const int n0 = units_at(0), incl0 = wave_scan(n0);
    int total = __builtin_amdgcn_readlane(incl0, kWave - 1);
    for (int b0 = kWave; b0 < batch; b0 += kWave)
      total += __builtin_amdgcn_readlane(wave_scan(units_at(b0)), kWave - 1);
    parts = min(parts, total);   // none of them empty
    const int begin = part < parts ? part_begin(part, total, parts) : 0;
    if (part < parts) left = part_begin(part + 1, total, parts) - begin;
    // the first workgroup leaves the requests' first units for the second kernel
    const bool first = group == 0 && ht == 0 && wave == 0;
    if (left == 0 && !first) return;
    int before = 0;
    b = -1;
    for (int b0 = 0; b0 < batch && (b < 0 || first); b0 += kWave) {
      const int n = b0 == 0 ? n0 : units_at(b0), incl = b0 == 0 ? incl0 : wave_scan(n);
      if (first && b0 + lane < batch) ws.first[b0 + lane] = before + incl - n;
      const uint64_t hit = __ballot(before + incl > begin);
      if (b < 0 && hit) {
        const int l = __ffsll((long long)hit) - 1;
        b = b0 + l;
        u = begin - (before + __builtin_amdgcn_readlane(incl - n, l));
      }
      before += __builtin_amdgcn_readlane(incl, kWave - 1);
    }
    if (first && lane == 0) ws.first[batch] = total;
    if (left == 0) return;
  }

  while (true) {   // pieces: the units of one request
    const int len = len_of(lenp, b, max_len);
    const int n = min(units_of(len) - u, left);
    const int k_begin = u * kUnit, k_end = min(k_begin + n * kUnit, len);
    const int32_t* const bt = pk.btab + (size_t)b * pk.max_pages;
    tile.load_q(Q + (size_t)b * q_stride + (size_t)head * HD, c < heads);

    // Reference maxima stay in score units (before the scale): the exponent is (s - m) * scale,
    // whose rounding error falls with the weight of the term.
    f32x4 o[DPL];
#pragma unroll
    for (int t = 0; t < DPL; ++t) o[t] = f32x4{0.f, 0.f, 0.f, 0.f};
    float m_ref = -INFINITY, l_run = 0.f;
    for (int k0 = k_begin + wave * kTile; k0 < k_end; k0 += kUnit) {
      const int page = min(max(bt[k0 >> pk.page_shift], 0), pk.num_pages - 1);
      const size_t row = ((size_t)page << pk.page_shift) + (k0 & slot_mask);
      tile.load_k(Kp + row * rs + kvh * HD, rs);
      tile.load_v(Vp + row * rs + kvh * HD, rs);
      f32x4 s[2];
      tile.scores(s);
      const int have = k_end - k0;   // rows past the request are the page's, not its own
      if (have < kTile) {
#pragma unroll
        for (int i = 0; i < 2; ++i)
#pragma unroll
          for (int r = 0; r < 4; ++r) s[i][r] = 16 * i + 4 * g + r < have ? s[i][r] : -INFINITY;
        tile.clear_v(have);
      }
      const float mx = quad_max(fmaxf(fmaxf(fmaxf(s[0][0], s[0][1]), fmaxf(s[0][2], s[0][3])),
                                      fmaxf(fmaxf(s[1][0], s[1][1]), fmaxf(s[1][2], s[1][3]))));
      const bool upd = (mx - m_ref) * scale_log2 > 8.f;   // move the reference by > 2^8 only
      if (__ballot(upd)) {
        const float nref = upd ? mx : m_ref;
        const float alpha = upd ? part_weight(m_ref, nref, scale_log2) : 1.f;
        l_run *= alpha;
#pragma unroll
        for (int t = 0; t < DPL; ++t) o[t] *= alpha;
        m_ref = nref;
      }
      const float mu = m_ref == -INFINITY ? 0.f : m_ref;
      float p[8];
#pragma unroll
      for (int j = 0; j < 8; ++j)
        p[j] = __builtin_amdgcn_exp2f((s[j >> 2][j & 3] - mu) * scale_log2);
      l_run += ((p[0] + p[1]) + (p[2] + p[3])) + ((p[4] + p[5]) + (p[6] + p[7]));
      tile.accumulate(p, o);
    }
    l_run = quad_sum(l_run);

    // ---- merge the waves: row r of output block t is dim (4 g + r) * DPL + t of head c
    {
      float* dst = &s_o[wave][c][g * (4 * DPL)];
#pragma unroll
      for (int r = 0; r < 4; ++r)
#pragma unroll
        for (int q = 0; q < DPL / 4; ++q)
          *(f32x4*)(dst + r * DPL + 4 * q) =
              f32x4{o[4 * q][r], o[4 * q + 1][r], o[4 * q + 2][r], o[4 * q + 3][r]};
      if (g == 0) {
        s_m[wave][c] = m_ref;
        s_l[wave][c] = l_run;
      }
    }
    __syncthreads();
    constexpr int TPR = HD / 4;   // threads per head, four dims each
    const bool whole = k_begin == 0 && k_end == len;
    const size_t piece =
        whole ? 0 : (((size_t)group * htiles + ht) * 2 + (k_begin == 0 ? 1 : 0)) * kHeads;
    for (int r = tid / TPR; r < heads; r += kThreads / TPR) {
      const int d = (tid % TPR) * 4;
      float M = -INFINITY, L = 0.f;
#pragma unroll
      for (int w = 0; w < kWaves; ++w) M = fmaxf(M, s_m[w][r]);
      f32x4 acc = {0.f, 0.f, 0.f, 0.f};
#pragma unroll
      for (int w = 0; w < kWaves; ++w) {
        const float l = s_l[w][r];
        const float a = part_weight(s_m[w][r], M, scale_log2);
        if (s_m[w][r] != -INFINITY) {   // else a wave without keys (or its scores are all NaN)
          L += a * l;
          acc += a * *(const f32x4*)&s_o[w][r][d];
        }
        if (l != l) L = l;              // a NaN score moves no maximum
      }
      if (whole) {
        store4(O + ((size_t)b * Hq + kvh * G + h0 + r) * HD + d, acc / L);
      } else {
        *(f32x4*)(ws.O + (piece + r) * HD + d) = acc;
        if (d == 0) ws.ML[piece + r] = make_float2(M, L);
      }
    }
    left -= n;
    if (left == 0) return;
    u = 0;
    do ++b;
    while (units_of(len_of(lenp, b, max_len)) == 0);   // `left` units are still to come
    __syncthreads();   // the merge is read before the next one is written
  }
}

// Adds the pieces of the requests that were cut: a workgroup per (request, query head), four
// dims per thread and a share of the pieces per group of HD / 4 threads.  Empty requests get
// zeros here.
constexpr int kCombineThreads = 256;
template <typename T, int HD>
__global__ __launch_bounds__(kCombineThreads) void decode_combine_kernel(
    const DecodeWs ws, int batch, int Hq, int Hkv, float scale_log2, int parts, int htiles,
    T* __restrict__ O) {
  constexpr int TPR = HD / 4, GROUPS = kCombineThreads / TPR;
  __shared__ f32x4 s_acc[GROUPS][TPR];
  __shared__ float s_m[GROUPS], s_l[GROUPS];
  const int h = blockIdx.x, b = blockIdx.y, G = Hq / Hkv, kvh = h / G;
  const int ht = (h - kvh * G) / kHeads, r = (h - kvh * G) % kHeads;
  const int grp = threadIdx.x / TPR, tr = threadIdx.x % TPR, d = tr * 4;
  const int u0 = ws.first[b], u1 = ws.first[b + 1], total = ws.first[batch];
  T* const out = O + ((size_t)b * Hq + h) * HD + d;
  if (u0 == u1) {
    if (grp == 0) store4(out, f32x4{0.f, 0.f, 0.f, 0.f});
    return;
  }
  // the parts that hold units u0 and u1 - 1
  parts = min(parts, total);
  const int j0 = (int)(((int64_t)(u0 + 1) * parts - 1) / total);
  const int j1 = (int)(((int64_t)u1 * parts - 1) / total);
  if (j0 == j1) return;   // written whole
  auto piece = [&](int j) -> size_t {
    return ((((size_t)j * Hkv + kvh) * htiles + ht) * 2 + (j == j0 ? 1 : 0)) * kHeads + r;
  };
  float M = -INFINITY, L = 0.f;
  f32x4 acc = {0.f, 0.f, 0.f, 0.f};
  constexpr int CH = 8;   // pieces whose loads are in flight together
  for (int s0 = j0 + grp; s0 <= j1; s0 += CH * GROUPS) {
    float2 ml[CH];
    f32x4 x[CH];
#pragma unroll
    for (int k = 0; k < CH; ++k) {
      const size_t p = piece(min(s0 + k * GROUPS, j1));
      ml[k] = ws.ML[p];
      x[k] = *(const f32x4*)(ws.O + p * HD + d);
    }
    float Mc = M;
#pragma unroll
    for (int k = 0; k < CH; ++k) Mc = fmaxf(Mc, ml[k].x);
    const float a = part_weight(M, Mc, scale_log2);
    L *= a;
    acc *= a;
#pragma unroll
    for (int k = 0; k < CH; ++k) {
      if (s0 + k * GROUPS > j1) continue;
      if (ml[k].x != -INFINITY) {
        const float w = part_weight(ml[k].x, Mc, scale_log2);
        L += w * ml[k].y;
        acc += w * x[k];
      }
      if (ml[k].y != ml[k].y) L = ml[k].y;
    }
    M = Mc;
  }
  s_acc[grp][tr] = acc;
  if (tr == 0) s_m[grp] = M, s_l[grp] = L;
  __syncthreads();
  if (grp != 0) return;
  float Mc = -INFINITY;
#pragma unroll
  for (int w = 0; w < GROUPS; ++w) Mc = fmaxf(Mc, s_m[w]);
  L = 0.f;
  acc = f32x4{0.f, 0.f, 0.f, 0.f};
#pragma unroll
  for (int w = 0; w < GROUPS; ++w) {
    const float l = s_l[w];
    if (s_m[w] != -INFINITY) {
      const float a = part_weight(s_m[w], Mc, scale_log2);
      L += a * l;
      acc += a * s_acc[w][tr];
    }
    if (l != l) L = l;
  }
  store4(out, acc / L);
}

DecodeWs ws_of(void* ws, const DecodePlan& p, int batch, int Hkv, int head_dim) {
  DecodeWs w;
  w.first = (int32_t*)ws;
  w.O = (float*)((char*)ws + (((size_t)batch + 1) * sizeof(int32_t) + 255) / 256 * 256);
  w.ML = (float2*)(w.O + (size_t)p.parts * Hkv * p.htiles * 2 * kHeads * head_dim);
  return w;
}

template <typename T, int HD>
hipError_t launch_t(const void* Q, int64_t q_stride, const void* K, const void* V,
                    const PagedKV& pk, const int32_t* len, int batch, int Hq, int Hkv,
                    int max_len, float scale, const DecodePlan& p, void* O, void* ws,
                    hipStream_t s) {
  const int groups = (p.parts ? p.parts : batch) * Hkv;
  const float sl2 = scale * 1.4426950408889634f;
  const DecodeWs w = p.parts ? ws_of(ws, p, batch, Hkv, HD) : DecodeWs{};
  // the blocks in rows of at most 2^22 (a multiple of 8: the XCD stays blockIdx.x % 8)
  const int64_t blocks = 8ll * p.htiles * ((groups + 7) / 8);
  const int64_t gx = std::min<int64_t>(blocks, 1ll << 22);
  decode_kernel<T, HD><<<dim3((unsigned)gx, (unsigned)((blocks + gx - 1) / gx)), kThreads, 0, s>>>(
      (const T*)Q, q_stride, (const T*)K, (const T*)V, pk, len, batch, Hq, Hkv, max_len, sl2,
      p.parts, p.htiles, groups, (T*)O, w);
  const hipError_t e = hipGetLastError();
  if (e != hipSuccess || p.parts == 0) return e;
  decode_combine_kernel<T, HD><<<dim3((unsigned)Hq, (unsigned)batch), kCombineThreads, 0, s>>>(
      w, batch, Hq, Hkv, sl2, p.parts, p.htiles, (T*)O);
  return hipGetLastError();
}

}  // namespace

// Equal parts for two workgroups per CU.  us a call with 256 / 512 / 768 / 1024 workgroups, from
// graphs over the same inputs: 128 requests of 512-32K keys (64/8 heads of 128, bf16) 720 / 741 / 756 / 752, 16 of
// 512-16K (32/8) 60 / 58 / 62 / 65, 64 of 256-4K 83 / 80 / 81 / 89, 256 of 64-2K 150 / 137 / 142
// / 152, 8 of 512-8K in fp32 (32/8 of 128) 40 / 36 / 41 / 42, one of 8K 12.9 / 12.7 / 12.6 / 12.7.
// One workgroup per (request, KV head, head tile) without the second kernel instead where all
// requests are short, or many and rather short.  At the borders, us a call without / with the
// second kernel (max_len one more; other inputs every call): 256 keys: one request (32/8 heads of
// 128) 6.2 / 9.0, 63 of 128-256 15 / 20, 8 in fp32 13 / 13; 1024 keys: 64 requests of 64-300 15 /
// 19, of 512-1024 47 / 52, 256 of 64-1024 94 / 94, 512 of 64-1024 (4/1 of 64) 20 / 25, 300 (34/1 of
// 128) 33 / 45, but 64 of 64-1024 in fp32 66 / 52.  By the batch: 63 of 64-1024 32 with the second
// kernel, 64 of them 35 without; 256 of 64-2K 137 with, 151 without.  max_len is the host's
// bound: short requests under a long one take the cut all the same (64 of 64-300: 19).
DecodePlan plan_decode(int batch, int Hq, int Hkv, int max_len) {
  DecodePlan p;
  p.htiles = (Hq / Hkv + kHeads - 1) / kHeads;
  const int64_t heads = (int64_t)Hkv * p.htiles;
  const bool whole = max_len <= 2 * kUnit || (batch * heads >= 512 && max_len <= 1024);
  p.parts = whole ? 0 : (int)std::max<int64_t>(1, 512 / heads);
  return p;
}

size_t decode_ws_bytes(const DecodePlan& p, int batch, int Hkv, int head_dim) {
  if (p.parts == 0) return 0;
  const DecodeWs w = ws_of(nullptr, p, batch, Hkv, head_dim);
  return (size_t)(uintptr_t)(w.ML + (size_t)p.parts * Hkv * p.htiles * 2 * kHeads);
}

hipError_t launch_decode(const void* Q, int64_t q_stride, const void* K, const void* V,
                         const PagedKV& pk, const int32_t* len, int batch, int Hq, int Hkv,
                         int head_dim, int max_len, int dtype, float scale, const DecodePlan& p,
                         void* O, void* ws, hipStream_t s) {
  if (batch <= 0) return hipSuccess;
  if (dtype == TAPS_BF16)
    return head_dim == 128 ? launch_t<__bf16, 128>(Q, q_stride, K, V, pk, len, batch, Hq, Hkv,
                                                   max_len, scale, p, O, ws, s)
                           : launch_t<__bf16, 64>(Q, q_stride, K, V, pk, len, batch, Hq, Hkv,
                                                  max_len, scale, p, O, ws, s);
  return head_dim == 128 ? launch_t<float, 128>(Q, q_stride, K, V, pk, len, batch, Hq, Hkv,
                                                max_len, scale, p, O, ws, s)
                         : launch_t<float, 64>(Q, q_stride, K, V, pk, len, batch, Hq, Hkv, max_len,
                                               scale, p, O, ws, s);
}

}  // namespace taps

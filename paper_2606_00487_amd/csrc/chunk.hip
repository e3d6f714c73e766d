// Attention of chunks of new tokens over a paged KV cache (chunk_attn_paged).
//
// Request b brings n new tokens; its cache holds kv rows, theirs the last n.  Token i is at
// position p = kv - n + i and sees the rows j <= p (within a window: p - window < j <= p):
// O[i,h] = softmax_j(scale * q_ih . k_jg) v_jg.  The query rows of a KV head are the tokens x the
// G query heads that share it, in tiles of M rows; keys go by in tiles of 64.
//
// Pieces.  A workgroup takes the keys of one (KV head, query tile), or a part of them: no piece of
// a tile that is cut has more than L units of 64 keys, L = all tiles' units / 256 (or 512), so that
// a few long requests fill the chip as well as many short ones.  The requests' lengths are device
// data: every workgroup forms L and finds its piece from prefix sums over the batch, or, of many
// requests, in an index that a first kernel writes.  Pieces of a tile that was cut leave (O, max,
// sum) in fp32, which a second kernel adds.
//
// bf16 (v_mfma_f32_32x32x16_bf16): eight waves (short prompts and head_dim 64: four) of 32 query
// rows each share the key tile.  S^T = K Q^T (A: keys from LDS, B: queries in registers) leaves a
// query's scores in two lanes; they go, as P^T, straight into the B operand of O^T += V^T P^T,
// whose key order follows the accumulators; the transposing LDS read takes V in that order.  K and
// V cycle through rings of three tiles (V of two where two workgroups are to share a CU), filled by
// loads straight into LDS two tiles ahead; S of the next tile is issued between this one's softmax
// and products, each matrix instruction among the vector and LDS instructions of the other part.
// Bound: the matrix instructions (4 head_dim flops a visible pair and head) and, for few rows over
// a long cache, HBM.  head_dim 128, 32/8 heads: a prompt of 16,384 tokens takes 1.88 ms, 1167
// TFLOP/s (a library product of 8192^3: 1219).  A step of 64 keys takes 3500 cycles of which the
// SIMD's matrix instructions fill 2048, at the clock of 1.86 GHz that the card holds under it; the
// library's product keeps them busier at 1.5 GHz, to the same product of the two.  16 tokens over
// 32,768 keys: 33 us, 4.1 TB/s with the join.  A piece costs 5.4 us besides its steps (finding it
// 1.0, its pages 1.4, the first tile 1.3, the first scores 0.4, its end 1.1), which bounds ragged
// batches; at head_dim 64 the vector unit (32 exponentials a step) is the fuller one.
// fp32 (v_mfma_f32_16x16x4_f32): four waves of 16 query rows, key tiles of 32 staged through
// registers, bound by the fp32 matrix instructions: a prompt of 2048 tokens, 32/8 heads of 128, 370
// us, 93 TFLOP/s (a library product: 145); 40 % of the LDS's active cycles are bank conflicts, 9 %
// of all (source not traced).  128 rows a tile take 352 us there, and 41 for 47 us for 16 tokens
// over 8K, but 254 for 225 us for 8 ragged requests.
#include <algorithm>
#include <climits>

#include "common.h"
#include "ldsload.h"
#include "scan.h"

namespace taps {
namespace {

typedef __bf16 bf16x8 __attribute__((ext_vector_type(8)));
typedef __bf16 bf16x4 __attribute__((ext_vector_type(4)));
typedef __bf16 bf16x2 __attribute__((ext_vector_type(2)));
typedef float f32x16 __attribute__((ext_vector_type(16)));
typedef float f32x4 __attribute__((ext_vector_type(4)));

constexpr int kUnit = 64;      // keys per unit of a piece's length

constexpr int kMF = 64;        // query rows of an fp32 tile; 128 or 256 in bf16

struct ChunkArgs {
  const unsigned char *Q, *K, *V;
  int64_t q_stride;   // elements
  PagedKV pk;
  const int32_t *q_start, *kv_len;
  int batch, rows, Hq, Hkv, max_len, window;
  float scale_log2;
  ChunkCut cut;
  unsigned char* O;
  float* wsO;     // [slots][M][HD]; null: no piece is cut
  float2* wsML;   // [slots][M]
  int slots;
  const int4* index;   // many requests: where each begins
};

// Most key units that one of a request's tiles sees of kv rows: with a window, the keys of a tile's
// first to last token's, wherever they begin in a unit
template <int M>
__device__ inline int units_of(const ChunkArgs& A, int kv, int G) {
  const int units = (kv + kUnit - 1) / kUnit;
  if (A.window <= 0) return units;
  const int64_t span = (int64_t)A.window + (M + G - 2) / G;
  return (int)min((int64_t)units, (span + kUnit - 2) / kUnit + 1);
}
// One request's share: n new tokens (rows q0 ..), kv rows, query tiles and units_of
struct Request {
  int q0, n, kv, tiles, units;
};
template <int M>
__device__ inline Request request_of(const ChunkArgs& A, int b, int G) {   // b >= batch: none
  const int at = min(b, A.batch - 1);
  const int q0 = A.q_start[at], q1 = A.q_start[at + 1], kv = A.kv_len[at];
  Request r;
  r.q0 = min(max(q0, 0), A.rows);
  r.n = b < A.batch ? max(min(max(q1, 0), A.rows) - r.q0, 0) : 0;
  r.kv = b < A.batch ? min(max(kv, 0), A.max_len) : 0;
  r.tiles = (int)(((int64_t)r.n * G + M - 1) / M);
  r.units = units_of<M>(A, r.kv, G);
  return r;
}

__device__ inline int64_t wave_scan_i64(int64_t v) { return (int64_t)wave_scan_u64((uint64_t)v); }
__device__ inline int64_t lane_i64(int64_t v, int l) { return (int64_t)lane_u64((uint64_t)v, l); }

// Key units per piece at most: the sum of tiles * units over the batch, times the KV heads, in
// `target` parts
__device__ inline int units_per_piece(const ChunkArgs& A, int64_t total) {
  const int64_t L = (total * A.Hkv + (1 << A.cut.target_log2) - 1) >> A.cut.target_log2;
  return (int)max((int64_t)A.cut.min_units, min(L, (int64_t)1 << 30));
}
// ... and the pieces of a tile of the request
__device__ inline int splits_of(const ChunkArgs& A, int units, int L) {
  return units - A.cut.gain > L ? (units + L - 1) / L : 1;
}

// Piece `item` of the batch (without the KV head), item counting the requests' tiles * splits.  The
// order within a request: splits, then its tiles from the last one, which sees the most keys.
// ROWS > 0: instead group `item` of ROWS query rows of the requests that are cut.
struct Piece {
  int b, q0, n, kv, tile, split, splits, L;
  int slot;    // of the tile's first split; splits of a tile are `tiles` apart
  int tiles;
  int group;   // ROWS > 0: the request's group of rows
  bool found;
};
constexpr int kWhole = 1 << 30;   // L where nothing is cut
// what a request has of the pieces and of the second kernel's groups of rows
struct Share {
  int splits;
  int64_t pieces, cut, groups;
};
__device__ inline Share share_of(const ChunkArgs& A, const Request& r, int L, int G, int rows) {
  Share h;
  h.splits = splits_of(A, r.units, L);
  h.pieces = (int64_t)r.tiles * h.splits;
  h.cut = h.splits > 1 ? h.pieces : 0;
  h.groups = h.splits > 1 ? (r.n * G + rows - 1) / rows : 0;
  return h;
}
// the `at`-th piece or group of a request
template <int M, int ROWS>
__device__ inline Piece piece_of(const Request& r, int b, int splits, int L, int at, int slot) {
  Piece p{};
  p.b = b, p.q0 = r.q0, p.n = r.n, p.kv = r.kv, p.tiles = r.tiles, p.splits = splits;
  p.L = splits > 1 ? L : kWhole;
  if constexpr (ROWS > 0) {
    p.group = at;
    p.tile = at / (M / ROWS);
  } else {
    p.split = splits == 1 ? 0 : at / p.tiles;
    p.tile = p.tiles - 1 - (at - p.split * p.tiles);
  }
  p.slot = slot + p.tile;
  p.found = true;
  return p;
}
template <int M, int ROWS>
__device__ inline Piece find_piece(const ChunkArgs& A, int G, int item) {
  const int lane = threadIdx.x & (kWave - 1);
  constexpr int rows = ROWS > 0 ? ROWS : 1;
  if (A.batch == 1) {   // no sums, all of it uniform
    const Request r = request_of<M>(A, 0, G);
    const int L = A.wsO ? units_per_piece(A, (int64_t)r.tiles * r.units) : kWhole;
    const Share h = share_of(A, r, L, G, rows);
    if (item >= (ROWS > 0 ? h.groups : h.pieces)) return Piece{};
    return piece_of<M, ROWS>(r, 0, h.splits, L, item, 0);
  }
  if (A.index == nullptr) {   // a request per lane at a time
    Request r = request_of<M>(A, lane, G);
    int L = kWhole;
    if (A.wsO) {
      int64_t total = lane_i64(wave_scan_i64((int64_t)r.tiles * r.units), kWave - 1);
      for (int b0 = kWave; b0 < A.batch; b0 += kWave) {
        const Request o = request_of<M>(A, b0 + lane, G);
        total += lane_i64(wave_scan_i64((int64_t)o.tiles * o.units), kWave - 1);
      }
      L = units_per_piece(A, total);
    }
    int64_t before = 0, cut_before = 0;
    for (int b0 = 0; b0 < A.batch; b0 += kWave) {
      if (b0 > 0) r = request_of<M>(A, b0 + lane, G);
      const Share h = share_of(A, r, L, G, rows);
      const int64_t count = ROWS > 0 ? h.groups : h.pieces;
      const int64_t incl = before + wave_scan_i64(count);
      const int64_t cut = cut_before + wave_scan_i64(h.cut);
      const uint64_t hit = __ballot(incl > item);
      if (hit) {
        const int l = __ffsll((long long)hit) - 1;
        auto of = [&](int x) { return (int)__builtin_amdgcn_readlane(x, l); };
        const Request q{of(r.q0), of(r.n), of(r.kv), of(r.tiles), of(r.units)};
        return piece_of<M, ROWS>(q, b0 + l, of(h.splits), L,
                                 item - (int)lane_i64(incl - count, l),
                                 (int)lane_i64(cut - h.cut, l));
      }
      before = lane_i64(incl, kWave - 1), cut_before = lane_i64(cut, kWave - 1);
    }
    return Piece{};
  }
  // the last request that begins at or before the item
  const int* const begins = (const int*)A.index + (ROWS > 0 ? 2 : 0);
  const int4 end = A.index[A.batch];
  if (item >= (ROWS > 0 ? end.z : end.x)) return Piece{};
  int b = 0;
  for (int n = A.batch; n > 1;) {
    const int step = (n + kWave - 1) / kWave;
    const bool in = lane * step < n;
    const int v = begins[(size_t)4 * (b + (in ? lane * step : 0))];
    const int k = __popcll(__ballot(in && v <= item)) - 1;
    b += k * step;
    n = min(step, n - k * step);
  }
  const int4 e = A.index[b];
  const Request r = request_of<M>(A, b, G);
  auto first = [](int x) { return (int)__builtin_amdgcn_readfirstlane(x); };
  const Request q{first(r.q0), first(r.n), first(r.kv), first(r.tiles), first(r.units)};
  return piece_of<M, ROWS>(q, b, first(e.w), first(end.w), item - first(ROWS > 0 ? e.z : e.x),
                           first(e.y));
}

// More than 256 requests (up to there every workgroup adds up the batch itself, 64 at a time):
// where each begins, [batch + 1] of (pieces, pieces of cut tiles, groups of `group_rows` rows of
// the second kernel, its splits; last: the sums and L).  One workgroup, 3 us.  us with / without,
// requests of 1 to 16 tokens over 100 to 1000 keys, 32/8 heads of 128: 100 requests 54 / 51, 256
// 123 / 123, 1024 438 / 730, 4096 1723 / 6930.
constexpr int kIndexThreads = 1024;
template <int M>
__global__ __launch_bounds__(kIndexThreads) void chunk_index_kernel(const ChunkArgs A,
                                                                    int group_rows, int4* index) {
  __shared__ int64_t s_sum[kIndexThreads / kWave];
  const int tid = threadIdx.x, lane = tid & (kWave - 1), wave = tid / kWave;
  const int G = A.Hq / A.Hkv;
  // inclusive sum over the workgroup's threads; total: over all of them
  auto scan = [&](int64_t v, int64_t& total) {
    const int64_t incl = wave_scan_i64(v);
    __syncthreads();
    if (lane == kWave - 1) s_sum[wave] = incl;
    __syncthreads();
    int64_t before = 0;
    total = 0;
#pragma unroll
    for (int w = 0; w < kIndexThreads / kWave; ++w) {
      if (w < wave) before += s_sum[w];
      total += s_sum[w];
    }
    return before + incl;
  };
  int L = kWhole;
  if (A.wsO) {
    int64_t sum = 0, total;
    for (int b = tid; b < A.batch; b += kIndexThreads) {
      const Request r = request_of<M>(A, b, G);
      sum += (int64_t)r.tiles * r.units;
    }
    scan(sum, total);
    L = units_per_piece(A, total);
  }
  // (starts that decrease name rows more than once: any number of pieces, of which the grid runs
  // the first; those that L cuts are few even so)
  int64_t begin = 0, others = 0;   // others: cut pieces and, in the upper half, groups
  for (int b0 = 0; b0 < A.batch; b0 += kIndexThreads) {
    const int b = b0 + tid;
    const Share h = share_of(A, request_of<M>(A, b, G), L, G, group_rows);
    const int64_t both = h.cut | h.groups << 32;
    int64_t total, total_others;
    const int64_t at = begin + scan(h.pieces, total) - h.pieces;
    const int64_t o = others + scan(both, total_others) - both;
    if (b < A.batch)
      index[b] = make_int4((int)min(at, (int64_t)INT_MAX), (int)o, (int)(o >> 32), h.splits);
    begin += total, others += total_others;
  }
  if (tid == 0)
    index[A.batch] = make_int4((int)min(begin, (int64_t)INT_MAX), (int)others,
                               (int)(others >> 32), L);
}

// Keys [lo, hi) that the tokens t0 .. t1 of a request see between them
__device__ inline void key_range(const ChunkArgs& A, const Piece& p, int t0, int t1, int& lo,
                                 int& hi) {
  const int base = p.kv - p.n;
  hi = max(base + t1 + 1, 0);
  lo = A.window > 0 ? max(base + t0 - A.window + 1, 0) : 0;
}

// max and sum over a lane and the one 32 further
__device__ inline float pair_max(float x) {
  const auto r = __builtin_amdgcn_permlane32_swap(__float_as_uint(x), __float_as_uint(x), false,
                                                  false);
  return fmaxf(__uint_as_float(r[0]), __uint_as_float(r[1]));
}
__device__ inline float pair_sum(float x) {
  const auto r = __builtin_amdgcn_permlane32_swap(__float_as_uint(x), __float_as_uint(x), false,
                                                  false);
  return __uint_as_float(r[0]) + __uint_as_float(r[1]);
}

// permutation of a row's 16-byte chunk index: the 16 rows that an LDS read of K touches at once,
// and the four of V, land on distinct banks (rows of 16 chunks: all four bits of the row; of 8, of
// which two rows fill the banks: the upper three)
template <int HD>
__device__ inline int chunk_perm(int r) {
  if constexpr (HD == 128) return ((r & 3) << 2) | ((r >> 2) & 3);
  else return ((r & 2) << 1) | ((r >> 2) & 3);
}

// the order of a region's instructions: N times a matrix product, DS LDS reads, V vector and T
// transcendental instructions
template <int N, int DS, int V, int T>
__device__ __attribute__((always_inline)) inline void interleave() {
#pragma unroll
  for (int i = 0; i < N; ++i) {
    __builtin_amdgcn_sched_group_barrier(0x008, 1, 0);
    __builtin_amdgcn_sched_group_barrier(0x100, DS, 0);
    __builtin_amdgcn_sched_group_barrier(0x002, V, 0);
    __builtin_amdgcn_sched_group_barrier(0x400, T, 0);
  }
}
template <int P>
struct Slot {
  static constexpr int value = P;
};
// W waves, 32 query rows each; VR tiles of V in LDS
template <int HD, int W, int VR>
__global__ __launch_bounds__(64 * W) void chunk_bf16_kernel(const ChunkArgs A) {
#if defined(__HIP_DEVICE_COMPILE__)
  constexpr int M = 32 * W;
  constexpr int KT = 64;              // keys per tile
  constexpr int RING = 3;             // tiles of K in LDS
  constexpr int ROWB = HD * 2, CPR = ROWB / 16;   // bytes and 16-byte chunks of a row
  constexpr int TILEB = KT * ROWB;
  constexpr int NKK = HD / 16, NDB = HD / 32;
  constexpr int HW = W / 2;                       // waves that load K; the others load V
  constexpr int BPW = TILEB / 1024 / HW;          // 1 KB loads per wave and tile
  constexpr int BROWS = 1024 / ROWB;              // rows per load: 4 or 8
  typedef __attribute__((address_space(3))) bf16x4 lds_bf16x4;
  __shared__ __attribute__((aligned(1024))) unsigned char s_k[RING * TILEB], s_v[VR * TILEB];

  const int G = A.Hq / A.Hkv;
  const int kvh = blockIdx.x % A.Hkv;
  const Piece p = find_piece<M, 0>(A, G, blockIdx.x / A.Hkv);
  if (!p.found) return;
  const int tid = threadIdx.x, lane = tid & 63, l32 = lane & 31, hl = lane >> 5;
  const int wave = __builtin_amdgcn_readfirstlane(tid >> 6);
  const int last = p.n * G - 1;                   // last query row
  const int row0 = p.tile * M;
  int lo, hi;
  key_range(A, p, row0 / G, min(row0 + M - 1, last) / G, lo, hi);
  // this piece's key tiles [k0, k0 + nt * 64)
  const int u0 = lo / kUnit, u1 = (hi + kUnit - 1) / kUnit;
  const int ub = u0 + min((int64_t)p.split * p.L, (int64_t)(u1 - u0));
  const int ue = (int)min((int64_t)ub + p.L, (int64_t)u1);
  const bool cut = p.splits > 1;
  if (cut && ub >= ue && p.split > 0) return;     // the tile has no such piece
  const int nt = __builtin_amdgcn_readfirstlane(max(ue - ub, 0));
  const int k0 = __builtin_amdgcn_readfirstlane(ub * kUnit);
  const int k_end = __builtin_amdgcn_readfirstlane(min(hi, ue * kUnit));
  const int k_lo = __builtin_amdgcn_readfirstlane(lo);

  // this wave's query rows, tokens and positions
  const int wrow0 = row0 + wave * 32;
  const int qrow = min(wrow0 + l32, last);
  const int tok = qrow / G, head = kvh * G + (qrow - tok * G);
  const bool live = wrow0 + l32 <= last;
  const int base = p.kv - p.n;
  const int place = live ? base + tok : -1;
  const int pos = min(place, k_end - 1);                           // sees keys <= pos
  const int from = A.window > 0 ? place - A.window + 1 : 0;        // and >= from
  // (uniform) first and last position of the wave's rows
  const int pos_lo = __builtin_amdgcn_readfirstlane(min(base + wrow0 / G, k_end - 1));
  const int pos_hi = __builtin_amdgcn_readfirstlane(
      wrow0 <= last ? base + min(wrow0 + 31, last) / G : -1);
  const int from_hi = A.window > 0 ? pos_hi - A.window + 1 : 0;

  bf16x8 q[NKK];   // the lane's query: dims 16 kk + 8 hl ..

  // ---- direct loads.  The first half of the waves loads K, the second V; of each tile one half
  // (32 keys, in one page) per HW / 2 waves, BPW blocks of 1 KB each.  Lane l holds the page of
  // this wave's half of tile pw + l.
  const uint32_t rsb = (uint32_t)A.Hkv * ROWB;
  const bool loads_k = wave < HW;
  const int half = wave % HW / (HW / 2), block0 = wave % (HW / 2) * BPW;
  const int32_t* const bt = A.pk.btab + (size_t)p.b * A.pk.max_pages;
  auto entries = [&](int t0) {
    const int r = min(k0 + (t0 + lane) * KT + half * 32, k_end - 1);   // rows of the piece only
    const int e = min(max(r, 0) >> A.pk.page_shift, A.pk.max_pages - 1);
    return min(max(bt[e], 0), A.pk.num_pages - 1);
  };
  int pw = 0, pages = 0, pages_next = 0;
  if (nt > 0) pages = entries(0), pages_next = entries(64);
  const uint32_t lds0 = __builtin_amdgcn_readfirstlane(lds_address(loads_k ? s_k : s_v)) +
                        (uint32_t)(half * (TILEB / 2) + block0 * 1024);
  const uint64_t src0 = (uint64_t)((loads_k ? A.K : A.V) + (size_t)kvh * ROWB);
  uint32_t ld_off[BPW];
#pragma unroll
  for (int j = 0; j < BPW; ++j) {
    const int r = (block0 + j) * BROWS + lane / CPR;                   // row in the half tile
    ld_off[j] = (uint32_t)r * rsb + (uint32_t)(((lane % CPR) ^ chunk_perm<HD>(r)) * 16);
  }
  // `next` is the resource over the half tile that this wave loads next, `key` its first key: its
  // address is formed among the matrix products, far from the barrier that the loads follow.
  // Past the piece nothing is read from memory; rows before the first visible key read 0 too.
  i32x4 next = {0, 0, 0, 0};
  int key = 0;
  auto prepare = [&](int t) __attribute__((always_inline)) {
    if (t - pw >= 64) {
      pw += 64;
      pages = pages_next;
      pages_next = entries(pw + 64);
    }
    key = k0 + t * KT + half * 32;
    const int rows = min(max(k_end - key, 0), 32);
    const int pg = __builtin_amdgcn_readlane(pages, (t - pw) & 63);
    const uint64_t prow = ((uint64_t)(uint32_t)pg << A.pk.page_shift) |
                          (uint32_t)(key & ((1 << A.pk.page_shift) - 1));
    next = buffer_rsrc((const void*)(src0 + prow * rsb), (uint32_t)rows * rsb);
  };
  auto issue = [&](int slot) __attribute__((always_inline)) {
    if (key < k_lo) {
      int ln = lane;
      asm volatile("" : "+v"(ln));                // (rare: nothing of it is kept in registers)
#pragma unroll
      for (int j = 0; j < BPW; ++j) {
        const int r = (block0 + j) * BROWS + ln / CPR;
        const uint32_t off = key + r < k_lo ? 0x7FFFFF00u : ld_off[j];
        load_lds16_at(next, lds0 + slot * TILEB + j * 1024, off);
      }
    } else {
#pragma unroll
      for (int j = 0; j < BPW; ++j) load_lds16_at(next, lds0 + slot * TILEB + j * 1024, ld_off[j]);
    }
  };

  // ---- LDS read addresses in slot 0, opaque so that the slots are constant offsets
  typedef __attribute__((address_space(3))) unsigned char lds_u8;
  typedef __attribute__((address_space(3))) bf16x8 lds_bf16x8;
  const int fk = chunk_perm<HD>(l32);
  uint32_t koff[NKK];
#pragma unroll
  for (int kk = 0; kk < NKK; ++kk) {
    koff[kk] = (uint32_t)(uintptr_t)(lds_u8*)s_k + l32 * ROWB + 16 * ((2 * kk + hl) ^ fk);
    asm volatile("" : "+v"(koff[kk]));
  }
  const int g16 = (lane >> 4) & 1, tq = (lane & 15) >> 2, qq = lane & 3;
  uint32_t voff[2][NDB];
#pragma unroll
  for (int h8 = 0; h8 < 2; ++h8)
#pragma unroll
    for (int db = 0; db < NDB; ++db) {
      const int r = 8 * h8 + 4 * hl + tq;
      voff[h8][db] = (uint32_t)(uintptr_t)(lds_u8*)s_v + r * ROWB + 8 * (qq & 1) +
                     16 * ((4 * db + 2 * g16 + (qq >> 1)) ^ chunk_perm<HD>(r));
      asm volatile("" : "+v"(voff[h8][db]));
    }

  f32x16 o[NDB];
#pragma unroll
  for (int db = 0; db < NDB; ++db)
#pragma unroll
    for (int v = 0; v < 16; ++v) o[db][v] = 0.f;
  float m_ref = -INFINITY, m_thr = -INFINITY, m_neg = 0.f;
  float l_run = 0.f;
  const float thr8 = 8.f / A.scale_log2;

  // Operands wait in registers: each is replaced by the one four k-steps (V: 16 keys) on as soon as
  // its product has been issued.
  bf16x8 ka[4], va[NDB];
  auto read_k = [&](int slot, int i) __attribute__((always_inline)) {   // i: key block, k-step
    ka[i & 3] = *(const lds_bf16x8*)(koff[i % NKK] + (slot * TILEB + i / NKK * 32 * ROWB));
  };
  auto read_v = [&](int slot, int hf, int db) __attribute__((always_inline)) {
    const uint32_t at = slot * TILEB + 16 * hf * ROWB;
    const bf16x4 a = __builtin_amdgcn_ds_read_tr16_b64_v4bf16((lds_bf16x4*)(voff[0][db] + at));
    const bf16x4 b = __builtin_amdgcn_ds_read_tr16_b64_v4bf16((lds_bf16x4*)(voff[1][db] + at));
    va[db] = __builtin_shufflevector(a, b, 0, 1, 2, 3, 4, 5, 6, 7);
  };
  // k-steps [a, b) of the scores of key block kb
  auto scores = [&](int slot, int kb, int a, int b, f32x16& s) __attribute__((always_inline)) {
#pragma unroll
    for (int kk = a; kk < b; ++kk) {
      if (kk == 0) {
#pragma unroll
        for (int v = 0; v < 16; ++v) s[v] = 0.f;
      }
      const int i = kb * NKK + kk;
      s = __builtin_amdgcn_mfma_f32_32x32x16_bf16(ka[i & 3], q[kk], s, 0, 0, 0);
      if (i + 4 < 2 * NKK) read_k(slot, i + 4);
    }
  };
  auto largest = [&](const f32x16& s) __attribute__((always_inline)) {
    float x = s[0], y = s[1];
#pragma unroll
    for (int v = 2; v < 16; v += 2) x = fmaxf(x, s[v]), y = fmaxf(y, s[v + 1]);
    return fmaxf(x, y);
  };
  // the tile's largest score per query (m0: of the first key block)
  auto tile_max = [&](f32x16& s0, f32x16& s1, int key, float m0) __attribute__((always_inline)) {
    if (key + KT - 1 > pos_lo || key < from_hi) {
      const int a = pos - key - 4 * hl, f = from - key - 4 * hl;   // the lane's keys f .. a
#pragma unroll
      for (int v = 0; v < 16; ++v) {
        const int k = 8 * (v >> 2) + (v & 3);
        s0[v] = k <= a && k >= f ? s0[v] : -INFINITY;
        s1[v] = k + 32 <= a && k + 32 >= f ? s1[v] : -INFINITY;
      }
      m0 = largest(s0);
    }
    return pair_max(fmaxf(m0, largest(s1)));
  };
  // the reference moves only when exceeded by > 2^8
  auto rescale = [&](float mx) __attribute__((always_inline)) {
    const bool upd = mx > m_thr;
    if (__ballot(upd)) {
      const float nref = upd ? mx * A.scale_log2 : m_ref;
      const float alpha = upd ? __builtin_amdgcn_exp2f(m_ref - nref) : 1.f;
      m_thr = upd ? mx + thr8 : m_thr;
      l_run *= alpha;
#pragma unroll
      for (int db = 0; db < NDB; ++db)
#pragma unroll
        for (int v = 0; v < 16; ++v) o[db][v] *= alpha;
      m_ref = nref;
      m_neg = m_ref == -INFINITY ? 0.f : -m_ref;
    }
  };
  // the weights of 16 keys (8 in this lane), the first or second half of a key block.  Their sum
  // takes the rounded ones, as the product does.  One bf16 each: outputs are 2.0e-3 to 2.35e-3 off
  // 64 bits, 1.5e-3 to 1.7e-3 by the last rounding alone.  A second one for what the rounding
  // leaves, as in the decode kernel, is half as much again for the matrix unit, which bounds
  // prompts.  Few rows leave that unit idle, but their piece is one wave's chain of steps, which it
  // makes longer: us without, as a second product and in the columns that 16 rows leave free, of 16
  // tokens over 32K keys 34 / 39.6 / 42, one token over 8K 17 / 18.6 / 18.7, 16 requests of one
  // token over 512 to 16K 75 / 80 / 78 (heads of 64: 26 / 30.5 / 31, 13 / 14 / 14, 44 / 50 / 46.5).
  auto weights = [&](const f32x16& s, int hf) __attribute__((always_inline)) {
    bf16x8 w;
#pragma unroll
    for (int t = 0; t < 8; ++t)
      w[t] = (__bf16)__builtin_amdgcn_exp2f(
          fmaf(s[hf * 8 + t], A.scale_log2, m_neg));
    const bf16x2 one = {(__bf16)1.f, (__bf16)1.f};
#pragma unroll
    for (int t = 0; t < 8; t += 2)
      l_run = __builtin_amdgcn_fdot2_f32_bf16(bf16x2{w[t], w[t + 1]}, one, l_run, false);
    return w;
  };
  auto product = [&](int slot, int hf, const bf16x8& w) __attribute__((always_inline)) {
#pragma unroll
    for (int db = 0; db < NDB; ++db) {
      o[db] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(va[db], w, o[db], 0, 0, 0);
      if (hf < 3) read_v(slot, hf + 1, db);
    }
  };

  // Begin of step t (slot P = t mod 3): V(t) and K(t + 1) have landed (the wave's loads of one more
  // tile may be out).  The barrier also says that every wave has read K(t) and V(t - 1), whose
  // slots are filled next.  (VR 2: V(t) was its waves' last load, and V(t + 1) takes the slot of
  // V(t - 1))
  auto advance = [&]() __attribute__((always_inline)) {
    if (VR == 3 || loads_k) TAPS_WAIT_VMCNT(BPW);
    else TAPS_WAIT_VMCNT(0);
    TAPS_LDS_BARRIER();
  };
  const int ahead = loads_k ? 3 : VR - 1;        // tiles from a step's to the one it loads
  auto fill = [&](int P, int PV) __attribute__((always_inline)) {
    issue(loads_k ? P : (PV + VR - 1) % VR);
  };
  // Step t: the weights and products of tile t, from its scores (s0, s1; m0: the largest of s0),
  // and the scores of tile t + 1 (past the last one: of zeros) into n0 and, when they are used
  // up, s0.
  float m0 = -INFINITY;
  auto step = [&](auto pt, auto pv, int t, f32x16& s0, f32x16& s1, f32x16& n0)
                  __attribute__((always_inline)) {
    constexpr int P = decltype(pt)::value, PN = (P + 1) % 3, PV = decltype(pv)::value;
    advance();
#pragma unroll
    for (int i = 0; i < 4; ++i) read_k(PN, i);
#pragma unroll
    for (int db = 0; db < NDB; ++db) read_v(PV, 0, db);
    rescale(tile_max(s0, s1, k0 + t * KT, m0));
    __builtin_amdgcn_sched_barrier(0);
    const bf16x8 w0 = weights(s0, 0);
    scores(PN, 0, 0, NKK, n0);
    interleave<NKK, 1, 24 / NKK - 1, 1>();
    __builtin_amdgcn_sched_barrier(0);
    fill(P, PV);
    __builtin_amdgcn_sched_barrier(0);
    product(PV, 0, w0);
    const bf16x8 w1 = weights(s0, 1);
    interleave<NDB, 2, 16 / NDB, 8 / NDB>();
    __builtin_amdgcn_sched_barrier(0);
    product(PV, 1, w1);
    scores(PN, 1, 0, NKK / 2, s0);
    const bf16x8 w2 = weights(s1, 0);
    interleave<NDB + NKK / 2, 2, 2, 1>();
    __builtin_amdgcn_sched_barrier(0);
    prepare(t + 1 + ahead);
    __builtin_amdgcn_sched_barrier(0);
    product(PV, 2, w2);
    scores(PN, 1, NKK / 2, NKK, s0);
    const bf16x8 w3 = weights(s1, 1);
    asm volatile("" : "+v"(l_run));               // (the sum is not put off to the next step)
    interleave<NDB + NKK / 2, 2, 2, 1>();
    __builtin_amdgcn_sched_barrier(0);
    product(PV, 3, w3);
    m0 = largest(n0);
    asm volatile("" : "+v"(m0));
  };

  if (nt > 0) {
    // K(0) .. K(2), V(0), V(1)
    prepare(0);
    issue(0);
    {
      const __bf16* const qp =
          (const __bf16*)A.Q + (size_t)(p.q0 + tok) * A.q_stride + (size_t)head * HD;
#pragma unroll
      for (int kk = 0; kk < NKK; ++kk) q[kk] = *(const bf16x8*)(qp + kk * 16 + hl * 8);
    }
    prepare(1);
    if (VR == 3 || loads_k) {
      issue(1);
      prepare(2);
    }
    if (loads_k) {
      issue(2);
      prepare(3);
      TAPS_WAIT_VMCNT(2 * BPW);                   // K(0), the queries: this wave's part
    }
    TAPS_LDS_BARRIER();                           // ... and every other wave's
    if (wrow0 > last) {                           // no rows: the wave only loads
      for (int t = 0, P = 0; t < nt; ++t, P = P == 2 ? 0 : P + 1) {
        advance();
        fill(P, VR == 3 ? P : t & 1);
        prepare(t + 1 + ahead);
      }
    } else {
      f32x16 a, b, c;
#pragma unroll
      for (int i = 0; i < 4; ++i) read_k(0, i);
      scores(0, 0, 0, NKK, a);
      scores(0, 1, 0, NKK, b);
      m0 = largest(a);
      if constexpr (VR == 3) {
        for (int t = 0; t < nt; t += 3) {   // (one exit: with three the accumulators moved about)
          step(Slot<0>(), Slot<0>(), t, a, b, c);
          if (t + 1 < nt) step(Slot<1>(), Slot<1>(), t + 1, c, a, b);
          if (t + 2 < nt) step(Slot<2>(), Slot<2>(), t + 2, b, c, a);
        }
      } else {
        for (int t = 0; t < nt; t += 6) {
          step(Slot<0>(), Slot<0>(), t, a, b, c);
          if (t + 1 < nt) step(Slot<1>(), Slot<1>(), t + 1, c, a, b);
          if (t + 2 < nt) step(Slot<2>(), Slot<0>(), t + 2, b, c, a);
          if (t + 3 < nt) step(Slot<0>(), Slot<1>(), t + 3, a, b, c);
          if (t + 4 < nt) step(Slot<1>(), Slot<0>(), t + 4, c, a, b);
          if (t + 5 < nt) step(Slot<2>(), Slot<1>(), t + 5, b, c, a);
        }
      }
    }
    TAPS_WAIT_VMCNT(0);   // (empty) loads past the piece land before the LDS is released
  }

  const float l = pair_sum(l_run);
  if (!live) return;
  if (!cut) {
    const float inv = l == 0.f ? 0.f : 1.f / l;   // no key: zeros
    __bf16* const out = (__bf16*)A.O + ((size_t)(p.q0 + tok) * A.Hq + head) * HD;
#pragma unroll
    for (int db = 0; db < NDB; ++db)
#pragma unroll
      for (int r = 0; r < 4; ++r) {
        bf16x4 x;
#pragma unroll
        for (int t = 0; t < 4; ++t) x[t] = (__bf16)(o[db][4 * r + t] * inv);
        *(bf16x4*)(out + db * 32 + 8 * r + 4 * hl) = x;
      }
    return;
  }
  const int64_t slot = ((int64_t)p.slot + (int64_t)p.split * p.tiles) * A.Hkv + kvh;
  if (slot >= A.slots) return;
  const size_t at = (size_t)slot * M + wave * 32 + l32;
  float* const out = A.wsO + at * HD;
#pragma unroll
  for (int db = 0; db < NDB; ++db)
#pragma unroll
    for (int r = 0; r < 4; ++r)
      *(f32x4*)(out + db * 32 + 8 * r + 4 * hl) =
          f32x4{o[db][4 * r], o[db][4 * r + 1], o[db][4 * r + 2], o[db][4 * r + 3]};
  if (hl == 0) A.wsML[at] = make_float2(m_ref, l);   // (base 2, after the scale)
#endif
}

// max and sum over the four lanes that share l % 16, in each of them
__device__ inline float quad_max(float x) {
  auto a = __builtin_amdgcn_permlane16_swap(__float_as_uint(x), __float_as_uint(x), false, false);
  x = fmaxf(__uint_as_float(a[0]), __uint_as_float(a[1]));
  return pair_max(x);
}
__device__ inline float quad_sum(float x) {
  auto a = __builtin_amdgcn_permlane16_swap(__float_as_uint(x), __float_as_uint(x), false, false);
  x = __uint_as_float(a[0]) + __uint_as_float(a[1]);
  return pair_sum(x);
}

// Lane (g = l / 16, c = l % 16).  S^T: the lane holds the dims 16 j + 4 g + 0..3 of key c and of
// query c, four k-steps a load, and ends with the scores of query c for the keys 4 g + 0..3 of the
// 16.  O^T += V^T P^T: k-step r takes the keys 4 g + r; row m of block t is dim m * HD / 16 + t, so
// that a lane reads HD / 16 consecutive dims of a V row.
constexpr int kThreads = 256;
template <int HD>
__global__ __launch_bounds__(kThreads) void chunk_f32_kernel(const ChunkArgs A) {
  constexpr int KT = 32;
  constexpr int DPL = HD / 16, J = HD / 16;
  constexpr int ROW = HD + 4;                     // LDS row stride: rows 4 banks apart
  constexpr int CPR = HD / 4;                     // 16-byte chunks of a row
  constexpr int LD = KT * CPR / kThreads;         // chunks per thread and tile: 4 or 2
  __shared__ float s_k[2][KT][ROW], s_v[2][KT][ROW];

  const int G = A.Hq / A.Hkv;
  const int kvh = blockIdx.x % A.Hkv;
  const Piece p = find_piece<kMF, 0>(A, G, blockIdx.x / A.Hkv);
  if (!p.found) return;
  const int tid = threadIdx.x, lane = tid & 63, c = lane & 15, g = lane >> 4;
  const int wave = __builtin_amdgcn_readfirstlane(tid >> 6);
  const int last = p.n * G - 1;
  const int row0 = p.tile * kMF;
  int lo, hi;
  key_range(A, p, row0 / G, min(row0 + kMF - 1, last) / G, lo, hi);
  const int u0 = lo / kUnit, u1 = (hi + kUnit - 1) / kUnit;
  const int ub = u0 + min((int64_t)p.split * p.L, (int64_t)(u1 - u0));
  const int ue = (int)min((int64_t)ub + p.L, (int64_t)u1);
  const bool cut = p.splits > 1;
  if (cut && ub >= ue && p.split > 0) return;
  const int k0 = ub * kUnit, k_end = min(hi, ue * kUnit);
  const int nt = k_end > k0 ? (k_end - k0 + KT - 1) / KT : 0;

  const int wrow0 = row0 + wave * 16;
  const int qrow = min(wrow0 + c, last);
  const int tok = qrow / G, head = kvh * G + (qrow - tok * G);
  const bool live = wrow0 + c <= last;
  const int base = p.kv - p.n;
  const int pos = live ? base + tok : -1;
  const int from = A.window > 0 ? pos - A.window + 1 : 0;
  const int pos_lo = base + wrow0 / G;
  const int pos_hi = wrow0 <= last ? base + min(wrow0 + 15, last) / G : -1;
  const int w_lo = A.window > 0 ? pos_lo - A.window + 1 : 0;
  const int from_hi = A.window > 0 ? pos_hi - A.window + 1 : 0;

  f32x4 q[J];
  {
    const float* const qp =
        (const float*)A.Q + (size_t)(p.q0 + tok) * A.q_stride + (size_t)head * HD;
#pragma unroll
    for (int j = 0; j < J; ++j) q[j] = *(const f32x4*)(qp + 16 * j + 4 * g);
  }
  const size_t rs = (size_t)A.Hkv * HD;
  const float* const Kp = (const float*)A.K + (size_t)kvh * HD;
  const float* const Vp = (const float*)A.V + (size_t)kvh * HD;
  const int32_t* const bt = A.pk.btab + (size_t)p.b * A.pk.max_pages;
  f32x4 xk[LD], xv[LD];
  auto page_of = [&](int t) {   // (past the piece: any)
    const int entry = bt[min((k0 + t * KT) >> A.pk.page_shift, A.pk.max_pages - 1)];
    return min(max(entry, 0), A.pk.num_pages - 1);
  };
  auto load = [&](int t, int page) {   // keys outside [lo, k_end) read as zeros
    const int r0 = k0 + t * KT;
    const size_t prow = ((size_t)page << A.pk.page_shift) + (r0 & ((1 << A.pk.page_shift) - 1));
#pragma unroll
    for (int j = 0; j < LD; ++j) {
      const int i = tid + j * kThreads, r = i / CPR, d = (i % CPR) * 4;
      const bool in = r0 + r >= lo && r0 + r < k_end;
      const f32x4 z = {0.f, 0.f, 0.f, 0.f};
      xk[j] = in ? *(const f32x4*)(Kp + (prow + r) * rs + d) : z;
      xv[j] = in ? *(const f32x4*)(Vp + (prow + r) * rs + d) : z;
    }
  };
  auto keep = [&](int buf) {
#pragma unroll
    for (int j = 0; j < LD; ++j) {
      const int i = tid + j * kThreads, r = i / CPR, d = (i % CPR) * 4;
      *(f32x4*)&s_k[buf][r][d] = xk[j];
      *(f32x4*)&s_v[buf][r][d] = xv[j];
    }
  };

  f32x4 o[DPL];
#pragma unroll
  for (int t = 0; t < DPL; ++t) o[t] = f32x4{0.f, 0.f, 0.f, 0.f};
  // the reference stays in score units: the exponent is (s - m) * scale, whose rounding error
  // falls with the weight of the term
  float m_ref = -INFINITY, l_run = 0.f;
  int page = 0;   // of the next tile to load
  if (nt > 0) {
    const int first = page_of(0);
    page = page_of(1);
    load(0, first);
    keep(0);
  }
  __syncthreads();
  for (int t = 0; t < nt; ++t) {
    const int key = k0 + t * KT, buf = t & 1;
    if (t + 1 < nt) {
      load(t + 1, page);
      page = page_of(t + 2);
    }
    if (key <= pos_hi && key + KT > w_lo) {
      f32x4 s[2];
#pragma unroll
      for (int i = 0; i < 2; ++i) {
        f32x4 sp[4];   // four partial sums per score: chains a quarter as long round less
#pragma unroll
        for (int e = 0; e < 4; ++e) sp[e] = f32x4{0.f, 0.f, 0.f, 0.f};
#pragma unroll
        for (int j = 0; j < J; ++j) {
          const f32x4 k = *(const f32x4*)&s_k[buf][16 * i + c][16 * j + 4 * g];
#pragma unroll
          for (int e = 0; e < 4; ++e)
            sp[e] = __builtin_amdgcn_mfma_f32_16x16x4f32(k[e], q[j][e], sp[e], 0, 0, 0);
        }
        s[i] = (sp[0] + sp[1]) + (sp[2] + sp[3]);
      }
      if (key + KT - 1 > pos_lo || key < from_hi) {
#pragma unroll
        for (int i = 0; i < 2; ++i)
#pragma unroll
          for (int r = 0; r < 4; ++r) {
            const int k = key + 16 * i + 4 * g + r;
            s[i][r] = k <= pos && k >= from ? s[i][r] : -INFINITY;
          }
      }
      const float mx = quad_max(fmaxf(fmaxf(fmaxf(s[0][0], s[0][1]), fmaxf(s[0][2], s[0][3])),
                                      fmaxf(fmaxf(s[1][0], s[1][1]), fmaxf(s[1][2], s[1][3]))));
      const bool upd = (mx - m_ref) * A.scale_log2 > 8.f;
      if (__ballot(upd)) {
        const float nref = upd ? mx : m_ref;
        const float alpha =
            !upd ? 1.f
                 : m_ref == -INFINITY ? 0.f : __builtin_amdgcn_exp2f((m_ref - nref) * A.scale_log2);
        l_run *= alpha;
#pragma unroll
        for (int d = 0; d < DPL; ++d) o[d] *= alpha;
        m_ref = nref;
      }
      const float mu = m_ref == -INFINITY ? 0.f : m_ref;
#pragma unroll
      for (int i = 0; i < 2; ++i) {
        float e[4];
#pragma unroll
        for (int r = 0; r < 4; ++r) e[r] = __builtin_amdgcn_exp2f((s[i][r] - mu) * A.scale_log2);
        l_run += (e[0] + e[1]) + (e[2] + e[3]);
#pragma unroll
        for (int r = 0; r < 4; ++r) {
          const float* const v = &s_v[buf][16 * i + 4 * g + r][DPL * c];
#pragma unroll
          for (int d = 0; d < DPL; d += 4) {
            const f32x4 x = *(const f32x4*)(v + d);
#pragma unroll
            for (int w = 0; w < 4; ++w)
              o[d + w] = __builtin_amdgcn_mfma_f32_16x16x4f32(x[w], e[r], o[d + w], 0, 0, 0);
          }
        }
      }
    }
    if (t + 1 < nt) keep(buf ^ 1);   // read last before the barrier behind step t - 1
    __syncthreads();
  }

  const float l = quad_sum(l_run);
  if (!live) return;
  // row r of block t is dim (4 g + r) * DPL + t of query c
  float* out;
  float inv = 1.f;
  if (!cut) {
    inv = l == 0.f ? 0.f : 1.f / l;
    out = (float*)A.O + ((size_t)(p.q0 + tok) * A.Hq + head) * HD;
  } else {
    const int64_t slot = ((int64_t)p.slot + (int64_t)p.split * p.tiles) * A.Hkv + kvh;
    if (slot >= A.slots) return;
    const size_t at = (size_t)slot * kMF + wave * 16 + c;
    out = A.wsO + at * HD;
    if (g == 0) A.wsML[at] = make_float2(m_ref, l);   // (in score units)
  }
#pragma unroll
  for (int r = 0; r < 4; ++r)
#pragma unroll
    for (int d = 0; d < DPL; d += 4)
      *(f32x4*)(out + (4 * g + r) * DPL + d) =
          f32x4{o[d][r], o[d + 1][r], o[d + 2][r], o[d + 3][r]} * inv;
}

// Adds the pieces of the tiles that were cut: ROWS query rows of a (KV head, request that is cut)
// at a time; 16 threads a row, and GROUPS of them share its pieces, kAhead of which load together.
// Bound: the pieces' bytes (512 tokens over 8K, 32/8 heads of 128: 33 MB in 9 us) or, for few rows,
// latency (5 us).
constexpr int kCombineThreads = 256, kAhead = 8;
__device__ inline void store4(float* p, const f32x4& x) { *(f32x4*)p = x; }
__device__ inline void store4(__bf16* p, const f32x4& x) {
  bf16x4 r;
#pragma unroll
  for (int t = 0; t < 4; ++t) r[t] = (__bf16)x[t];
  *(bf16x4*)p = r;
}
// weight of a part about the reference m where the sum's is M: both of base 2 in bf16, whose parts
// were summed about that very number, and in fp32 in score units, as in the parts' own exponents
template <typename T>
__device__ inline float part_weight(const ChunkArgs& A, float m, float M) {
  if (m == -INFINITY) return 0.f;
  return __builtin_amdgcn_exp2f(sizeof(T) == 4 ? (m - M) * A.scale_log2 : m - M);
}
template <typename T, int HD, int M, int ROWS, int GROUPS>
__global__ __launch_bounds__(kCombineThreads) void chunk_combine_kernel(const ChunkArgs A) {
  constexpr int W = HD / 64;   // 16-byte vectors per thread
  static_assert(kCombineThreads == 16 * ROWS * GROUPS, "16 threads a row and group");
  __shared__ f32x4 s_acc[GROUPS][ROWS][16][W];
  __shared__ float2 s_ml[GROUPS][ROWS];
  const int G = A.Hq / A.Hkv, kvh = blockIdx.x % A.Hkv;
  const int tr = threadIdx.x & 15, rr = (threadIdx.x >> 4) % ROWS;
  const int grp = threadIdx.x / (16 * ROWS);
  for (int item = blockIdx.x / A.Hkv;; item += gridDim.x / A.Hkv) {
    const Piece p = find_piece<M, ROWS>(A, G, item);
    if (!p.found) return;
    const int last = p.n * G - 1, row0 = p.tile * M;
    const int row = min(p.group * ROWS + rr, last);
    int lo, hi;
    key_range(A, p, row0 / G, min(row0 + M - 1, last) / G, lo, hi);
    const int units = (hi + kUnit - 1) / kUnit - lo / kUnit;
    const int pieces = max(1, (units + p.L - 1) / p.L);
    // (never: the slots are bounded by the lengths themselves)
    if (((int64_t)p.slot + (int64_t)(pieces - 1) * p.tiles) * A.Hkv + kvh >= A.slots) return;
    float Mx = -INFINITY, L = 0.f;
    f32x4 acc[W];
#pragma unroll
    for (int w = 0; w < W; ++w) acc[w] = f32x4{0.f, 0.f, 0.f, 0.f};
    for (int s0 = grp; s0 < pieces; s0 += kAhead * GROUPS) {
      float2 ml[kAhead];
      f32x4 x[kAhead][W];
#pragma unroll
      for (int k = 0; k < kAhead; ++k) {
        const int s = min(s0 + k * GROUPS, pieces - 1);
        const size_t i =
            ((size_t)((int64_t)p.slot + (int64_t)s * p.tiles) * A.Hkv + kvh) * M + (row - row0);
        ml[k] = A.wsML[i];
#pragma unroll
        for (int w = 0; w < W; ++w) x[k][w] = *(const f32x4*)(A.wsO + i * HD + 64 * w + 4 * tr);
      }
      float Mc = Mx;
#pragma unroll
      for (int k = 0; k < kAhead; ++k) Mc = fmaxf(Mc, ml[k].x);
      const float a = part_weight<T>(A, Mx, Mc);
      L *= a;
#pragma unroll
      for (int w = 0; w < W; ++w) acc[w] *= a;
#pragma unroll
      for (int k = 0; k < kAhead; ++k) {
        if (s0 + k * GROUPS >= pieces) continue;
        if (ml[k].x != -INFINITY) {
          const float e = part_weight<T>(A, ml[k].x, Mc);
          L += e * ml[k].y;
#pragma unroll
          for (int w = 0; w < W; ++w) acc[w] += e * x[k][w];
        }
        if (ml[k].y != ml[k].y) L = ml[k].y;   // a NaN score moves no maximum
      }
      Mx = Mc;
    }
    if (grp > 0) {
#pragma unroll
      for (int w = 0; w < W; ++w) s_acc[grp - 1][rr][tr][w] = acc[w];
      if (tr == 0) s_ml[grp - 1][rr] = make_float2(Mx, L);
    }
    __syncthreads();
    if (grp == 0 && p.group * ROWS + rr <= last) {
      float Mc = Mx;
#pragma unroll
      for (int g = 0; g < GROUPS - 1; ++g) Mc = fmaxf(Mc, s_ml[g][rr].x);
      const float a = part_weight<T>(A, Mx, Mc);
      L *= a;
#pragma unroll
      for (int w = 0; w < W; ++w) acc[w] *= a;
#pragma unroll
      for (int g = 0; g < GROUPS - 1; ++g) {
        const float2 ml = s_ml[g][rr];
        if (ml.x != -INFINITY) {
          const float e = part_weight<T>(A, ml.x, Mc);
          L += e * ml.y;
#pragma unroll
          for (int w = 0; w < W; ++w) acc[w] += e * s_acc[g][rr][tr][w];
        }
        if (ml.y != ml.y) L = ml.y;
      }
      const int tok = row / G, head = kvh * G + (row - tok * G);
      T* const out = (T*)A.O + ((size_t)(p.q0 + tok) * A.Hq + head) * HD + 4 * tr;
      const float inv = L == 0.f ? 0.f : 1.f / L;
#pragma unroll
      for (int w = 0; w < W; ++w) store4(out + 64 * w, acc[w] * inv);
    }
    __syncthreads();   // the groups' parts are read before the next ones are written
  }
}

template <typename T, int HD, int M>
hipError_t launch_combine(const ChunkArgs& A, const ChunkPlan& p, hipStream_t s) {
  const unsigned grid = (unsigned)(p.cut_groups * A.Hkv);
  if (p.cut_rows == 16) chunk_combine_kernel<T, HD, M, 16, 1><<<grid, kCombineThreads, 0, s>>>(A);
  else chunk_combine_kernel<T, HD, M, 4, 4><<<grid, kCombineThreads, 0, s>>>(A);
  return hipGetLastError();
}

template <typename T, int HD>
hipError_t launch_t(const ChunkArgs& A, const ChunkPlan& p, hipStream_t s) {
  const unsigned grid = (unsigned)(p.items * A.Hkv);
  if (A.index) {
    int4* const index = const_cast<int4*>(A.index);
    const int g = p.cut_rows;
    if (sizeof(T) == 4) chunk_index_kernel<kMF><<<1, kIndexThreads, 0, s>>>(A, g, index);
    else if (p.rows == 256) chunk_index_kernel<256><<<1, kIndexThreads, 0, s>>>(A, g, index);
    else chunk_index_kernel<128><<<1, kIndexThreads, 0, s>>>(A, g, index);
    const hipError_t e = hipGetLastError();
    if (e != hipSuccess) return e;
  }
  if constexpr (sizeof(T) == 4) chunk_f32_kernel<HD><<<grid, kThreads, 0, s>>>(A);
  else if (p.rows == 256) chunk_bf16_kernel<HD, HD == 128 ? 8 : 4, 3><<<grid, 512, 0, s>>>(A);
  else if (p.pair) chunk_bf16_kernel<HD, 4, HD == 128 ? 2 : 3><<<grid, 256, 0, s>>>(A);
  else chunk_bf16_kernel<HD, 4, 3><<<grid, 256, 0, s>>>(A);
  const hipError_t e = hipGetLastError();
  if (e != hipSuccess || p.slots == 0) return e;
  if constexpr (sizeof(T) == 2)
    return p.rows == 256 ? launch_combine<T, HD, 256>(A, p, s)
                         : launch_combine<T, HD, 128>(A, p, s);
  else
    return launch_combine<T, HD, kMF>(A, p, s);
}

}  // namespace

// Tiles of 256 query rows use each key tile in LDS twice as often as those of 128.  128 spread a
// short prompt over more CUs; with a ring of two tiles of V two workgroups share a CU (pair), so
// that one computes while the other begins or ends; at head_dim 64, where the exponentials bound
// the kernel, three do with rings of three.  us a call (32/8 heads of 128) with 256 rows / 128
// alone / 128 in pairs: prompts of 1024, 1536, 2048 and 2560 tokens 40 / 27.5 / 29, 52 / 42 / 45,
// 67 / 61 / 58 and 80 / 90 / 72, of 4096 145 / 182 / 160; 1200 after 1200 67 / 73 / 63; 8 prompts
// of 1000 122 / - / 111, 8 of 100 to 1000 46 / 50 / 39; 512 after 8K 92 / 105 / 98; 64 requests of
// one token after 50 to 300 keys - / 20 / 15, 256 of them - / 70 / 48, 16 after 512 to 16K 95 / 84
// / 79.  Ragged batches, 256 / 128 rows, differ little: 16 requests of 1 to 200 tokens after 100 to
// 2000 keys 33 / 34.5, 32 of 1 to 500 after up to 2000 46.5 / 46, 8 of 100 to 1000 after up to 1500
// 54 / 48.5, 16 of 1 to 1024 after 1 to 16K 63.5 / 63.5, but under a bound of 4000 keys the rule
// gives up 10 %: 16 of 1 to 500 after 100 to 4000 46.5 / 41.7, 64 of 1 to 200 104 / 97.  head_dim
// 64, 256 / 128 rows: prompts of 1024 and 2048 29 / 20 and 47 / 39, 16 requests of
// 1 to 1024 tokens over 16K to 1 47 / 39, 512 over 8K 60 / 63.
// Cuts.  Pieces: one per CU, or two where there are many tiles (16 requests of one token 79 us with
// 512 for 86 with 256, one of 16 tokens after 32K 39 for 33) and at head_dim 64 (16 requests of 1
// to 1024 tokens 39 for 44); fp32: 512.  min_units: mostly a piece's start and end.  gain: what the
// second kernel costs; an fp32 unit takes as long as four in bf16.  Where 64 tiles or more take
// part the pieces may be longer, and where max_len then lets none be cut the second kernel is not
// launched: a prompt of 1024 takes 27 us with 8 and 30 with 4, 16 tokens over 900 keys 21 and 15.
// Bounds of what the device finds.  Tiles: the requests' rows / M, and one more per request.
// With L >= (sum of tiles * units) * Hkv / target, the cut requests (units > L) have at most
// target / Hkv tiles between them, and at most twice as many pieces as their tiles * units / L.
ChunkPlan plan_chunk(int batch, int rows, int Hq, int Hkv, int head_dim, int max_len,
                     int dtype) {
  ChunkPlan p;
  const int64_t heads = (int64_t)rows * Hq;       // query rows of all heads
  const bool small = max_len <= 2560 || (int64_t)rows * (Hq / Hkv) <= (int64_t)64 * batch;
  p.rows = dtype == TAPS_FP32 ? kMF : head_dim == 64 || small ? 128 : 256;
  p.pair = p.rows == 128 && head_dim == 128 &&
           (max_len > 2560 || heads / 128 + (int64_t)batch * Hkv > 300);
  p.cut = p.rows == kMF ? ChunkCut{9, 2, 1}
          : p.rows == 256
              ? ChunkCut{8, 4, 6}
              : ChunkCut{head_dim == 64 || (int64_t)batch * Hkv >= 128 ? 9 : 8,
                         heads > 8192 ? 8 : 4, 8};
  const int64_t M = p.rows, target = (int64_t)1 << p.cut.target_log2;
  const int64_t tiles = std::min<int64_t>((int64_t)rows * (Hq / Hkv) / M + batch,
                                          (int64_t)rows * (Hq / Hkv));
  const bool may_cut = max_len > (p.cut.min_units + p.cut.gain) * kUnit;
  const int64_t cut = std::min<int64_t>(tiles, std::max<int64_t>(1, target / Hkv));
  // Their groups of rows in the second kernel, by their tiles and by all requests' rows; it takes
  // more than about 1024 of them in turns.  Few rows have many pieces each, which four groups of
  // threads share: us of 16 tokens (32/8 heads) over 32K, 31 pieces, with groups of 4 rows / 16
  // 5.7 / 10.4; of 512 tokens over 8K, 4 pieces, 28 / 9.3.
  p.cut_rows = heads <= 4096 ? 4 : 16;
  const int64_t groups = std::min<int64_t>(cut * (M / p.cut_rows),
                                           (int64_t)rows * (Hq / Hkv) / p.cut_rows + batch);
  p.cut_groups = may_cut ? std::min<int64_t>(groups, std::max(1, 1024 / Hkv)) : 0;
  p.slots = may_cut ? (int64_t)Hkv * std::max<int64_t>(1, 2 * target / Hkv) : 0;
  p.items = tiles + p.slots / Hkv;
  p.indexed = batch > 4 * kWave ? batch + 1 : 0;
  return p;
}

size_t chunk_ws_bytes(const ChunkPlan& p, int head_dim) {
  return (size_t)p.indexed * sizeof(int4) +
         (size_t)p.slots * p.rows * (head_dim * sizeof(float) + sizeof(float2));
}

hipError_t launch_chunk(const void* Q, int64_t q_stride, const void* K, const void* V,
                        const PagedKV& pk, const int32_t* q_start, const int32_t* kv_len,
                        int batch, int rows, int Hq, int Hkv, int head_dim, int max_len,
                        int window, int dtype, float scale, const ChunkPlan& p, void* O, void* ws,
                        hipStream_t s) {
  if (batch <= 0 || rows <= 0) return hipSuccess;
  ChunkArgs A;
  A.Q = (const unsigned char*)Q, A.K = (const unsigned char*)K, A.V = (const unsigned char*)V;
  A.q_stride = q_stride, A.pk = pk, A.q_start = q_start, A.kv_len = kv_len;
  A.batch = batch, A.rows = rows, A.Hq = Hq, A.Hkv = Hkv, A.max_len = max_len, A.window = window;
  A.scale_log2 = scale * 1.4426950408889634f;
  A.cut = p.cut;
  A.O = (unsigned char*)O;
  A.slots = (int)p.slots;
  A.index = p.indexed ? (const int4*)ws : nullptr;
  A.wsO = p.slots ? (float*)((int4*)ws + p.indexed) : nullptr;
  A.wsML = p.slots ? (float2*)(A.wsO + (size_t)p.slots * p.rows * head_dim) : nullptr;
  if (dtype == TAPS_BF16)
    return head_dim == 128 ? launch_t<__bf16, 128>(A, p, s) : launch_t<__bf16, 64>(A, p, s);
  return head_dim == 128 ? launch_t<float, 128>(A, p, s) : launch_t<float, 64>(A, p, s);
}

}  // namespace taps

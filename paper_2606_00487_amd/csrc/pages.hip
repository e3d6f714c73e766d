// The paged cache's bookkeeping: pages for a batch's requests out of a free-page stack, block
// tables and slot maps (kv_reserve_paged), and new rows into the pools by slot
// (kv_append_paged).
#include <algorithm>

#include "common.h"
#include "scan.h"

namespace taps {

namespace {

// ----------------------------------------------------------------------------------
// kv_reserve_paged.  With want_b = ceil((ctx_b + new_b) / page_rows), rel_b = max(held_b -
// want_b, 0) and need_b = max(want_b - held_b, 0):
//   pushes  page i of request b's rel_b last ones goes to stack position n_free +
//           (sum of rel before b) + i;
//   takes   page i of need_b is stack entry size - 1 - (sum of need before b) - i of the stack
//           after the pushes, where that sum with need_b included is at most size.
// Both sums are over the whole batch, whose lengths (12 bytes a request) are so few that every
// workgroup adds them up itself: one launch without a word between workgroups.  A take at or
// above n_free is a page that this call pushes; it is read from the table row that gives it
// (found by its place in the prefix sums), which no other workgroup writes, so that the kernel
// nowhere reads what it writes.  Grid (runs of requests, slices of the slot map).
// Bound: latency (two dependent reads, a block scan, the page reads): 5 us for 16 requests; 6.5 for
// 1024, whose sums every workgroup forms; and the slot map's bytes: 14.4 us with 4096 slots a
// request (34 MB, which take 5.8 at the memory's rate).  (With a page looked up for every slot of
// it instead of once: 27 us.)
constexpr int kReserveThreads = 256;
constexpr int kSlotsPerGroup = 4096;   // slot map columns per workgroup
constexpr int kReserveGroups = 512;    // runs of requests, at most

struct Lengths {
  int held, ctx, nnew, want;
  bool fits;      // the rows fit the table
  int rel, need;  // pages given back, pages to take
};

__device__ inline Lengths lengths(const int32_t* held, const int32_t* ctx, const int32_t* nnew,
                                  int b, int max_pages, int shift, int max_new) {
  Lengths r;
  r.held = min(max(held[b], 0), max_pages);
  // max_pages << shift is at most 2^30 and max_new 2^27: the sum fits 32 bits, and a longer
  // context fits no table either.  (In 64 bits hipcc 7.2 selects `want` by a stale condition
  // code: the comparison of uniform 64-bit values goes to VCC, the select reads SCC.)
  r.ctx = min(max(ctx[b], 0), (1 << 30) + 1);
  r.nnew = min(max(nnew[b], 0), max_new);
  const int want = (r.ctx + r.nnew + ((1 << shift) - 1)) >> shift;
  r.fits = want <= max_pages;
  r.want = r.fits ? want : r.held;
  r.rel = max(r.held - r.want, 0);
  r.need = max(r.want - r.held, 0);
  return r;
}

__global__ __launch_bounds__(kReserveThreads) void reserve_kernel(
    int32_t* __restrict__ table, int max_pages, const int32_t* __restrict__ held,
    const int32_t* __restrict__ ctx, const int32_t* __restrict__ nnew, int batch, int run,
    int32_t* __restrict__ stack, const int32_t* __restrict__ n_free, int num_pages, int shift,
    int max_new, int64_t* __restrict__ slots, int32_t* __restrict__ held_out,
    int32_t* __restrict__ n_free_out, int32_t* __restrict__ n_short) {
  __shared__ int64_t s_rel[kMaxReserveBatch];   // pages given back by the requests before
  __shared__ int32_t s_want[kMaxReserveBatch];
  __shared__ int64_t s_need[kMaxReserveBatch / kReserveGroups];   // pages taken before, this run
  __shared__ int32_t s_page[kSlotsPerGroup / 32 + 1];             // a slice's pages
  __shared__ int64_t s_wave[2][kReserveThreads / kWave];
  __shared__ int64_t s_taken;
  __shared__ int s_unfit, s_unserved;
  const int tid = threadIdx.x, lane = tid & (kWave - 1), wave = tid / kWave;
  const int run0 = blockIdx.x * run, run1 = min(run0 + run, batch);
  const int per = (batch + kReserveThreads - 1) / kReserveThreads;
  if (tid == 0) s_unfit = s_unserved = 0, s_taken = 0;
  const int nf = min(max(*n_free, 0), num_pages);

  // this thread's requests [first, last): their sums, then their prefix over the block
  const int first = min(tid * per, batch), last = min(first + per, batch);
  int64_t rel = 0, need = 0;
  int unfit = 0;
#pragma unroll 4
  for (int j = first; j < last; ++j) {
    const Lengths r = lengths(held, ctx, nnew, j, max_pages, shift, max_new);
    rel += r.rel;
    need += r.need;
    unfit += r.fits ? 0 : 1;
    s_want[j] = r.want;
    s_rel[j] = ((int64_t)r.rel << 32) | (uint32_t)r.need;   // both for the second loop
  }
  int64_t irel = (int64_t)wave_scan_u64((uint64_t)rel);
  int64_t ineed = (int64_t)wave_scan_u64((uint64_t)need);
  if (lane == kWave - 1) s_wave[0][wave] = irel, s_wave[1][wave] = ineed;
  __syncthreads();
  int64_t rel_all = 0, need_all = 0;
#pragma unroll
  for (int w = 0; w < kReserveThreads / kWave; ++w) {
    if (w < wave) irel += s_wave[0][w], ineed += s_wave[1][w];
    rel_all += s_wave[0][w];
    need_all += s_wave[1][w];
  }
  if (unfit) atomicAdd(&s_unfit, unfit);
  const int64_t size = min((int64_t)nf + rel_all, (int64_t)num_pages);
  {
    int64_t r0 = irel - rel, n0 = ineed - need, taken = 0;
    int unserved = 0;
    for (int j = first; j < last; ++j) {
      const int64_t both = s_rel[j];
      const int jneed = (int)(uint32_t)both;
      s_rel[j] = r0;
      if (j >= run0 && j < run1) s_need[j - run0] = n0;
      r0 += both >> 32;
      n0 += jneed;
      if (jneed > 0) {
        if (n0 <= size) taken = n0;
        else ++unserved;
      }
    }
    // the sums grow with the request: the last one served has taken the most
    if (need_all > size) {
      if (taken) atomicMax((unsigned long long*)&s_taken, (unsigned long long)taken);
      if (unserved) atomicAdd(&s_unserved, unserved);
    }
  }
  __syncthreads();
  if (blockIdx.x == 0 && blockIdx.y == 0 && tid == 0) {
    *n_free_out = (int32_t)(size - (need_all > size ? s_taken : need_all));
    *n_short = s_unfit + s_unserved;
  }

  // the nth page that the batch takes, from the top of the stack after the pushes
  auto take = [&](int64_t nth) -> int32_t {
    const int64_t e = size - 1 - nth;
    if (e < nf) return stack[e];
    const int64_t r = e - nf;
    int lo = 0, hi = batch - 1;   // the last request whose pushes start at or before r
    while (lo < hi) {
      const int mid = (lo + hi + 1) / 2;
      if (s_rel[mid] <= r) lo = mid;
      else hi = mid - 1;
    }
    return table[(size_t)lo * max_pages + s_want[lo] + (r - s_rel[lo])];
  };
  for (int b = run0; b < run1; ++b) {
    const Lengths me = lengths(held, ctx, nnew, b, max_pages, shift, max_new);
    const int64_t n0 = s_need[b - run0];
    const bool served = me.fits && (me.need == 0 || n0 + me.need <= size);
    int32_t* const row = table + (size_t)b * max_pages;
    if (blockIdx.y == 0) {
      if (tid == 0) held_out[b] = served ? me.want : me.held;
      const int64_t p0 = nf + s_rel[b];
      for (int i = tid; i < me.rel && p0 + i < num_pages; i += kReserveThreads)
        stack[p0 + i] = row[me.want + i];
      if (served)
        for (int i = tid; i < me.need; i += kReserveThreads) row[me.held + i] = take(n0 + i);
    }
    if (slots == nullptr) continue;
    const int i0 = blockIdx.y * kSlotsPerGroup, i1 = min(i0 + kSlotsPerGroup, max_new);
    int64_t* const out = slots + (size_t)b * max_new;
    const int have = min(served ? me.nnew : 0, i1);
    // the slice's pages, once each (rows are below max_pages << shift: 32 bits hold them)
    const int q0 = (me.ctx + i0) >> shift;
    if (b > run0) __syncthreads();   // the last request's pages are read
    if (i0 < have) {
      const int pages = ((me.ctx + have - 1) >> shift) - q0 + 1;
      for (int i = tid; i < pages; i += kReserveThreads)
        s_page[i] = q0 + i < me.held ? row[q0 + i] : take(n0 + (q0 + i - me.held));
    }
    __syncthreads();
    for (int i = i0 + tid; i < i1; i += kReserveThreads) {
      const int r = me.ctx + i;
      out[i] = i < have
                   ? ((int64_t)s_page[(r >> shift) - q0] << shift) | (r & ((1 << shift) - 1))
                   : (int64_t)-1;
    }
  }
}

// ----------------------------------------------------------------------------------
// kv_append_paged: row t of K_new and V_new to row slot_map[t] of the pools, 16 bytes per
// thread and access; slots outside the pool are left out.  Bound: HBM (65536 rows of 2 KB, K and V:
// 94 us, 5.7 TB/s read and written); for few rows the launch.
constexpr int kAppendThreads = 256;
typedef uint32_t u32x4 __attribute__((ext_vector_type(4)));

__global__ __launch_bounds__(kAppendThreads) void append_kernel(
    const unsigned char* __restrict__ Kn, const unsigned char* __restrict__ Vn, int64_t k_stride,
    int64_t v_stride, const int64_t* __restrict__ slots, int rows, int row_chunks,
    unsigned char* __restrict__ Kp, unsigned char* __restrict__ Vp, int64_t pool_rows) {
  const int64_t total = (int64_t)rows * 2 * row_chunks;
  const int64_t step = (int64_t)gridDim.x * kAppendThreads;
  for (int64_t i = (int64_t)blockIdx.x * kAppendThreads + threadIdx.x; i < total; i += step) {
    const int t = (int)(i / (2 * row_chunks)), c = (int)(i - (int64_t)t * 2 * row_chunks);
    const bool v = c >= row_chunks;
    const int cc = v ? c - row_chunks : c;
    const int64_t s = slots[t];
    if (s < 0 || s >= pool_rows) continue;
    const u32x4 x =
        *(const u32x4*)((v ? Vn + (size_t)t * v_stride : Kn + (size_t)t * k_stride) + 16 * cc);
    *(u32x4*)((v ? Vp : Kp) + ((size_t)s * row_chunks + cc) * 16) = x;
  }
}

}  // namespace

hipError_t launch_reserve(int32_t* table, int max_pages, const int32_t* held, const int32_t* ctx,
                          const int32_t* n_new, int batch, int32_t* stack, const int32_t* n_free,
                          int num_pages, int page_shift, int max_new, int64_t* slots,
                          int32_t* held_out, int32_t* n_free_out, int32_t* n_short,
                          hipStream_t s) {
  if (batch <= 0) return hipSuccess;
  const int run = (batch + kReserveGroups - 1) / kReserveGroups;
  const int slices = slots ? std::max(1, (max_new + kSlotsPerGroup - 1) / kSlotsPerGroup) : 1;
  const dim3 grid((unsigned)((batch + run - 1) / run), (unsigned)slices);
  reserve_kernel<<<grid, kReserveThreads, 0, s>>>(
      table, max_pages, held, ctx, n_new, batch, run, stack, n_free, num_pages, page_shift, max_new,
      slots, held_out, n_free_out, n_short);
  return hipGetLastError();
}

hipError_t launch_append(const void* K_new, const void* V_new, int64_t k_stride_bytes,
                         int64_t v_stride_bytes, const int64_t* slots, int rows, int row_bytes,
                         void* K_pages, void* V_pages, int64_t pool_rows, hipStream_t s) {
  if (rows <= 0) return hipSuccess;
  const int row_chunks = row_bytes / 16;
  const int64_t groups = ((int64_t)rows * 2 * row_chunks + kAppendThreads - 1) / kAppendThreads;
  append_kernel<<<(unsigned)std::min<int64_t>(groups, 1 << 20), kAppendThreads, 0, s>>>(
      (const unsigned char*)K_new, (const unsigned char*)V_new, k_stride_bytes, v_stride_bytes,
      slots, rows, row_chunks, (unsigned char*)K_pages, (unsigned char*)V_pages, pool_rows);
  return hipGetLastError();
}

}  // namespace taps

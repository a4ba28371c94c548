// kv_extend.hip -- pages, slots and positions of a batch's new tokens, from
// lengths that stay on the GPU (include/eb_attention.h, eb_kv_extend).
//
// With a_b new tokens and n_b new pages of sequence b, row r belongs to the
// sequence with start_b <= r < start_b + a_b, start = exclusive sums of a, and
// its token is at p = cached_b + r - start_b.  The i-th new page of b is number
// sum_{c < b} n_c + i from the top of the stack.  Where the step has fewer rows
// than tokens, one sequence (the cut) gets rows for some of its tokens and those
// after it for none: the sums of pages up to the cut are those of whole sequences,
// so one scan gives them, and the cut alone counts its pages again.
//
// One launch: every workgroup sums over the whole batch itself (8 bytes per
// sequence, from L2) and keeps the sums in LDS, then fills its own rows; a row
// that begins a page writes the table's entry for it.  So no workgroup waits
// for another, and pages taken in this call are read from the stack, never
// from table entries that another workgroup writes.  The work is latency: one
// read of the lengths, 9 scan steps per 512 sequences, a binary search in LDS
// per row and one dependent read of the page: 8 sequences 3.6 us, 512 sequences with
// some 23000 rows 5.7 us (means of 40 launches).
#include <hip/hip_runtime.h>

#include "attention.h"

namespace eb {
namespace {

constexpr int kThreads = 512;
// Sums stop here: past any number of rows or pages.  Two of them still fit 32 bits
// without a sign, not with one.
constexpr uint32_t kMost = 1u << 30;

__device__ inline int64_t nonneg(int32_t v) { return v > 0 ? v : 0; }
__device__ inline uint32_t add_most(uint32_t a, uint32_t b) { return min(a + b, kMost); }

// Inclusive sums (rows, pages), each at most kMost, over the workgroup's threads;
// *total is that of all.
__device__ inline uint2 block_scan(uint2 v, uint2 *red, uint2 *total) {
  const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
#pragma unroll
  for (int d = 1; d < 64; d <<= 1) {
    const uint32_t x = __shfl_up(v.x, d), y = __shfl_up(v.y, d);
    if (lane >= d) v = make_uint2(add_most(v.x, x), add_most(v.y, y));
  }
  if (lane == 63) red[wave] = v;
  __syncthreads();
  uint2 before = make_uint2(0, 0), all = make_uint2(0, 0);
#pragma unroll
  for (int w = 0; w < kThreads / 64; ++w) {
    const uint2 u = red[w];
    if (w < wave) before = make_uint2(add_most(before.x, u.x), add_most(before.y, u.y));
    all = make_uint2(add_most(all.x, u.x), add_most(all.y, u.y));
  }
  *total = all;
  return make_uint2(add_most(v.x, before.x), add_most(v.y, before.y));
}

__global__ void __launch_bounds__(kThreads) kv_extend_kernel(eb_kv_extend_op o, int page_shift) {
  extern __shared__ int32_t lds[];
  int32_t *start = lds;                // [batch + 1], at most o.rows
  int32_t *taken = lds + o.batch + 1;  // [batch], at most kMost; behind the cut not used
  int32_t *cached = taken + o.batch;   // [batch]
  __shared__ uint2 red[2][kThreads / 64];
  __shared__ int64_t lost;
  __shared__ uint32_t cut_pages;  // of the sequences up to the cut
  const int32_t page = o.page;
  const int64_t capacity = (int64_t)o.table_stride << page_shift;  // tokens of a table row
  const bool first = blockIdx.x == 0;
  const int32_t n_free = min(max(o.n_free[0], 0), o.free_capacity);
  if (threadIdx.x == 0) cut_pages = kMost;  // (a barrier of the scan is before its other use)

  uint2 before = make_uint2(0, 0);
  for (int32_t b0 = 0; b0 < o.batch; b0 += kThreads) {
    const int32_t b = b0 + (int32_t)threadIdx.x;
    const bool ok = b < o.batch;
    const int64_t have = ok ? nonneg(o.cached[b]) : 0, add = ok ? nonneg(o.added[b]) : 0;
    const int64_t held = (min(have, capacity) + page - 1) >> page_shift;
    auto pages = [&](int64_t n) { return (uint32_t)(((min(have + n, capacity) + page - 1) >> page_shift) - held); };
    const uint32_t need = ok ? pages(add) : 0;
    const uint32_t rows = (uint32_t)min(add, (int64_t)o.rows + 1);
    uint2 all;
    // (the two halves of red in turn: one barrier a chunk of sequences)
    const uint2 in = block_scan(make_uint2(rows, need), red[(b0 / kThreads) & 1], &all);
    if (ok) {
      // (rows <= 2^24 + 1 and need <= 2^26 of a sequence, so a sum that stopped at kMost
      // less its own part is still past every row and every page of the stack)
      const uint32_t most = (uint32_t)o.rows, at = add_most(before.x, in.x - rows);
      const int32_t joined = (int32_t)(min(add_most(at, rows), most) - min(at, most));
      start[b] = (int32_t)min(at, most);
      taken[b] = (int32_t)add_most(before.y, in.y - need);
      cached[b] = (int32_t)have;
      if (at <= most && joined < add) cut_pages = add_most((uint32_t)taken[b], pages(joined));
      if (first) {
        o.q_start[b] = start[b];
        o.kv_len[b] = (int32_t)min(have + joined, capacity);
      }
    }
    before = make_uint2(add_most(before.x, all.x), add_most(before.y, all.y));
  }
  if (threadIdx.x == 0) {
    start[o.batch] = (int32_t)min(before.x, (uint32_t)o.rows);
    lost = 0;
  }
  __syncthreads();
  const int32_t took = min((int32_t)min(before.y, cut_pages), n_free);  // pages
  if (first && threadIdx.x == 0) {
    o.q_start[o.batch] = start[o.batch];
    o.n_free_out[0] = n_free - took;
  }

  // The last sequence b in [0, batch) with sums[b] <= v (sums ascend).
  auto find = [&](const int32_t *sums, int32_t v) {
    int32_t lo = 0, hi = o.batch;
    while (hi - lo > 1) {
      const int32_t mid = (lo + hi) >> 1;
      if (sums[mid] <= v)
        lo = mid;
      else
        hi = mid;
    }
    return lo;
  };
  auto valid = [&](int32_t p) { return p >= 0 && p < o.pages ? p : -1; };
  auto fresh = [&](int64_t nth) { return nth < n_free ? valid(o.free_pages[n_free - 1 - nth]) : -1; };

  const int32_t live = start[o.batch];
  for (int64_t r = (int64_t)blockIdx.x * kThreads + threadIdx.x; r < o.rows;
       r += (int64_t)gridDim.x * kThreads) {
    int32_t slot = -1, pos = 0;
    if (r < live) {
      const int32_t b = find(start, (int32_t)r);
      const int64_t have = cached[b], p = have + r - start[b];
      pos = (int32_t)min(p, (int64_t)0x7fffffff);
      if (p < capacity) {
        const int64_t held = (have + page - 1) >> page_shift, at = p >> page_shift;
        int32_t *entry = o.table + (int64_t)b * o.table_stride + at;
        int32_t id;
        if (at < held) {
          id = valid(*entry);
        } else {
          id = fresh(taken[b] + at - held);
          if ((p & (page - 1)) == 0) *entry = id;
        }
        if (id >= 0) slot = (id << page_shift) + (int32_t)(p & (page - 1));
      }
    }
    o.slots[r] = slot;
    o.positions[r] = pos;
  }
  if (!first) return;

  // Tokens without a page: those past the step's rows, those past a table row, those on
  // a held page that is missing, those on new pages that the stack does not have, and
  // those on new pages whose entry in the stack is no page.
  int64_t miss = 0;
  for (int32_t b = threadIdx.x; b < o.batch; b += kThreads) {
    const int64_t have = cached[b], joined = start[b + 1] - start[b];
    const int64_t all = have + joined, total = min(all, capacity);
    miss += nonneg(o.added[b]) - joined;
    if (joined == 0) continue;
    miss += max(all - max(have, capacity), (int64_t)0);
    const int64_t held = (min(have, capacity) + page - 1) >> page_shift;
    const int64_t end = min(total, held << page_shift);
    if (have < end && valid(o.table[(int64_t)b * o.table_stride + held - 1]) < 0) miss += end - have;
    const int64_t got = max(n_free - taken[b], 0);
    miss += max(total - max(have, (held + got) << page_shift), (int64_t)0);
  }
  for (int32_t i = threadIdx.x; i < took; i += kThreads) {
    if (fresh(i) >= 0) continue;
    const int32_t b = find(taken, i);
    const int64_t have = cached[b], total = min(have + start[b + 1] - start[b], capacity);
    const int64_t at = ((have + page - 1) >> page_shift) + i - taken[b];
    miss += min((at + 1) << page_shift, total) - (at << page_shift);
  }
#pragma unroll
  for (int d = 32; d >= 1; d >>= 1) miss += __shfl_xor(miss, d);
  if ((threadIdx.x & 63) == 0 && miss > 0)
    atomicAdd(reinterpret_cast<unsigned long long *>(&lost), (unsigned long long)miss);
  __syncthreads();
  if (threadIdx.x == 0) o.short_rows[0] = (int32_t)min(lost, (int64_t)0x7fffffff);
}

}  // namespace

hipError_t launch_kv_extend(const eb_kv_extend_op &o, hipStream_t s) {
  const int shift = __builtin_ctz((unsigned)o.page);
  // a row per thread up to 2 workgroups per CU's worth of rows, then several
  const int64_t wgs = ((int64_t)o.rows + kThreads - 1) / kThreads;
  const unsigned grid = (unsigned)(wgs < 1 ? 1 : (wgs > 512 ? 512 : wgs));
  const size_t lds = sizeof(int32_t) * (3 * (size_t)o.batch + 1);
  kv_extend_kernel<<<grid, kThreads, lds, s>>>(o, shift);
  return hipGetLastError();
}

}  // namespace eb

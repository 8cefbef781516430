// Bookkeeping of the paged cache (gfx950): which pages a sequence has, how many
// sequences have a page, and the pages' contents when they move.
//
// A page is free where refs is 0, and the free pages that a call takes are the lowest
// ones in ascending order, so what a call does follows from the state alone.  The plan of
// a call (which items are sound, how many pages they need, which ones they get) is made
// by one workgroup: it is a prefix sum over a few thousand numbers, and a second
// kernel over the whole chip moves the data and writes the table rows.
#pragma once

#include "paged.hpp"

namespace sats {

constexpr int kPlanThreads = 1024;
constexpr int kPlanPer = 16;  // refs that a thread looks at in one step of the free list's scan

struct PagesArgs {
  int32_t *table, *len, *refs;
  int64_t n_seqs, max_pages, n_pages;
  int page, shift;
  const int32_t *seqs, *other;  // items: sequences (null: 0, 1, ..); added tokens, or the forks' destinations
  const int32_t *begin, *end;   // ranges to release, or null
  int n;                        // items
  int32_t *status;              // [0] pages that were missing, [1] items left out; or null
  int32_t *n_used;
  // scratch
  int32_t *off;                 // [n + 1] first new page of an item in `ids`
  int32_t *ids;                 // free pages that the call takes / pages that move away
  int32_t *to;                  // compaction: where a page goes, [n_pages]
  int32_t *src, *dst, *valid;   // moves: from, to, tokens (0: none)
  int32_t *ctl;                 // [0] 1 where the call goes ahead, [1] moves
};

struct CopyArgs {
  char *k, *v;                  // the pools of every layer
  int64_t n_pages, layers;
  int n_kv, page, row_bytes;    // row: a token's head
  const int32_t *src, *dst, *valid;  // valid null: whole pages
  const int32_t *ctl;           // or null: n moves
  int n;
};

// Exclusive prefix over the workgroup of one int per thread; *total its sum.
__device__ __forceinline__ int plan_scan(int v, int *lds, int *total) {
  const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
  int inc = v;
#pragma unroll
  for (int d = 1; d < 64; d <<= 1) {
    const int o = __shfl_up(inc, d);
    if (lane >= d) inc += o;
  }
  __syncthreads();  // (lds may still be read by the call before)
  if (lane == 63) lds[wave] = inc;
  __syncthreads();
  int base = 0, sum = 0;
#pragma unroll
  for (int w = 0; w < kPlanThreads / 64; ++w) {
    if (w < wave) base += lds[w];
    sum += lds[w];
  }
  *total = sum;
  return base + inc - v;
}

__device__ __forceinline__ int item_seq(const PagesArgs &a, int i) { return a.seqs ? a.seqs[i] : i; }

// Calls f(page, rank) for the first `want` pages whose refs satisfy `is`, in ascending order,
// from page `from` up to `to`; the number found.
template <typename Is, typename F>
__device__ __forceinline__ int pages_where(const PagesArgs &a, int64_t from, int64_t to, int64_t want, int *lds, Is is, F f) {
  int64_t found = 0;
  for (int64_t base = from; base < to && found < want; base += kPlanThreads * kPlanPer) {
    const int64_t p0 = base + (int64_t)threadIdx.x * kPlanPer;
    uint32_t hit = 0;
#pragma unroll
    for (int i = 0; i < kPlanPer; ++i)
      if (p0 + i < to && is(a.refs[p0 + i])) hit |= 1u << i;
    int total;
    int64_t r = found + plan_scan(__popc(hit), lds, &total);
    for (; hit; hit &= hit - 1, ++r)
      if (r < want) f(p0 + __ffs(hit) - 1, r);
    found += total;
  }
  __syncthreads();
  return (int)(found < want ? found : want);
}

// The last page of a sequence of n tokens where n ends inside it and the page is there, else -1.
__device__ __forceinline__ int32_t part_page(const PagesArgs &a, int s, int n) {
  if (!(n & (a.page - 1)) || n >> a.shift >= a.max_pages) return -1;
  const int32_t p = a.table[s * a.max_pages + (n >> a.shift)];
  return p >= 0 && p < a.n_pages ? p : -1;
}

// Plan of an extension (FORK false: item i's sequence grows by other[i] tokens; a shared
// last page that it ends inside of is replaced by a copy) or of a fork (item i: sequence
// other[i], which has to be empty, becomes a copy of seqs[i]; its last page, where it is
// not full, is copied).  All items or, for want of pages, none.
template <bool FORK>
__global__ __launch_bounds__(kPlanThreads) void pages_plan_kernel(PagesArgs a) {
  __shared__ int lds[kPlanThreads / 64];
  __shared__ int left_out;
  if (threadIdx.x == 0) left_out = 0;
  __syncthreads();
  int total = 0;
  for (int base = 0; base < a.n; base += kPlanThreads) {
    const int i = base + threadIdx.x;
    int need = 0, src = -1;
    if (i < a.n) {
      const int64_t s = item_seq(a, i), o = a.other[i];
      bool ok = s >= 0 && s < a.n_seqs;
      const int64_t n = ok ? a.len[s] : 0;
      ok = ok && n >= 0 && n <= a.max_pages << a.shift;
      if (FORK) {
        ok = ok && o >= 0 && o < a.n_seqs && o != s && a.len[o] == 0;
        if (ok) src = part_page(a, (int)s, (int)n), need = src >= 0;
      } else {
        ok = ok && o >= 0 && n + o <= a.max_pages << a.shift;
        if (ok && o > 0) {
          src = part_page(a, (int)s, (int)n);
          if (src >= 0 && a.refs[src] <= 1) src = -1;
          need = (int)(((n + o + a.page - 1) >> a.shift) - ((n + a.page - 1) >> a.shift)) + (src >= 0);
        }
      }
      if (!ok) atomicAdd(&left_out, 1), need = -1;
      a.src[i] = src;
    }
    int sum;
    const int at = total + plan_scan(need > 0 ? need : 0, lds, &sum);
    if (i < a.n) a.off[i] = need < 0 ? -1 - at : at;  // (negative: left out)
    total += sum;
  }
  if (threadIdx.x == 0) a.off[a.n] = total;
  const int found = pages_where(a, 0, a.n_pages, total, lds, [](int r) { return r == 0; },
                                [&](int64_t p, int64_t r) { a.ids[r] = (int32_t)p; });
  const bool go = found == total;
  if (threadIdx.x == 0) {
    a.ctl[0] = go;
    a.ctl[1] = a.n;
    if (a.status) a.status[0] = total - found, a.status[1] = left_out;
  }
  if (!go) return;
  // what the items get (the scratch arrays written above are this workgroup's own)
  for (int i = threadIdx.x; i < a.n; i += kPlanThreads) {
    const int o = a.off[i];
    a.dst[i] = -1;
    a.valid[i] = 0;
    if (o < 0) continue;
    const int s = item_seq(a, i), n = a.len[s];
    if (a.src[i] >= 0) {
      a.dst[i] = a.ids[o];
      a.valid[i] = n & (a.page - 1);
    }
    if (FORK) {
      a.len[a.other[i]] = n;
    } else {
      if (a.src[i] >= 0 && n >> a.shift < a.max_pages) {
        a.table[s * a.max_pages + (n >> a.shift)] = a.ids[o];
        atomicSub(&a.refs[a.src[i]], 1);
      }
      a.len[s] = n + a.other[i];
    }
  }
  for (int r = threadIdx.x; r < total; r += kPlanThreads) a.refs[a.ids[r]] = 1;
  if (FORK) return;
  __syncthreads();
  // new pages into the table: page r of the call belongs to the last item that starts at or before it
  for (int r = threadIdx.x; r < total; r += kPlanThreads) {
    int lo = 0, hi = a.n - 1;
    while (lo < hi) {
      const int mid = (lo + hi + 1) >> 1, m = a.off[mid];
      if ((m < 0 ? -1 - m : m) <= r) lo = mid;
      else hi = mid - 1;
    }
    // (items that take nothing share their start with the next one; the last of them does not)
    const int s = item_seq(a, lo), at = r - a.off[lo] - (a.src[lo] >= 0);
    if (at < 0) continue;  // the copy of a shared page, above
    const int64_t j = ((a.len[s] - a.other[lo] + a.page - 1) >> a.shift) + at;
    if (j < a.max_pages) a.table[s * a.max_pages + j] = a.ids[r];
  }
}

// Releases the pages that lie wholly in tokens [begin, end) of an item's sequence; an
// end at or past its length also cuts the sequence there.  A workgroup per item.
__global__ __launch_bounds__(kThreads) void pages_free_kernel(PagesArgs a) {
  const int i = blockIdx.x;
  const int64_t s = item_seq(a, i);
  if (s < 0 || s >= a.n_seqs) return;
  const int64_t n = a.len[s], begin = a.begin ? (a.begin[i] > 0 ? a.begin[i] : 0) : 0;
  const bool cut = !a.end || a.end[i] >= n;
  const int64_t first = (begin + a.page - 1) >> a.shift, to = cut ? a.max_pages : a.end[i] >> a.shift;
  const int64_t last = to < a.max_pages ? to : a.max_pages;
  __syncthreads();  // every thread has read the length
  for (int64_t j = first + threadIdx.x; j < last; j += kThreads) {
    const int32_t p = a.table[s * a.max_pages + j];
    if (p < 0) continue;
    a.table[s * a.max_pages + j] = -1;
    if (p < a.n_pages) atomicSub(&a.refs[p], 1);
  }
  if (cut && threadIdx.x == 0 && begin < n) a.len[s] = (int32_t)begin;
}

// Plan of a compaction: of n_used pages in use, the ones at or past n_used move, in
// ascending order, to the free ones below it.
__global__ __launch_bounds__(kPlanThreads) void pages_compact_plan_kernel(PagesArgs a) {
  __shared__ int lds[kPlanThreads / 64];
  int64_t used = 0;
  for (int64_t base = 0; base < a.n_pages; base += kPlanThreads * kPlanPer) {
    int c = 0, total;
#pragma unroll
    for (int i = 0; i < kPlanPer; ++i) {
      const int64_t p = base + (int64_t)threadIdx.x * kPlanPer + i;
      if (p >= a.n_pages) break;
      c += a.refs[p] != 0;
      a.to[p] = (int32_t)p;
    }
    plan_scan(c, lds, &total);
    used += total;
  }
  const int64_t all = a.n_pages;
  const int holes = pages_where(a, 0, used, all, lds, [](int r) { return r == 0; },
                                [&](int64_t p, int64_t r) { a.dst[r] = (int32_t)p; });
  pages_where(a, used, a.n_pages, all, lds, [](int r) { return r != 0; }, [&](int64_t p, int64_t r) { a.src[r] = (int32_t)p; });
  for (int r = threadIdx.x; r < holes; r += kPlanThreads) {
    const int32_t p = a.src[r], q = a.dst[r];
    a.to[p] = q;
    a.refs[q] = a.refs[p];
    a.refs[p] = 0;
  }
  if (threadIdx.x == 0) {
    a.ctl[0] = 1;
    a.ctl[1] = holes;
    if (a.n_used) *a.n_used = (int32_t)used;
  }
}

// Table rows of a fork: the source's full pages shared, its part page replaced by the copy.
__global__ __launch_bounds__(kThreads) void pages_fork_rows_kernel(PagesArgs a) {
  const int i = blockIdx.y;
  const int64_t j = (int64_t)blockIdx.x * kThreads + threadIdx.x;
  if (!a.ctl[0] || j >= a.max_pages || a.off[i] < 0) return;
  const int64_t s = item_seq(a, i), o = a.other[i], n = a.len[s];
  int32_t p = -1;
  if (j < n >> a.shift) {
    p = a.table[s * a.max_pages + j];
    if (p < 0 || p >= a.n_pages) p = -1;
    else atomicAdd(&a.refs[p], 1);
  } else if (j == n >> a.shift && a.valid[i]) {
    p = a.dst[i];
  }
  a.table[o * a.max_pages + j] = p;
}

__global__ __launch_bounds__(kThreads) void pages_remap_kernel(PagesArgs a) {
  const int64_t i = (int64_t)blockIdx.x * kThreads + threadIdx.x;
  if (i >= a.n_seqs * a.max_pages) return;
  const int32_t p = a.table[i];
  if (p >= 0 && p < a.n_pages) a.table[i] = a.to[p];
}

// Moves the pages' contents: a wave takes the tokens of one (move, layer, keys or
// values, head), which are contiguous, in 16-byte pieces.
__global__ __launch_bounds__(kThreads) void pages_copy_kernel(CopyArgs a) {
  if (a.ctl && !a.ctl[0]) return;
  const int n = a.ctl ? a.ctl[1] : a.n;
  const int lane = threadIdx.x & 63;
  const int64_t per = a.layers * 2 * a.n_kv, units = per * n;
  for (int64_t u = ((int64_t)blockIdx.x * kThreads + threadIdx.x) >> 6; u < units;
       u += (int64_t)gridDim.x * (kThreads / 64)) {
    const int64_t m = u / per;
    const int x = (int)(u - m * per), h = x % a.n_kv, kv = x / a.n_kv % 2;
    const int64_t layer = x / a.n_kv / 2, src = a.src[m], dst = a.dst[m];
    const int valid = a.valid ? a.valid[m] : a.page;
    if (src < 0 || dst < 0 || src >= a.n_pages || dst >= a.n_pages || src == dst) continue;
    char *pool = kv ? a.v : a.k;
    const int64_t run = (int64_t)a.page * a.row_bytes;
    const char *from = pool + ((layer * a.n_pages + src) * a.n_kv + h) * run;
    char *to = pool + ((layer * a.n_pages + dst) * a.n_kv + h) * run;
    const int bytes = valid * a.row_bytes;
    for (int b = lane * 16; b < bytes; b += 64 * 16)
      *reinterpret_cast<u32x4 *>(to + b) = *reinterpret_cast<const u32x4 *>(from + b);
  }
}

}  // namespace sats

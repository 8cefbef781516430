// Bookkeeping of the paged cache (gfx950): which pages a sequence has, how many
// sequences have a page, and the pages' contents when they move.
//
// A page is free where refs is 0, and the free pages that a call takes are the lowest
// ones in ascending order, so what a call does follows from the state alone.  The plan of
// a call (which items are sound, how many pages they need, which ones they get) is made
// by one workgroup: it is a prefix sum over a few thousand numbers, and a second
// kernel over the whole chip moves the data, and writes the table rows of a fork and the
// numbers that a compaction changes.
//
// The plans are latency: 256 extensions 8.5 us (15 us the call, with the free before it), 64
// forks 6.2, a compaction of 768 pages 8.8.  The moves are a copy: 64 pages of 2 MB 29 to 34 us (part
// pages: 128 MB read and written, in runs of 256 bytes to 3.8 KB), 805 MB of a compaction 159 us,
// 5.1 TB/s.
#pragma once

#include "paged.hpp"

namespace sats {

constexpr int kPlanThreads = 1024;
constexpr int kPlanPer = 16;  // refs that a thread looks at in one step of the free list's scan
constexpr int kPlanItems = 1024, kPlanIds = 4096;  // items and new pages whose lists are held in LDS
constexpr int kNoPart = -2;  // an item's page to copy: none, and the page that its sequence ends inside of is not there

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
  int32_t *off;                 // [n] first new page of an item in `ids`
  int32_t *len_of;              // [n] its sequence's length
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
  int table_wgs;                // the launch's first workgroups, which see to the table
};

// Exclusive prefix over the workgroup of one number per thread; *total its sum.
template <typename N> __device__ __forceinline__ N plan_scan(N v, N *lds, N *total) {
  const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
  N inc = v;
#pragma unroll
  for (int d = 1; d < 64; d <<= 1) {
    const N o = __shfl_up(inc, d);
    if (lane >= d) inc += o;
  }
  __syncthreads();  // (lds may still be read by the call before)
  if (lane == 63) lds[wave] = inc;
  __syncthreads();
  N base = 0, sum = 0;
#pragma unroll
  for (int w = 0; w < kPlanThreads / 64; ++w) {
    if (w < wave) base += lds[w];
    sum += lds[w];
  }
  *total = sum;
  return base + inc - v;
}

__device__ __forceinline__ int item_seq(const PagesArgs &a, int i) { return a.seqs ? a.seqs[i] : i; }

// refs p0 .. p0 + 15 of pages below `to` (0xffffffff past it).
__device__ __forceinline__ void load_refs(const int32_t *refs, int64_t p0, int64_t to, int32_t (&r)[kPlanPer]) {
  if (p0 + kPlanPer <= to && ((uintptr_t)(refs + p0) & 15) == 0) {
#pragma unroll
    for (int i = 0; i < kPlanPer; i += 4) {
      const u32x4 v = *reinterpret_cast<const u32x4 *>(refs + p0 + i);
      r[i] = (int32_t)v.x, r[i + 1] = (int32_t)v.y, r[i + 2] = (int32_t)v.z, r[i + 3] = (int32_t)v.w;
    }
  } else {
#pragma unroll
    for (int i = 0; i < kPlanPer; ++i) r[i] = p0 + i < to ? refs[p0 + i] : -1;
  }
}

// Calls f(page, rank) for the first `want` pages from `from` up to `to` whose refs are 0 (FREE)
// or not, in ascending order; the number found.
template <bool FREE, typename F>
__device__ __forceinline__ int64_t pages_where(const int32_t *refs, int64_t from, int64_t to, int64_t want, int *lds, F f) {
  int64_t found = 0;
  for (int64_t base = from; base < to && found < want; base += kPlanThreads * kPlanPer) {
    const int64_t p0 = base + (int64_t)threadIdx.x * kPlanPer;
    int32_t v[kPlanPer];
    load_refs(refs, p0, to, v);
    uint32_t hit = 0;
#pragma unroll
    for (int i = 0; i < kPlanPer; ++i)
      if (p0 + i < to && (v[i] == 0) == FREE) hit |= 1u << i;
    int total;
    int64_t r = found + plan_scan((int)__popc(hit), lds, &total);
    for (; hit && r < want; hit &= hit - 1, ++r) f(p0 + __ffs(hit) - 1, r);
    found += total;
  }
  __syncthreads();
  return found < want ? found : want;
}

// The last page of a sequence of n tokens where n ends inside it and the page is there, else -1.
__device__ __forceinline__ int32_t part_page(const PagesArgs &a, int s, int n) {
  if (!(n & (a.page - 1)) || n >> a.shift >= a.max_pages) return -1;
  const int32_t p = a.table[s * a.max_pages + (n >> a.shift)];
  return p >= 0 && p < a.n_pages ? p : -1;
}

// Plan of an extension (FORK false: item i's sequence grows by other[i] tokens; a shared
// last page that it ends inside of is replaced by a copy, one that is not there by a new one) or of a fork (item i: sequence
// other[i], which has to be empty, becomes a copy of seqs[i]; its last page, where it is
// not full, is copied).  All items or, for want of pages, none.
template <bool FORK>
__global__ __launch_bounds__(kPlanThreads) void pages_plan_kernel(PagesArgs a) {
  __shared__ int lds[kPlanThreads / 64];
  __shared__ long long lds_need[kPlanThreads / 64];
  __shared__ int left_out;
  __shared__ int32_t lds_off[kPlanItems], lds_src[kPlanItems], lds_len[kPlanItems], lds_ids[kPlanIds];
  // what the steps hand to each other: in LDS where it fits (a step is then a few hundred
  // nanoseconds, in memory a microsecond)
  int32_t *off = a.n <= kPlanItems ? lds_off : a.off, *src_of = a.n <= kPlanItems ? lds_src : a.src;
  int32_t *len_of = a.n <= kPlanItems ? lds_len : a.len_of;
  if (threadIdx.x == 0) left_out = 0;
  __syncthreads();
  long long total = 0;  // (a sum of needs may pass 32 bits; where it can be met it does not)
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
          // (a sequence that was cut inside of pages that it had given back has no such page)
          if (src < 0) src = n & (a.page - 1) ? kNoPart : -1;
          else if (a.refs[src] <= 1) src = -1;
          need = (int)(((n + o + a.page - 1) >> a.shift) - ((n + a.page - 1) >> a.shift)) + (src != -1);
        }
      }
      if (!ok) atomicAdd(&left_out, 1), need = -1;
      src_of[i] = src;
      len_of[i] = (int32_t)n;
    }
    long long sum;
    const int at = (int)(total + plan_scan<long long>(need > 0 ? need : 0, lds_need, &sum));
    if (i < a.n) {
      off[i] = need < 0 ? -1 - at : at;  // (negative: left out)
      if (FORK) a.off[i] = off[i];
    }
    total += sum;
  }
  int32_t *ids = total <= kPlanIds ? lds_ids : a.ids;
  const int64_t found = pages_where<true>(a.refs, 0, a.n_pages, total, lds, [&](int64_t p, int64_t r) { ids[r] = (int32_t)p; });
  const bool go = found == total;
  if (threadIdx.x == 0) {
    a.ctl[0] = go;
    a.ctl[1] = a.n;
    if (a.status) a.status[0] = (int32_t)(total - found < 0x7fffffff ? total - found : 0x7fffffff), a.status[1] = left_out;
  }
  if (!go) return;
  // what the items get
  for (int i = threadIdx.x; i < a.n; i += kPlanThreads) {
    const int o = off[i], src = src_of[i], n = len_of[i];
    const bool copy = o >= 0 && src >= 0;
    a.src[i] = src;
    a.dst[i] = copy ? ids[o] : -1;
    a.valid[i] = copy ? n & (a.page - 1) : 0;
    if (o < 0) continue;
    if (FORK) {
      a.len[a.other[i]] = n;
    } else {
      const int s = item_seq(a, i);
      if (copy) {
        a.table[s * a.max_pages + (n >> a.shift)] = ids[o];
        atomicSub(&a.refs[src], 1);
      }
      a.len[s] = n + a.other[i];
    }
  }
  for (int r = threadIdx.x; r < total; r += kPlanThreads) {
    a.refs[ids[r]] = 1;
    if (FORK) continue;
    // page r of the call belongs to the last item that starts at or before it (items that take
    // nothing share their start with the next one; the last of them does not)
    int lo = 0, hi = a.n - 1;
    while (lo < hi) {
      const int mid = (lo + hi + 1) >> 1, m = off[mid];
      if ((m < 0 ? -1 - m : m) <= r) lo = mid;
      else hi = mid - 1;
    }
    const int at = r - off[lo] - (src_of[lo] != -1);
    if (at >= 0 || src_of[lo] == kNoPart)  // (not the copy of a shared page, above)
      a.table[item_seq(a, lo) * a.max_pages + ((len_of[lo] + a.page - 1) >> a.shift) + at] = ids[r];
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
    const int64_t p0 = base + (int64_t)threadIdx.x * kPlanPer;
    int32_t v[kPlanPer];
    load_refs(a.refs, p0, a.n_pages, v);
    int c = 0, total;
#pragma unroll
    for (int i = 0; i < kPlanPer; ++i)
      if (p0 + i < a.n_pages) c += v[i] != 0, a.to[p0 + i] = (int32_t)(p0 + i);
    plan_scan(c, lds, &total);
    used += total;
  }
  const int64_t all = a.n_pages;
  const int holes = (int)pages_where<true>(a.refs, 0, used, all, lds, [&](int64_t p, int64_t r) { a.dst[r] = (int32_t)p; });
  pages_where<false>(a.refs, used, a.n_pages, all, lds, [&](int64_t p, int64_t r) { a.src[r] = (int32_t)p; });
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

// What a call does to the table beside the moves of contents, by the first workgroups of
// their launch, an entry a thread.
enum { PAGES_ONLY = 0, PAGES_FORK = 1, PAGES_REMAP = 2 };
// A row of a fork: the source's full pages shared, its part page replaced by the copy.
__device__ __forceinline__ void fork_entry(const PagesArgs &a, int64_t e) {
  const int i = (int)(e / a.max_pages);
  const int64_t j = e - i * a.max_pages;
  if (i >= a.n || a.off[i] < 0) return;
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
__device__ __forceinline__ void remap_entry(const PagesArgs &a, int64_t e) {
  if (e >= a.n_seqs * a.max_pages) return;
  const int32_t p = a.table[e];
  if (p >= 0 && p < a.n_pages) a.table[e] = a.to[p];
}

// Moves the pages' contents: a wave takes the tokens of one (move, layer, keys or
// values, head), which are contiguous, in 16-byte pieces.
template <int TABLE>
__global__ __launch_bounds__(kThreads) void pages_copy_kernel(CopyArgs a, PagesArgs t) {
  if (a.ctl && !a.ctl[0]) return;
  if (TABLE != PAGES_ONLY && (int)blockIdx.x < a.table_wgs) {
    const int64_t e = (int64_t)blockIdx.x * kThreads + threadIdx.x;
    if (TABLE == PAGES_FORK) fork_entry(t, e);
    else remap_entry(t, e);
    return;
  }
  const int wg = (int)blockIdx.x - a.table_wgs, wgs = (int)gridDim.x - a.table_wgs;
  const int n = a.ctl ? a.ctl[1] : a.n;
  const int lane = threadIdx.x & 63;
  const int64_t per = a.layers * 2 * a.n_kv, units = per * n;
  for (int64_t u = ((int64_t)wg * kThreads + threadIdx.x) >> 6; u < units; u += (int64_t)wgs * (kThreads / 64)) {
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
      __builtin_nontemporal_store(__builtin_nontemporal_load(reinterpret_cast<const u32x4 *>(from + b)), reinterpret_cast<u32x4 *>(to + b));
  }
}

}  // namespace sats

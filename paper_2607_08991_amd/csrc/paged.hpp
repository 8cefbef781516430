// Device views of the paged cache and of a batch of sequences in it, shared by the
// serving kernels.  Contents of the device arrays are not trusted: lengths and page
// numbers are clamped or refused here, so that a wrong one reads and writes nothing
// outside the arrays.
#pragma once

#include "elem.hpp"

namespace sats {

struct BatchView {
  const int32_t *table, *q_start, *kv_len;
  int n_seqs;
  int64_t max_pages, n_tokens;
  int64_t max_q, max_kv;
};

struct PoolView {
  int64_t n_pages;
  int n_kv, page, shift;  // page = 1 << shift
};

// Sequence s: its first token, its new tokens and its length, in range.
struct SeqView {
  int64_t start, len;
  int n_new;
};
__device__ __forceinline__ SeqView seq_view(const BatchView &b, const PoolView &p, int s) {
  const int64_t lo = b.q_start[s], hi = b.q_start[s + 1];
  SeqView v;
  v.start = lo < 0 ? 0 : lo > b.n_tokens ? b.n_tokens : lo;
  const int64_t end = hi < v.start ? v.start : hi > b.n_tokens ? b.n_tokens : hi;
  v.n_new = (int)(end - v.start < b.max_q ? end - v.start : b.max_q);
  const int64_t top = b.max_kv < b.max_pages << p.shift ? b.max_kv : b.max_pages << p.shift;
  const int64_t n = b.kv_len[s];
  v.len = n < 0 ? 0 : n > top ? top : n;
  return v;
}

// The place of new token t in its sequence (*seq): kv_len - new tokens + index (-1: in none).
__device__ __forceinline__ int64_t token_place(const BatchView &b, int64_t t, int *seq) {
  int lo = 0, hi = b.n_seqs - 1;  // the last sequence that starts at or before t
  while (lo < hi) {
    const int mid = (lo + hi + 1) >> 1;
    if (b.q_start[mid] <= t) lo = mid;
    else hi = mid - 1;
  }
  *seq = lo;
  if (t < b.q_start[lo] || t >= b.q_start[lo + 1]) return -1;
  return (int64_t)b.kv_len[lo] - b.q_start[lo + 1] + t;
}

// Row (of head_dim elements) of token `place`'s head 0 in a layer's pool, or -1 where
// the table has no page for it.
__device__ __forceinline__ int64_t pool_row(const BatchView &b, const PoolView &p, int seq, int64_t place) {
  if (place < 0 || place >> p.shift >= b.max_pages) return -1;
  const int64_t page = b.table[seq * b.max_pages + (place >> p.shift)];
  if (page < 0 || page >= p.n_pages) return -1;
  return ((page * p.n_kv) << p.shift) + (place & (p.page - 1));
}

// V rounded elements at p (V > 1: 16 bytes, aligned).
template <typename T, int V> __device__ __forceinline__ void store_vec(T *p, const T (&o)[V]) {
  if constexpr (V == 1) {
    *p = o[0];
  } else {
    static_assert(V * sizeof(T) == 16, "16-byte stores");
    u32x4 v;
    __builtin_memcpy(&v, o, 16);
    *reinterpret_cast<u32x4 *>(p) = v;
  }
}

}  // namespace sats

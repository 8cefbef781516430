// Attention of new tokens over the paged cache (gfx950).
//
//   o = sum_j p_j v_j,  p = softmax over the visible keys of scale (q . k_j)
//
// A token at place i of its sequence sees the keys j <= i with i - j < window or
// j < sinks (window 0: all of them); keys whose page is absent are not seen.  One
// pass over the keys with the running maximum and sum of each row, float32.
//
// The rows that read one cache head (a token's n_q / n_kv query heads, token after
// token) share its keys, so a workgroup takes a tile of them.  Both kernels form
// S^T = K Q^T and O^T = V^T P^T: in the accumulators of S^T a lane holds four
// consecutive keys of one row, which is what a lane has to hold of P^T as the next
// product's operand, so P moves between no lanes, and a row's maximum, sum and factor
// are one lane's scalars.  V^T comes out of LDS by transposing reads.
//
// Keys that no row of the tile sees are read as zeros (from a row of zeros: whatever
// their slots hold does no harm) and left out of the softmax.  Where rows of a tile
// disagree on a key, p is exactly 0 for those that do not see it; in a block in which such
// a key's values hold infinities or NaN, the product takes these as zeros and they are
// added one by one for the rows that see them.
//
// Keys are taken in blocks: first the ones that hold the sinks, then those from the
// first row's window on.  The blocks of a tile can be split over several workgroups
// (`per_split` each); their partial results are joined by a second launch in a fixed
// order.
//
// Where sequences of a batch share a prefix, the work is in two phases (KeyPhase): the shared keys of a
// group for the rows of all its sequences, which are one tile's rows there, and then each sequence's
// own keys.  Every part of a row is kept, and joined as the parts of a split tile are.
#pragma once

#include "cache8.hpp"

namespace sats {

typedef short i16x4_t __attribute__((ext_vector_type(4)));
typedef float f32x16_t __attribute__((ext_vector_type(16)));
typedef __attribute__((address_space(3))) i16x4_t lds_i16x4;

struct AttendArgs {
  const void *q;
  int64_t q_stride;
  const void *k, *v;  // of the layer
  void *out;
  float *lse;         // or null
  BatchView batch;
  PoolView pool;
  int n_q, group, dim;  // group: query heads of a cache head
  float scale;
  int64_t window, sinks;
  int splits;         // workgroups a tile's blocks are split over, at most
  int per_split;      // key blocks of a split
  int small, large;   // which sequences the launch takes: at most 16 rows a head, more
  float *part;        // [tiles * n_kv][splits][rows of a tile][dim]
  float *part_ml;     // [tiles * n_kv][splits][rows of a tile][2]
  const uint8_t *k_scale, *v_scale;  // of the layer, 8-bit caches
  // shared prefixes: sequences seq_start[g] .. seq_start[g + 1] - 1 have their first shared[g] tokens in common
  int phase, n_groups;
  const int32_t *seq_start, *shared;
  int64_t max_tokens, max_len, max_own;  // of a group's new tokens, of a prefix, of a sequence's other keys
  int32_t *group_rows;  // or null: [n_groups][group_width] pages of the prefixes (attend_group_pages_kernel)
  int64_t group_width;
};
enum : int { kWhole = 0, kShared = 1, kOwn = 2 };  // phase: all keys, those of the groups, those of a sequence alone

// A call in phases: its tiles, of 16 rows and of 128, of the groups and of the sequences.  One launch takes them
// all, the groups' first, which take longest.  (By turns, 64 to 256 workgroups of each, they take as long.)
struct PhaseSet {
  int64_t tiles;
  int splits, per_split, small, large;  // as in AttendArgs
  int row0, rows;                       // its parts' rows among those of all sets
};
enum : int { kSharedSmall = 0, kSharedLarge = 1, kOwnSmall = 2, kOwnLarge = 3 };
struct RowParts {  // where a row's first part is of its own keys, and of its prefix (-1: none)
  int own, shared;
};
struct PhaseArgs {
  PhaseSet set[4];
  float *part, *part_ml;  // of all sets
  RowParts *parts;        // [n_tokens * n_q]
};

static __device__ u32x4 attend_zeros[64];  // a row of zeros
constexpr uint32_t kNoRow = 0x80000000u;  // an offset past every buffer: the load returns zeros
__device__ __forceinline__ __amdgpu_buffer_rsrc_t rows_rsrc(const char *base) {
  return __builtin_amdgcn_make_buffer_rsrc(const_cast<char *>(base), (short)0, 0x7fffffff, 0x00020000);
}

constexpr float kLog2e = 1.44269504088896340736f, kLn2 = 0.69314718055994530942f;
__device__ __forceinline__ float exp2_fast(float x) { return __builtin_amdgcn_exp2f(x); }

// A tile of rows: rows first .. first + count - 1 of (token, group) pairs of a sequence.
struct RowTile {
  int seq;          // -1: none (of a group: its first)
  int first, count;
  int64_t start, place0, len;  // sequence's first token; place of its first new token; length
  // (in phases) the first key that counts; the group's sequences, whose tokens the tile's rows are
  int64_t lo;
  int seq0, seq_end;
  const int32_t *pages;  // (in phases) their row of a table
};

__device__ __forceinline__ bool takes(const AttendArgs &a, int rows) { return rows <= 16 ? a.small : a.large; }

// Group g: its sequences, its tokens and the length of its prefix, in range.
struct GroupView {
  int s0, s1, n;
  int64_t start, len;
};
__device__ __forceinline__ GroupView group_view(const AttendArgs &a, int g) {
  const int lo = a.seq_start[g], hi = a.seq_start[g + 1];
  GroupView v;
  v.s0 = lo < 0 ? 0 : lo > a.batch.n_seqs ? a.batch.n_seqs : lo;
  v.s1 = hi < v.s0 ? v.s0 : hi > a.batch.n_seqs ? a.batch.n_seqs : hi;
  const int64_t n = a.batch.n_tokens, t0 = a.batch.q_start[v.s0], t1 = a.batch.q_start[v.s1];
  v.start = t0 < 0 ? 0 : t0 > n ? n : t0;
  const int64_t end = t1 < v.start ? v.start : t1 > n ? n : t1;
  v.n = v.s0 == v.s1 ? 0 : (int)(end - v.start < a.max_tokens ? end - v.start : a.max_tokens);
  int64_t top = a.batch.max_kv < a.batch.max_pages << a.pool.shift ? a.batch.max_kv : a.batch.max_pages << a.pool.shift;
  if (a.max_len < top) top = a.max_len;
  const int64_t p = a.shared[g];
  v.len = p < 0 ? 0 : p > top ? top : p;
  return v;
}
// The first group that sequence s is in, or -1.  (All lanes of a wave call it.)
__device__ __forceinline__ int group_of(const AttendArgs &a, int s) {
  const int lane = threadIdx.x & 63;
  for (int g0 = 0; g0 < a.n_groups; g0 += 64) {
    const int g = g0 + lane;
    const uint64_t in = __ballot(g < a.n_groups && a.seq_start[g < a.n_groups ? g : 0] <= s &&
                                 a.seq_start[g < a.n_groups ? g + 1 : 0] > s);
    if (in) return __builtin_amdgcn_readfirstlane(g0 + __builtin_ctzll(in));
  }
  return -1;
}
// The first sequence of a group that is as long as its prefix (where none is: that is as long as any), whose
// pages are read for all of them.  (All lanes call it.)
__device__ __forceinline__ int group_leader(const AttendArgs &a, const GroupView &v) {
  const int lane = threadIdx.x & 63;
  int most = 0;
  for (int s = v.s0 + lane; s < v.s1; s += 64) most = a.batch.kv_len[s] > most ? a.batch.kv_len[s] : most;
#pragma unroll
  for (int d = 32; d; d >>= 1) {
    const int o = __shfl_xor(most, d);
    most = o > most ? o : most;
  }
  if (most > v.len) most = (int)v.len;
  for (int base = v.s0; base < v.s1; base += 64) {
    const uint64_t long_enough = __ballot(base + lane < v.s1 && a.batch.kv_len[base + lane < v.s1 ? base + lane : v.s0] >= most);
    if (long_enough) return __builtin_amdgcn_readfirstlane(base + __builtin_ctzll(long_enough));
  }
  return v.s0;
}
// Under a window sequences give back the pages behind it, each its own: the rows of the table that are read for the
// groups then, where a place has the page of the longest sequence that has one there (so it has all keys that any of them
// has there).  32 places a workgroup, by 8 threads each: 64 sequences on 32000 shared keys under a window of 2048 take
// 184 us with it, 181 from one sequence's pages.  (The kernels that attend looking for a page that is not there
// themselves cost every call 1 to 14 %, by the registers that it takes.)
inline __global__ __launch_bounds__(256) void attend_group_pages_kernel(AttendArgs a) {
  __shared__ int64_t best[8][32];
  const GroupView v = group_view(a, blockIdx.y);
  const int at = threadIdx.x & 31, slice = threadIdx.x >> 5;
  const int64_t place = (int64_t)blockIdx.x * 32 + at, key = place << a.pool.shift;
  const bool in = key < v.len;
  int64_t most = -1;  // a length, then the page
  if (in) {
#pragma unroll 4
    for (int s = v.s0 + slice; s < v.s1; s += 8) {
      const int64_t kv = a.batch.kv_len[s], p = a.batch.table[s * a.batch.max_pages + place];
      if (p >= 0 && p < a.pool.n_pages && kv > key && (kv << 32 | p) > most) most = kv << 32 | p;
    }
  }
  best[slice][at] = most;
  __syncthreads();
  if (slice || !in) return;
#pragma unroll
  for (int i = 1; i < 8; ++i) most = best[i][at] > most ? best[i][at] : most;
  a.group_rows[blockIdx.y * a.group_width + place] = most < 0 ? -1 : (int)most;
}
// The place of token `tok` in the one of sequences s0 .. s1 - 1 that it is of (-1: of none).  (All lanes call it.)
__device__ __forceinline__ int64_t group_place(const AttendArgs &a, int s0, int s1, int64_t tok) {
  const int lane = threadIdx.x & 63;
  int64_t place = -1;
  bool done = false;
  for (int base = s0; base < s1; base += 64) {
    const bool in = base + lane < s1;
    const int end = in ? a.batch.q_start[base + lane + 1] : 0x7fffffff, kv = in ? a.batch.kv_len[base + lane] : 0;
    int at = 0;  // the first of these sequences that ends behind the token
#pragma unroll
    for (int d = 32; d; d >>= 1) at += __shfl(end, at + d - 1) <= tok ? d : 0;
    const int e = __shfl(end, at), n = __shfl(kv, at);
    if (!done && e > tok && base + at < s1) place = (int64_t)n - e + tok, done = true;
    if (__all(done)) break;
  }
  return place;
}

// Tiles of the groups, in their order: tile `t` of those that a launch takes.
template <int R> __device__ __forceinline__ RowTile find_group_tile(const AttendArgs &a, int t) {
  RowTile o;
  o.seq = -1;
  int g = -1, idx = 0;
  if (a.max_tokens * a.group <= R) {  // a tile per group
    if (t < a.n_groups) g = t;
  } else {
    const int lane = threadIdx.x & 63;
    int base = 0;
    for (int g0 = 0; g0 < a.n_groups; g0 += 64) {
      int n = 0;
      if (g0 + lane < a.n_groups) {
        const int rows = group_view(a, g0 + lane).n * a.group;
        if (takes(a, rows)) n = (rows + R - 1) / R;
      }
      int inc = n;
#pragma unroll
      for (int d = 1; d < 64; d <<= 1) {
        const int x = __shfl_up(inc, d);
        if (lane >= d) inc += x;
      }
      const uint64_t past = __ballot(base + inc > t);
      if (past) {
        const int at = __builtin_ctzll(past);
        g = g0 + at;
        idx = t - base - (__shfl(inc, at) - __shfl(n, at));
        break;
      }
      base += __shfl(inc, 63);
    }
  }
  if (g < 0) return o;
  g = __builtin_amdgcn_readfirstlane(g);
  idx = __builtin_amdgcn_readfirstlane(idx);
  const GroupView v = group_view(a, g);
  if (!v.n || !takes(a, v.n * a.group)) return o;
  o.seq = v.s0, o.seq0 = v.s0, o.seq_end = v.s1;
  o.pages = a.group_rows ? a.group_rows + g * a.group_width : a.batch.table + group_leader(a, v) * a.batch.max_pages;
  o.first = idx * R;
  const int rows = v.n * a.group - o.first;
  o.count = rows < R ? rows : R;
  o.start = v.start;
  o.place0 = 0;
  o.lo = 0, o.len = v.len;
  return o;
}

// Tile `t` of the batch (rows in tiles of R; a sequence's last rows, which see most keys, first).
template <int R, bool PHASED = false>
__device__ __forceinline__ RowTile find_tile(const AttendArgs &a, int t) {
  if (PHASED && a.phase == kShared) return find_group_tile<R>(a, t);
  RowTile o;
  o.seq = -1;
  o.lo = 0;
  const int lane = threadIdx.x & 63;
  int base = 0, idx = 0, n = 0;
  if (a.batch.max_q * a.group <= R) {  // a tile per sequence
    if (t < a.batch.n_seqs) {
      o.seq = t;
      const SeqView v = seq_view(a.batch, a.pool, t);
      if (!v.n_new || !takes(a, v.n_new * a.group)) o.seq = -1;
    }
  } else {
    for (int s0 = 0; s0 < a.batch.n_seqs; s0 += 64) {
      n = 0;
      if (s0 + lane < a.batch.n_seqs) {
        const SeqView v = seq_view(a.batch, a.pool, s0 + lane);
        if (takes(a, v.n_new * a.group)) n = (v.n_new * a.group + R - 1) / R;
      }
      int inc = n;
#pragma unroll
      for (int d = 1; d < 64; d <<= 1) {
        const int x = __shfl_up(inc, d);
        if (lane >= d) inc += x;
      }
      const uint64_t past = __ballot(base + inc > t);
      if (past) {
        const int at = __builtin_ctzll(past);
        o.seq = s0 + at;
        n = __shfl(n, at);
        idx = t - base - (__shfl(inc, at) - n);
        break;
      }
      base += __shfl(inc, 63);
    }
    idx = n - 1 - idx;
  }
  if (o.seq < 0) return o;
  o.seq = __builtin_amdgcn_readfirstlane(o.seq);
  idx = __builtin_amdgcn_readfirstlane(idx);
  const SeqView v = seq_view(a.batch, a.pool, o.seq);
  o.first = idx * R;
  const int rows = v.n_new * a.group - o.first;
  o.count = rows < R ? rows : R;
  o.start = v.start;
  // (as token_place counts: from the length as it is given)
  o.place0 = (int64_t)a.batch.kv_len[o.seq] - (a.batch.q_start[o.seq + 1] - v.start);
  o.len = v.len;
  if (PHASED && a.phase == kOwn) {
    o.pages = a.batch.table + o.seq * a.batch.max_pages;
    const int g = group_of(a, o.seq);
    if (g >= 0) o.lo = group_view(a, g).len;
    if (o.len - o.lo > a.max_own) o.len = o.lo + a.max_own;
  }
  return o;
}

// (Phases) the places of a tile's rows, row r in lane r % 64; they are those of one sequence, or of the
// sequences of a group.
template <int R> struct RowPlaces {
  static constexpr int kPer = (R + 63) / 64;
  int64_t p[kPer];
  __device__ __forceinline__ void find(const AttendArgs &a, const RowTile &t) {
#pragma unroll
    for (int i = 0; i < kPer; ++i) {
      const int r = (threadIdx.x & 63) + 64 * i, in = t.first + (r < t.count ? r : t.count - 1);
      p[i] = a.phase == kShared ? group_place(a, t.seq0, t.seq_end, t.start + in / a.group) : t.place0 + in / a.group;
    }
  }
  __device__ __forceinline__ int64_t of(int r) const {
    int64_t v = __shfl(p[0], r & 63);
    if constexpr (kPer > 1) {
      const int64_t w = __shfl(p[1], r & 63);
      v = r < 64 ? v : w;
    }
    return v;
  }
};
// One number for all lanes, as what branches and addresses of a wave are made from.
__device__ __forceinline__ int64_t uniform(int64_t v) {
  const uint32_t lo = __builtin_amdgcn_readfirstlane((int)(uint32_t)v), hi = __builtin_amdgcn_readfirstlane((int)(v >> 32));
  return (int64_t)((uint64_t)hi << 32 | lo);
}
// The smallest and largest of a number of each of N lanes (a power of two; other lanes have the same).
template <int N> __device__ __forceinline__ void range_of(int64_t v, int64_t *low, int64_t *high) {
  int64_t lo = v, hi = v;
#pragma unroll
  for (int d = 1; d < N; d <<= 1) {
    const int64_t x = __shfl_xor(lo, d), y = __shfl_xor(hi, d);
    lo = x < lo ? x : lo, hi = y > hi ? y : hi;
  }
  *low = uniform(lo), *high = uniform(hi);
}

// The blocks of B keys that a tile's rows see.
struct KeyBlocks {
  int64_t low, high;  // places of the first and last row
  int n_sink;         // blocks of sinks before the window
  int64_t first;      // first block of the window
  int n;              // all
  int64_t lo, sink0;  // (phases) the first key, and its block
};
template <int B> __device__ __forceinline__ void count_blocks(const AttendArgs &a, int64_t lo, int64_t len, KeyBlocks &k) {
  const int64_t end = k.high + 1 < len ? k.high + 1 : len;
  int64_t from = a.window ? k.low - a.window + 1 : 0;
  from = from < lo ? lo : from;
  k.first = from / B;
  k.lo = lo, k.sink0 = lo / B;
  const int64_t last = end > 0 ? (end + B - 1) / B : 0, sink = a.window ? (a.sinks + B - 1) / B : 0;
  int64_t s = sink < k.first ? sink : k.first;
  if (s > last) s = last;
  k.n_sink = (int)(s > k.sink0 ? s - k.sink0 : 0);
  k.n = k.n_sink + (int)(last > k.first ? last - k.first : 0);
}
template <int B> __device__ __forceinline__ KeyBlocks key_blocks(const AttendArgs &a, const RowTile &t) {
  KeyBlocks k;
  k.low = t.place0 + t.first / a.group;
  k.high = t.place0 + (t.first + t.count - 1) / a.group;
  count_blocks<B>(a, 0, t.len, k);
  return k;
}
// (Phases: all lanes of a wave call it.)
template <int B, int R> __device__ __forceinline__ KeyBlocks key_blocks(const AttendArgs &a, const RowTile &t, const RowPlaces<R> &p) {
  KeyBlocks k;
  if (a.phase == kShared) {
    range_of<64>(p.p[0], &k.low, &k.high);
    if constexpr (RowPlaces<R>::kPer > 1) {
      int64_t low, high;
      range_of<64>(p.p[1], &low, &high);
      k.low = low < k.low ? low : k.low, k.high = high > k.high ? high : k.high;
    }
  } else {
    k.low = t.place0 + t.first / a.group;
    k.high = t.place0 + (t.first + t.count - 1) / a.group;
  }
  count_blocks<B>(a, t.lo, t.len, k);
  return k;
}
__device__ __forceinline__ int64_t block_key(const KeyBlocks &k, int b, int keys) {
  return (b < k.n_sink ? k.sink0 + b : k.first + (b - k.n_sink)) * keys;
}

// Which keys of the block from j0 on the token at `place` sees: key j0 + i where
// i <= last and (i >= from or i < sink).  (Differences cut off to 32 bits: a block is short.)
struct Sight {
  int last, from, sink;
  __device__ __forceinline__ bool sees(int i) const { return (i <= last) & ((i >= from) | (i < sink)); }
};
__device__ __forceinline__ int cut_off(int64_t v) {
  return (int)(v < -(1 << 30) ? -(1 << 30) : v > 1 << 30 ? 1 << 30 : v);
}
__device__ __forceinline__ Sight sight_of(const AttendArgs &a, int64_t place, int64_t j0) {
  return {cut_off(place - j0), a.window ? cut_off(place - j0 - a.window + 1) : 0, cut_off(a.sinks - j0)};
}
// Whether any row of a tile at places low .. high sees key j.
template <bool PHASED = false>
__device__ __forceinline__ bool any_sees(const AttendArgs &a, const KeyBlocks &k, int64_t len, int64_t j) {
  return j < len && (!PHASED || j >= k.lo) && j <= k.high && (!a.window || k.low - j < a.window || j < a.sinks);
}

// The table's entry for key j where some row sees it, else -1.  (Whether it is a page is looked at where it is
// used, a step later: a comparison here would wait for it, and for every load before it.)
template <bool PHASED = false>
__device__ __forceinline__ int key_entry(const AttendArgs &a, const RowTile &t, const KeyBlocks &k, int64_t j) {
  int p = -1;
  if (any_sees<PHASED>(a, k, t.len, j)) p = (PHASED ? t.pages : a.batch.table + t.seq * a.batch.max_pages)[j >> a.pool.shift];
  return p;
}
__device__ __forceinline__ int page_or_none(const AttendArgs &a, int entry) {
  return entry >= 0 && entry < a.pool.n_pages ? entry : -1;
}

// Four elements of a row's result, from dim d on: o and l relative to the maximum m.
template <typename T>
__device__ __forceinline__ void put_row(const AttendArgs &a, const RowTile &t, int r, int kvh, int d, const f32x4 &o,
                                        float m, float l) {
  const int64_t tok = t.start + (t.first + r) / a.group;
  const int64_t row = tok * a.n_q + kvh * a.group + (t.first + r) % a.group;
  const float f = l == 0.0f ? 0.0f : 1.0f / l;
  if (d < a.dim) {
    T x[4];
#pragma unroll
    for (int i = 0; i < 4; ++i) x[i] = Elem<T>::round(l == 0.0f ? 0.0f : o[i] * f);
    T *dst = (T *)a.out + row * a.dim + d;
    if constexpr (sizeof(T) == 2) {
      uint64_t w;
      __builtin_memcpy(&w, x, 8);
      *reinterpret_cast<uint64_t *>(dst) = w;
    } else {
      *reinterpret_cast<f32x4 *>(dst) = f32x4{x[0], x[1], x[2], x[3]};
    }
  }
  if (d == 0 && a.lse) a.lse[row] = l == 0.0f ? -INFINITY : (m + __log2f(l)) * kLn2;
}
// The same as a part: `at` counts the rows of (tile, head, split) slots.
__device__ __forceinline__ void put_part(const AttendArgs &a, int64_t at, int d, const f32x4 &o, float m, float l) {
  if (d < a.dim) *reinterpret_cast<f32x4 *>(a.part + at * a.dim + d) = o;
  if (d == 0) a.part_ml[at * 2] = m, a.part_ml[at * 2 + 1] = l;
}

// (Phases) split z of a tile has nothing to add: its part is empty.
template <int R> __device__ __forceinline__ void put_nothing(const AttendArgs &a, const RowTile &t, int x, int z) {
  if ((int)threadIdx.x >= t.count) return;
  const int64_t at = ((int64_t)x * a.splits + z) * R + threadIdx.x;
  a.part_ml[at * 2] = -INFINITY, a.part_ml[at * 2 + 1] = 0.0f;
}
// The set of workgroup `block` of a call in phases, into a; its number there (tiles and heads first, then splits).
__device__ __forceinline__ int take_set(AttendArgs &a, const PhaseArgs &p, int64_t block, int *x, int *z) {
  int i = kSharedLarge;
  int64_t heads = p.set[i].tiles * a.pool.n_kv;
  for (int next : {kSharedSmall, kOwnLarge, kOwnSmall}) {
    const int64_t wgs = heads * p.set[i].splits;
    if (block < wgs) break;
    block -= wgs;
    i = next, heads = p.set[i].tiles * a.pool.n_kv;
  }
  const PhaseSet &s = p.set[i];
  a.phase = i >= kOwnSmall ? kOwn : kShared;
  a.part = p.part + (int64_t)s.row0 * a.dim, a.part_ml = p.part_ml + (int64_t)s.row0 * 2;
  a.splits = s.splits, a.per_split = s.per_split, a.small = s.small, a.large = s.large;
  *z = (int)(block / heads), *x = (int)(block % heads);
  return i;
}
// The parts of an own tile's rows, in p.parts (by the tile's first split; all lanes call it).
template <int R>
__device__ __forceinline__ void put_row_parts(const AttendArgs &a, const PhaseArgs &p, int x, int z) {
  if (a.phase != kOwn || z) return;
  const RowTile t = find_tile<R, true>(a, x / a.pool.n_kv);
  if (t.seq < 0) return;
  const int kvh = x % a.pool.n_kv, lane = threadIdx.x & 63;
  // the group's rows: where this tile's first is among them, which launch took them, tiles before them
  int in0 = -1, rows_g = 0, c = 0, tile0 = 0;
  const int g = group_of(a, t.seq);
  if (g >= 0) {
    const GroupView v = group_view(a, g);
    rows_g = v.n * a.group;
    in0 = (int)(t.start - v.start) * a.group + t.first;
    c = rows_g <= 16 ? (p.set[kSharedSmall].small ? kSharedSmall : kSharedLarge)
                     : (p.set[kSharedLarge].large ? kSharedLarge : kSharedSmall);
    const int tall = c == kSharedLarge ? 128 : 16;
    if (a.max_tokens * a.group > tall) {
      for (int g0 = 0; g0 < g; g0 += 64) {
        int m = 0;
        if (g0 + lane < g) {
          const int of = group_view(a, g0 + lane).n * a.group;
          if (of <= 16 ? p.set[c].small : p.set[c].large) m = (of + tall - 1) / tall;
        }
#pragma unroll
        for (int d = 32; d; d >>= 1) m += __shfl_xor(m, d);
        tile0 += m;
      }
    } else {
      tile0 = g;
    }
  }
  const PhaseSet &pre = p.set[c], &own = p.set[R == 16 ? kOwnSmall : kOwnLarge];
  const int tall = c == kSharedLarge ? 128 : 16, r = threadIdx.x, in = in0 + r, tile = tile0 + in / tall;
  if (r >= t.count) return;
  RowParts o = {own.row0 + (x * own.splits) * R + r, -1};
  if (in0 >= 0 && in < rows_g && tile < pre.tiles)  // (groups that overlap may have more tiles than a launch has)
    o.shared = pre.row0 + (tile * a.pool.n_kv + kvh) * pre.splits * tall + in % tall;
  const int64_t tok = t.start + (t.first + r) / a.group;
  p.parts[tok * a.n_q + kvh * a.group + (t.first + r) % a.group] = o;
}

template <typename T> __device__ __forceinline__ bool odd_value(const u32x4 &q) {  // an infinity or NaN among them
  bool odd = false;
#pragma unroll
  for (int i = 0; i < 4; ++i) {
    if constexpr (sizeof(T) == 2) odd |= (q[i] & 0x7f80u) == 0x7f80u || (q[i] & 0x7f800000u) == 0x7f800000u;
    else odd |= (q[i] & 0x7f800000u) == 0x7f800000u;
  }
  return odd;
}

__device__ __forceinline__ bool odd_bits(uint16_t b) { return (b & 0x7f80u) == 0x7f80u; }
__device__ __forceinline__ i16x4_t sane(i16x4_t v) {  // infinities and NaN as zeros
#pragma unroll
  for (int i = 0; i < 4; ++i)
    if (odd_bits((uint16_t)v[i])) v[i] = 0;
  return v;
}
__device__ __forceinline__ bool odd_of(float v) { return (__float_as_uint(v) & 0x7f800000u) == 0x7f800000u; }

template <int N> struct Const { static constexpr int value = N; };
struct Plain { static constexpr bool kOdd = false; };
struct Odd { static constexpr bool kOdd = true; };

// ------------------------------------------------------------------ tiles of 16 rows

// Decode and short chunks (and float32 of any length): each of the four waves takes
// every fourth block of a tile's keys with a softmax of its own, joined in LDS at the end.
// K goes from memory straight to the lanes that multiply it; V through LDS, a wave's
// own part, for the transposing reads.  The next block's loads are in flight while
// one is worked on.
//
// Bound by the cache's bytes: 64 sequences of 500 to 8000 keys (8 heads of 128, four rows each,
// bf16, 711 MB) take 146 us with the join, 4.9 TB/s (counters: 712 MB fetched, no bank
// conflicts); one sequence of 32768 keys (134 MB) 29.7 us in this kernel, 4.5 TB/s, and 8.3 in
// the join.  Of other widths the same sequences reach, in TB/s, 4.2 (64), 3.8 (80), 3.3 (96, which
// spills registers at three waves a SIMD), 3.0 (136) to 4.3 (256: one workgroup a compute unit);
// float32 4.8 at 128.  Few keys are latency, not products: 12 heads of 80 on 4 (float32), a token
// alone on 16 keys takes 6.6 us, the sequence, the table, the keys and the end, each after the
// other; six sequences in 208 tiles with a window of 16 9.2, and from there 3.3 us for each block of
// a wave (window 512, three blocks: 22.2; 1024, six: 32.2), of which its 40 products are 1.3.
// 16 rows are what a matrix instruction has columns for.  Of float32 it is eight
// products of 16 x 16 x 4 where bf16 has one of 16 x 16 x 32: a chunk of 512 tokens on 1000
// earlier ones (32 heads of 128) runs at 56 TFLOP/s, a third of a large float32 product's 154.
template <typename T> struct RowsOf {
  static constexpr int kKeys = sizeof(T) == 2 ? 32 : 16;  // keys of a block
};

// The end of a tile of 16 rows: the sums of its four waves (row lane % 16; m, l: of this lane's group's keys)
// into results, or into split z's part.  lds: 16 x DT floats for each wave.
template <typename T, int DT>
__device__ __forceinline__ void finish_rows(const AttendArgs &a, const RowTile &t, int x, int z, bool split, float m, float l,
                                            const f32x4 (&acc)[DT / 16], uint8_t *mine, uint8_t *const (&lds)[4], float (&ml)[4][16][2]) {
  const int kvh = x % a.pool.n_kv;
  const int lane = threadIdx.x & 63, w = threadIdx.x >> 6, row = lane & 15, g = lane >> 4;
  // a row's sums: over the four lane groups, then over the waves
  l += __shfl_xor(l, 16);
  l += __shfl_xor(l, 32);
  if (g == 0) ml[w][row][0] = m, ml[w][row][1] = l;
  __syncthreads();
  float top = -INFINITY, fw[4], total = 0.0f;
#pragma unroll
  for (int i = 0; i < 4; ++i) top = fmaxf(top, ml[i][row][0]);
  const float at0 = top == -INFINITY ? 0.0f : top;
#pragma unroll
  for (int i = 0; i < 4; ++i) {
    fw[i] = exp2_fast(ml[i][row][0] - at0);
    total += ml[i][row][1] * fw[i];
  }
  // each wave's sums, scaled to the common maximum: [dim / 4][row][4]
#pragma unroll
  for (int o = 0; o < DT / 16; ++o)
    *reinterpret_cast<f32x4 *>(reinterpret_cast<float *>(mine) + ((4 * o + g) * 16 + row) * 4) = acc[o] * fw[w];
  __syncthreads();
  for (int i = threadIdx.x >> 4; i < DT / 4; i += 16) {
    f32x4 o = f32x4{0, 0, 0, 0};
#pragma unroll
    for (int y = 0; y < 4; ++y) o += *reinterpret_cast<const f32x4 *>(reinterpret_cast<const float *>(lds[y]) + (i * 16 + row) * 4);
    if (row >= t.count) continue;
    if (split) put_part(a, ((int64_t)x * a.splits + z) * 16 + row, 4 * i, o, top, total);
    else put_row<T>(a, t, row, kvh, 4 * i, o, top, total);
  }
}

// FULL: heads of DT dims.  Else every load leaves out the dims that a head has not (they are the
// next slot's, or lie behind the cache), and up to DT = 128 the products do too.  Of 256 they
// multiply zeros there: leaving them out spills 989 registers (bf16; 683 float32), all of them none.
// x: tile and cache head; z: split.  lds: kPart bytes for each wave.
template <typename T, int DT> struct RowsPart {
  // V's rows lie a little apart, so that the rows that are read together (bf16: 32 bytes of 8
  // rows; float32: 64 bytes of 4 rows, 4 apart) are in different banks
  static constexpr int kPitch = DT * (int)sizeof(T) + (sizeof(T) == 2 ? 32 : 16);
  static constexpr int kV = RowsOf<T>::kKeys * kPitch;
  static constexpr int kBytes = kV > 16 * DT * 4 ? kV : 16 * DT * 4;  // (the waves' sums are joined there)
};
template <typename T, int DT, bool FULL, bool PHASED>
__device__ __forceinline__ void attend_rows(const AttendArgs &a, int x, int z, uint8_t *const (&lds)[4], float (&ml)[4][16][2]) {
  constexpr int kKeys = RowsOf<T>::kKeys, kVec = Elem<T>::kVec, kRow = DT * (int)sizeof(T), kChunks = kRow / 16;
  constexpr bool kSkip = !FULL && DT <= 128;
  constexpr int kTiles = kKeys / 16, kSteps = kChunks / 4, kLoads = kKeys * kChunks / 64, kOut = DT / 16;
  constexpr int kPitch = RowsPart<T, DT>::kPitch;

  const int kvh = x % a.pool.n_kv;
  const RowTile t = find_tile<16, PHASED>(a, x / a.pool.n_kv);
  if (t.seq < 0) return;
  RowPlaces<16> places;
  if constexpr (PHASED) places.find(a, t);
  KeyBlocks kb;
  if constexpr (PHASED) kb = key_blocks<kKeys>(a, t, places);
  else kb = key_blocks<kKeys>(a, t);
  const int parts = kb.n > a.per_split ? (kb.n + a.per_split - 1) / a.per_split : 1;
  if (z >= parts) {
    if constexpr (PHASED) put_nothing<16>(a, t, x, z);
    return;
  }
  const int b_end = kb.n < (z + 1) * a.per_split ? kb.n : (z + 1) * a.per_split;
  const int lane = threadIdx.x & 63, w = threadIdx.x >> 6, row = lane & 15, g = lane >> 4;
  int64_t place;
  if constexpr (PHASED) place = places.of(row);
  else place = t.place0 + (t.first + (row < t.count ? row : t.count - 1)) / a.group;
  const bool several = kb.low != kb.high;

  // Q as the second operand: this lane's row, its pieces of k
  u32x4 qv[kSteps];
  {
    const int r = t.first + (row < t.count ? row : t.count - 1);
    const T *q = (const T *)a.q + (t.start + r / a.group) * a.q_stride + (int64_t)(kvh * a.group + r % a.group) * a.dim;
#pragma unroll
    for (int s = 0; s < kSteps; ++s) {
      const int c = g + 4 * s;
      qv[s] = c * kVec < a.dim ? *reinterpret_cast<const u32x4 *>(q + c * kVec) : u32x4{0, 0, 0, 0};
    }
  }
  const float scale2 = a.scale * kLog2e;
  const char *zeros = reinterpret_cast<const char *>(attend_zeros);
  const int64_t head_bytes = ((int64_t)kvh << a.pool.shift) * a.dim * (int)sizeof(T);
  const int64_t page_bytes = ((int64_t)a.pool.n_kv << a.pool.shift) * a.dim * (int)sizeof(T);
  const char *kp = (const char *)a.k + head_bytes, *vp = (const char *)a.v + head_bytes;
  const int row_bytes = a.dim * (int)sizeof(T);

  u32x4 kr[kLoads], vr[kLoads];
  auto entry_of = [&](int b) {  // of key lane % kKeys of a block
    return b < b_end ? key_entry<PHASED>(a, t, kb, block_key(kb, b, kKeys) + (lane & (kKeys - 1))) : -1;
  };
  auto load = [&](int b, int page, uint32_t there) {
    const int j0 = (int)(block_key(kb, b, kKeys) & (a.pool.page - 1));  // (blocks and pages are powers of two)
    if (a.pool.shift >= 4) {
      // 16 keys are in one page: one address for them, and offsets that read zeros (past the
      // buffer's end) for keys and dims that are not there
#pragma unroll
      for (int kt = 0; kt < kTiles; ++kt) {
        const uint32_t here = there >> (16 * kt) & 0xffffu;
        const int64_t p = here ? __builtin_amdgcn_readlane(page, 16 * kt + __builtin_ctz(here)) : 0;
        const int64_t at = p * page_bytes + ((j0 + 16 * kt) & (a.pool.page - 1)) * row_bytes;
        const __amdgpu_buffer_rsrc_t rk = rows_rsrc(kp + at), rv = rows_rsrc(vp + at);
        const uint32_t k_off = here >> row & 1 ? row * row_bytes + g * 16 : kNoRow;
#pragma unroll
        for (int s = 0; s < kSteps; ++s)
          kr[kt * kSteps + s] = __builtin_bit_cast(
              u32x4, __builtin_amdgcn_raw_buffer_load_b128(
                         rk, FULL || (4 * s + g) * kVec < a.dim ? k_off + 64 * s : kNoRow, 0, 0));
#pragma unroll
        for (int i = 0; i < kLoads / kTiles; ++i) {
          const int r = (i * 64 + lane) / kChunks, c = (i * 64 + lane) % kChunks;
          const uint32_t off = (here >> r & 1) && (FULL || c * kVec < a.dim) ? r * row_bytes + c * 16 : kNoRow;
          vr[kt * (kLoads / kTiles) + i] = __builtin_bit_cast(u32x4, __builtin_amdgcn_raw_buffer_load_b128(rv, off, 0, 0));
        }
      }
      return;
    }
    // address of piece c of key i's row
    auto addr = [&](const char *base, int i, int c) {
      const int p = __shfl(page, i);
      const int slot = (j0 + i) & (a.pool.page - 1);
      return p >= 0 && c * kVec < a.dim ? base + p * page_bytes + slot * row_bytes + c * 16 : zeros;
    };
#pragma unroll
    for (int kt = 0; kt < kTiles; ++kt)
#pragma unroll
      for (int s = 0; s < kSteps; ++s)
        kr[kt * kSteps + s] = *reinterpret_cast<const u32x4 *>(addr(kp, 16 * kt + row, g + 4 * s));
#pragma unroll
    for (int i = 0; i < kLoads; ++i) {
      const int at = i * 64 + lane;
      vr[i] = *reinterpret_cast<const u32x4 *>(addr(vp, at / kChunks, at % kChunks));
    }
  };

  f32x4 acc[kOut];
#pragma unroll
  for (int i = 0; i < kOut; ++i) acc[i] = f32x4{0, 0, 0, 0};
  float m = -INFINITY, l = 0.0f;
  uint8_t *mine = w == 0 ? lds[0] : w == 1 ? lds[1] : w == 2 ? lds[2] : lds[3];

  int b = z * a.per_split + w;
  int page = page_or_none(a, entry_of(b));
  uint32_t there = (uint32_t)__ballot(page >= 0);
  if (b < b_end) load(b, page, there);
  int entry_next = entry_of(b + 4);
  for (; b < b_end; b += 4) {
    const int64_t j0 = block_key(kb, b, kKeys);
    const uint32_t here = there & (uint32_t)((1ull << kKeys) - 1);
    const bool whole = here == (uint32_t)((1ull << kKeys) - 1) && j0 + kKeys - 1 <= kb.low &&
                       (!a.window || kb.high - j0 < a.window || j0 + kKeys <= a.sinks);
    // scores: lane (row, keys 16 kt + 4 g + i)
    f32x4 s[kTiles], s2 = {0, 0, 0, 0};  // (s2: float32's second chain of products)
#pragma unroll
    for (int kt = 0; kt < kTiles; ++kt) {
      s[kt] = f32x4{0, 0, 0, 0};
#pragma unroll
      for (int st = 0; st < kSteps; ++st) {
        if (kSkip && st * 4 * kVec >= a.dim) break;
        if constexpr (sizeof(T) == 2) {
          s[kt] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(__builtin_bit_cast(bf16x8_t, kr[kt * kSteps + st]),
                                                          __builtin_bit_cast(bf16x8_t, qv[st]), s[kt], 0, 0, 0);
        } else {
#pragma unroll
          for (int e = 0; e < 4; ++e) {
            f32x4 &to = e & 1 ? s2 : s[0];
            to = __builtin_amdgcn_mfma_f32_16x16x4f32(__uint_as_float(kr[st][e]), __uint_as_float(qv[st][e]), to, 0, 0, 0);
          }
        }
      }
    }
    if constexpr (sizeof(T) == 4) s[0] += s2;
    // V to LDS, and the next block's loads
    bool odd = false;
    if (several && !whole) {
#pragma unroll
      for (int i = 0; i < kLoads; ++i) odd |= odd_value<T>(vr[i]);
      odd = __any(odd);
    }
#pragma unroll
    for (int i = 0; i < kLoads; ++i) {
      const int at = i * 64 + lane, r = at / kChunks;
      *reinterpret_cast<u32x4 *>(mine + r * kPitch + at % kChunks * 16) = vr[i];
    }
    page = page_or_none(a, entry_next);
    there = (uint32_t)__ballot(page >= 0);
    if (b + 4 < b_end) {
      load(b + 4, page, there);
      entry_next = entry_of(b + 8);
    }
#pragma unroll
    for (int kt = 0; kt < kTiles; ++kt) s[kt] *= scale2;
    if (!whole) {
      const Sight sight = sight_of(a, place, j0);
      const uint32_t mine = here >> (4 * g);
#pragma unroll
      for (int kt = 0; kt < kTiles; ++kt)
#pragma unroll
        for (int i = 0; i < 4; ++i)
          s[kt][i] = ((mine >> (16 * kt + i) & 1) != 0) & sight.sees(16 * kt + 4 * g + i) ? s[kt][i] : -INFINITY;
    }
    float top = -INFINITY;
#pragma unroll
    for (int kt = 0; kt < kTiles; ++kt)
#pragma unroll
      for (int i = 0; i < 4; ++i) top = fmaxf(top, s[kt][i]);
    top = fmaxf(top, __shfl_xor(top, 16));
    top = fmaxf(top, __shfl_xor(top, 32));
    const float mn = fmaxf(m, top), at0 = mn == -INFINITY ? 0.0f : mn, f = exp2_fast(m - at0);
    m = mn;
    float sum = 0.0f;
#pragma unroll
    for (int kt = 0; kt < kTiles; ++kt)
#pragma unroll
      for (int i = 0; i < 4; ++i) {
        // (a key that is not seen weighs 0 also where the maximum is NaN)
        s[kt][i] = exp2_fast(s[kt][i] - at0);
        sum += s[kt][i];
      }
    l = l * f + sum;
#pragma unroll
    for (int i = 0; i < kOut; ++i) acc[i] *= f;
    auto product = [&](auto kind) {
      constexpr bool kOdd = decltype(kind)::kOdd;
      if constexpr (sizeof(T) == 2) {
        // contraction slot (g, e): key 4 g + e of tile 0, then of tile 1.  A weight goes in as its
        // first 8 bits and, in a second product, the rest (to 16): the cache's bytes are the bound,
        // so it costs 0 to 1 % (64 sequences 148.0 us both ways, 4 tokens each 156.1 -> 157.3), and the
        // error is the result's rounding alone (0.0017 of the norm, 0.0021 with 8 bits).  The rest
        // of a weight above 0 is above 0 (by 2^-20 of it), so that an infinity that is seen stays one.
        bf16x8_t p, rest;
#pragma unroll
        for (int e = 0; e < 8; ++e) {
          const float x = s[e >> 2][e & 3], top = __uint_as_float(__float_as_uint(x) & 0xffff0000u);
          p[e] = (__bf16)top, rest[e] = (__bf16)fmaf(x, 1.0f + 0x1p-20f, -top);
        }
#pragma unroll
        for (int o = 0; o < kOut; ++o) {
          if (kSkip && 16 * o >= a.dim) break;
          i16x4_t v2[2];
#pragma unroll
          for (int kt = 0; kt < 2; ++kt) {
            const int r = 16 * kt + 4 * g + (row >> 2);
            v2[kt] = __builtin_amdgcn_ds_read_tr16_b64_v4i16((lds_i16x4 *)(mine + r * kPitch + 32 * o + (row & 3) * 8));
            if (kOdd) v2[kt] = sane(v2[kt]);
          }
          bf16x8_t v8;
          __builtin_memcpy(&v8, v2, 16);
          acc[o] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(v8, p, acc[o], 0, 0, 0);
          acc[o] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(v8, rest, acc[o], 0, 0, 0);
        }
      } else {
#pragma unroll
        for (int o = 0; o < kOut; ++o) {
          if (kSkip && 16 * o >= a.dim) break;
#pragma unroll
          for (int i = 0; i < 4; ++i) {
            float v = *reinterpret_cast<const float *>(mine + (4 * g + i) * kPitch + (16 * o + row) * 4);
            if (kOdd) v = odd_of(v) ? 0.0f : v;
            acc[o] = __builtin_amdgcn_mfma_f32_16x16x4f32(v, s[0][i], acc[o], 0, 0, 0);
          }
        }
      }
    };
    if (!odd) {
      product(Plain{});
    } else {
      product(Odd{});
      const Sight sight = sight_of(a, place, j0);
#pragma unroll 1
      for (int k = 0; k < kKeys; ++k) {
        const bool seen = ((here >> k & 1) != 0) & sight.sees(k);  // (its weight may have underflowed to 0)
        float p = 0.0f;
#pragma unroll
        for (int kt = 0; kt < kTiles; ++kt)
#pragma unroll
          for (int i = 0; i < 4; ++i)
            if ((k >> 4) == kt && (k & 3) == i) p = s[kt][i];
        p = __shfl(p, row + 16 * ((k >> 2) & 3));
#pragma unroll
        for (int o = 0; o < kOut; ++o)
#pragma unroll
          for (int e = 0; e < 4; ++e) {
            const int d = 16 * o + 4 * g + e;
            const float v = Elem<T>::get(reinterpret_cast<const T *>(mine + k * kPitch) + d);
            if (seen && odd_of(v)) acc[o][e] += p * v;
          }
      }
    }
  }

  finish_rows<T, DT>(a, t, x, z, parts > 1 || PHASED, m, l, acc, mine, lds, ml);
}

template <typename T, int DT, bool FULL>
__global__ __launch_bounds__(256, DT > 128 ? 1 : DT > 96 ? 2 : 3) void attend_rows_kernel(AttendArgs a) {
  __shared__ __align__(16) uint8_t lds[4][RowsPart<T, DT>::kBytes];
  __shared__ float ml[4][16][2];
  uint8_t *const part[4] = {lds[0], lds[1], lds[2], lds[3]};
  attend_rows<T, DT, FULL, false>(a, blockIdx.x, blockIdx.y, part, ml);
}
// The same in phases, of tiles of 16 rows only (decode over short groups, float32).  Four sequences of 32 heads of
// 128 on 8 that share 2000 keys, with up to 300 of their own (bf16, 9.8 MB): 12.3 us, and the join 5.0; the chain of a
// workgroup's numbers, table, keys and end, as without groups, bounds it.  Float32 groups of any size are tiles of 16 rows
// here, each of which reads the prefix: 64 sequences on 32000 shared keys (256 rows a cache head, 16 tiles) 540 us, where bf16
// takes 103 and the float32 products' rate would be 222.
template <typename T, int DT, bool FULL>
__global__ __launch_bounds__(256, DT > 128 ? 1 : DT > 64 ? 2 : 3) void attend_rows_phases_kernel(AttendArgs a, PhaseArgs p) {
  __shared__ __align__(16) uint8_t lds[4][RowsPart<T, DT>::kBytes];
  __shared__ float ml[4][16][2];
  uint8_t *const part[4] = {lds[0], lds[1], lds[2], lds[3]};
  int x, z;
  take_set(a, p, blockIdx.x, &x, &z);
  attend_rows<T, DT, FULL, true>(a, x, z, part, ml);
  put_row_parts<16>(a, p, x, z);
}

// ------------------------------------------------------------------ tiles of 128 rows

// Prompts and chunks of bf16: four waves of 32 rows, blocks of 64 keys that the workgroup
// loads into LDS straight from memory, one block ahead.  Rows of K and V lie in LDS
// with their 16-byte pieces exchanged: the same piece of 16 rows of K is in 16 different places
// of a row's 256 bytes, and two pieces of 4 rows of V are in eight.  For V that is not enough:
// the counters show two cycles of bank conflicts for each read of V, whatever the width (heads of
// 128: 64 for each wave and block, a third of the LDS's cycles), as where a cycle serves 32 lanes and
// with them four pieces of 4 rows, of which two rows' coincide.
//
// Bound by issue: a chunk of 2048 tokens on 4096 earlier ones (32 heads of 128, 172 Gflop) takes
// 199 us in calls one after another, 863 TFLOP/s, where a large bf16 product reaches 1140 (221
// where each call is waited for, 217 to 245 under a tracer).  Without its loads it took 181
// us and without the exponentials 192 (scratch builds, when it took 206): what is left is the
// matrix and the vector instructions of a wave that do not overlap.  32 rows a wave fill the
// 32 x 32 x 16 instruction; 256 rows a workgroup were slower (one workgroup a compute unit
// leaves nothing to run at its barriers).
// Other widths, the same chunk, with 4096 dims in all but 80 and 96 (32 heads): 64 662 TFLOP/s, as
// many matrix cycles and 1.8 x the vector instructions (half the products for an exponential);
// 80 574 and 96 676, whose rows lie in LDS, and are read, as if of 128; 256 619, one workgroup a
// compute unit (131 KB of LDS), so nothing runs at its barriers.
constexpr int kTileRows = 128, kTileKeys = 64;

// 16 bytes of each lane into LDS at dst + OFF + 16 * lane, from src + OFF (dst the same for
// the whole wave).
template <int OFF> __device__ __forceinline__ void load_to_lds(const char *src, uint8_t *dst) {
  __builtin_amdgcn_global_load_lds((const __attribute__((address_space(1))) void *)src,
                                   (__attribute__((address_space(3))) void *)dst, 16, OFF, 0);
}
// The same from base + off, base the same for the whole wave.
template <int OFF> __device__ __forceinline__ void load_to_lds(const char *base, uint32_t off, uint8_t *dst) {
  __builtin_amdgcn_raw_ptr_buffer_load_lds(rows_rsrc(base), (__attribute__((address_space(3))) void *)dst, 16, (int)off, 0, OFF, 0);
}

// Every load of this wave has landed, and every wave is here.
__device__ __forceinline__ void stage_barrier() {
  asm volatile("" ::: "memory");
  __builtin_amdgcn_s_waitcnt(0);
  __builtin_amdgcn_s_barrier();
  asm volatile("" ::: "memory");
}

// Pages of a tile's keys: lane i holds the table's entry held + i, -1 where there is no such page.
struct HeldPages {
  int64_t first = -1;
  int page = -1;
};

// A wave's 32 rows.  The matrix products of block b + 1's scores are issued among the
// exponentials of block b, and the maximum of b + 1 among the products of P and V of b:
// neither the matrix cores nor the vector unit waits for the other.
template <int DT, bool FULL> struct TileWave {
  static constexpr int kRow = DT * 2, kChunks = kRow / 16, kOut = DT / 32, kSteps = DT / 16;
  static constexpr int kLine = kRow < 256 ? 256 / kRow : 1, kMask = (kRow / 32 < 8 ? kRow / 32 : 8) - 1;
  // where piece c of row r lies
  __device__ __forceinline__ static int k_place(int r, int c) { return c ^ ((r / kLine) & (2 * kMask + 1)); }
  __device__ __forceinline__ static int v_place(int r, int c) { return c ^ (2 * ((r / kLine) & kMask)); }

  bf16x8_t q[kSteps];
  f32x16_t acc[kOut];
  float m, l;  // of this lane's row: maximum (of the scores before the scale), sum
  float scale2;
  int64_t place, low, high;  // of this lane's row, of the wave's first and last row
  int dim;                   // (where not FULL, products of dims that a head has not are passed over)

  // Offsets of this lane's first pieces; the others' differ in fixed bits.  (Formed anew for
  // each block: kept, they would take the registers of a whole operand.)
  __device__ __forceinline__ static int k_base() {
    const int lane = threadIdx.x & 63, r = lane & 31;
    int at = r * kRow + k_place(r, lane >> 5) * 16;
    asm volatile("" : "+v"(at));
    return at;
  }
  __device__ __forceinline__ static int v_base() {
    const int lane = threadIdx.x & 63, r = 4 * (lane >> 5) + ((lane & 15) >> 2);
    int at = r * kRow + v_place(r, 2 * ((lane >> 4) & 1) + ((lane & 3) >> 1)) * 16 + (lane & 1) * 8;
    asm volatile("" : "+v"(at));
    return at;
  }
  // K's piece for product st of keys 32 x .. (piece 2 st + hf of row 32 x + lane % 32)
  __device__ __forceinline__ static bf16x8_t k_piece(const uint8_t *kt, int base, int x, int st) {
    return __builtin_bit_cast(bf16x8_t, *reinterpret_cast<const u32x4 *>(kt + (base ^ (32 * st)) + 32 * x * kRow));
  }
  // V^T's piece for keys 16 st .., dims 32 o ..: slot (hf, e) is key 16 st + 8 (e / 4) + 4 hf + e % 4
  template <bool SANE> __device__ __forceinline__ static bf16x8_t v_piece(const uint8_t *vt, int base, int st, int o) {
    i16x4_t v2[2];
#pragma unroll
    for (int y = 0; y < 2; ++y) {
      const int r = 16 * st + 8 * y;  // (and the row of v_base; 8 rows on, the pieces' exchange differs where a row is short)
      const int at = (base ^ (v_place(r, 4 * o) * 16)) + r * kRow;
      v2[y] = __builtin_amdgcn_ds_read_tr16_b64_v4i16((lds_i16x4 *)(vt + at));
      if (SANE) v2[y] = sane(v2[y]);
    }
    bf16x8_t v8;
    __builtin_memcpy(&v8, v2, 16);
    return v8;
  }

  // The places of this lane's row (r_in of the tile) and of the wave's first and last row.
  __device__ __forceinline__ void take_places(const AttendArgs &a, const RowTile &t, int w, int r_in) {
    place = t.place0 + (t.first + r_in) / a.group;
    low = t.place0 + (t.first + (32 * w < t.count ? 32 * w : t.count - 1)) / a.group;
    high = t.place0 + (t.first + (32 * w + 31 < t.count ? 32 * w + 31 : t.count - 1)) / a.group;
  }
  __device__ __forceinline__ void take_places(const RowPlaces<kTileRows> &p, int w, int col) {
    place = p.of(32 * w + col);
    range_of<32>(place, &low, &high);
  }
  __device__ __forceinline__ void take_rows(const AttendArgs &a, const RowTile &t, int kvh, int r_in) {
    dim = a.dim;
    scale2 = a.scale == 0.0f ? 1.0f : fabsf(a.scale) * kLog2e;
    // q with the scale's sign (zeros for a scale of 0), so that the largest product is the largest score
    const int r = t.first + r_in;
    const uint16_t *qr = (const uint16_t *)a.q + (t.start + r / a.group) * a.q_stride +
                         (int64_t)(kvh * a.group + r % a.group) * a.dim;
#pragma unroll
    for (int s = 0; s < kSteps; ++s) {
      const int c = 2 * s + ((threadIdx.x & 63) >> 5);
      u32x4 x = c * 8 < a.dim && a.scale != 0.0f ? *reinterpret_cast<const u32x4 *>(qr + c * 8) : u32x4{0, 0, 0, 0};
      if (a.scale < 0.0f) x ^= 0x80008000u;
      q[s] = __builtin_bit_cast(bf16x8_t, x);
    }
  }
  // This lane's results: the row's, or split z's part of it.
  __device__ __forceinline__ void put(const AttendArgs &a, const RowTile &t, int x, int row, int z, bool split) {
    float sum = l;
    sum += __shfl_xor(sum, 32);
    if (row >= t.count) return;
    const float top = m * scale2;
#pragma unroll
    for (int o = 0; o < kOut; ++o)
#pragma unroll
      for (int e = 0; e < 4; ++e) {
        const f32x4 v = {acc[o][4 * e], acc[o][4 * e + 1], acc[o][4 * e + 2], acc[o][4 * e + 3]};
        const int d = 32 * o + 8 * e + 4 * ((threadIdx.x & 63) >> 5);
        if (split) put_part(a, ((int64_t)x * a.splits + z) * kTileRows + row, d, v, top, sum);
        else put_row<uint16_t>(a, t, row, x % a.pool.n_kv, d, v, top, sum);
      }
  }

  __device__ __forceinline__ void clear() {
#pragma unroll
    for (int o = 0; o < kOut; ++o)
#pragma unroll
      for (int i = 0; i < 16; ++i) acc[o][i] = 0.0f;
    m = -INFINITY, l = 0.0f;
  }

  // Scores of the block in kt.
  __device__ __forceinline__ void scores(const uint8_t *kt, f32x16_t (&s)[2]) const {
    const int kx = k_base();
#pragma unroll
    for (int x = 0; x < 2; ++x)
#pragma unroll
      for (int i = 0; i < 16; ++i) s[x][i] = 0.0f;
#pragma unroll
    for (int st = 0; st < kSteps; ++st) {
      if (!FULL && 16 * st >= dim) break;
#pragma unroll
      for (int x = 0; x < 2; ++x) s[x] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(k_piece(kt, kx, x, st), q[st], s[x], 0, 0, 0);
    }
  }

  // -inf for the keys that a row does not see (`there`: the keys that some row of the tile sees).
  __device__ __forceinline__ bool whole(const AttendArgs &a, uint64_t there, int64_t j0) const {
    return there == ~0ull && j0 + kTileKeys - 1 <= low && (!a.window || high - j0 < a.window || j0 + kTileKeys <= a.sinks);
  }
  __device__ __forceinline__ void mask(const AttendArgs &a, uint64_t there, int64_t j0, f32x16_t (&s)[2]) const {
    const int hf = (threadIdx.x & 63) >> 5;
    const Sight sight = sight_of(a, place, j0 + 4 * hf);
    const uint64_t here = there >> (4 * hf);
#pragma unroll
    for (int x = 0; x < 2; ++x)
#pragma unroll
      for (int i = 0; i < 16; ++i) {
        const int k = 32 * x + 8 * (i >> 2) + (i & 3);
        s[x][i] = ((here >> k & 1) != 0) & sight.sees(k) ? s[x][i] : -INFINITY;
      }
  }
  // Whether a block's values hold infinities or NaN.
  __device__ __forceinline__ static bool odd_block(const uint8_t *vt) {
    bool odd = false;
    for (int c = threadIdx.x & 63; c < kTileKeys * kChunks; c += 64)
      odd |= odd_value<uint16_t>(*reinterpret_cast<const u32x4 *>(vt + c * 16));
    return __any(odd);
  }

  // The row's maximum moves to `top` (a lane's own), and the sums are scaled to it, only where a
  // weight would pass 2^8.  (Each row for itself, so that its result does not depend on the others';
  // a maximum that is NaN stays out, the weights are NaN then.)
  __device__ __forceinline__ void rescale(float top) {
    top = fmaxf(top, __shfl_xor(top, 32));
    const bool past = (top - m) * scale2 > 8.0f;
    if (__any(past)) {
      const float mn = past ? top : m, f = past ? exp2_fast((m - mn) * scale2) : 1.0f;
      m = mn;
      l *= f;
#pragma unroll
      for (int o = 0; o < kOut; ++o)
#pragma unroll
        for (int i = 0; i < 16; ++i) acc[o][i] *= f;
    }
  }

  // Weights of block b (scores s, in place) and, where NEXT, the scores of the next block.
  template <bool NEXT> __device__ __forceinline__ void weights(f32x16_t (&s)[2], const uint8_t *kt, f32x16_t (&sn)[2]) {
    const float base = m == -INFINITY ? 0.0f : -m * scale2;
    float sum[2] = {0.0f, 0.0f};
    constexpr int kSlots = 2 * kSteps, kPer = 32 / (kSlots < 32 ? kSlots : 32), kAhead = 4;
    bf16x8_t ring[kAhead];
    const int kx = k_base();
    if (NEXT) {
#pragma unroll
      for (int i = 0; i < kAhead; ++i) ring[i] = k_piece(kt, kx, i & 1, i >> 1);
#pragma unroll
      for (int x = 0; x < 2; ++x)
#pragma unroll
        for (int i = 0; i < 16; ++i) sn[x][i] = 0.0f;
    }
#pragma unroll
    for (int i = 0; i < kSlots; ++i) {
      if (NEXT && (FULL || 16 * (i >> 1) < dim)) {
        sn[i & 1] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(ring[i % kAhead], q[i >> 1], sn[i & 1], 0, 0, 0);
        if (i + kAhead < kSlots) ring[i % kAhead] = k_piece(kt, kx, (i + kAhead) & 1, (i + kAhead) >> 1);
      }
#pragma unroll
      for (int e = i * kPer; e < (i + 1) * kPer && e < 32; ++e) {
        s[e >> 4][e & 15] = exp2_fast(fmaf(s[e >> 4][e & 15], scale2, base));
        sum[e & 1] += s[e >> 4][e & 15];
      }
      if (NEXT) __builtin_amdgcn_sched_barrier(0);
    }
    l += sum[0] + sum[1];
  }

  // O^T += V^T P^T, and (NEXT) the largest of the next scores sn in *top (a lane's own).  P is rounded
  // to bf16 for the instruction, l is the sum of the float32 weights: the error of a result is 0.0023
  // of the norm where its own rounding makes 0.0016.  A second product with the rest of each weight,
  // as the tiles of 16 rows have, brings it down to that, and 2048 tokens on 4096 from 199 us to 262.
  // REST: with that second product.  In phases tiles have it, since the rows of a group can be single tokens', which have those
  // bits where each sequence is attended to by itself.  us without and with it: 64 tokens on 32000 shared keys 99.6, 103 (E4M3
  // 106, 114); groups with chunks 75, 89 (E4M3 88, 97); 64 chunks of 16 on 8000 shared keys 255, 313.  Only for groups that have
  // single tokens, chosen in the kernel: 120, 96 and 294, by the registers that both ways of it take.
  template <bool SANE, bool NEXT, bool REST>
  __device__ __forceinline__ void product(const f32x16_t (&s)[2], const uint8_t *vt, const f32x16_t (&sn)[2], float *top) {
    constexpr int kSlots = 4 * kOut, kAhead = 4;
    bf16x8_t ring[kAhead], p, rest;
    float t = sn[0][0];
    const int vx = v_base();
#pragma unroll
    for (int i = 0; i < kAhead; ++i) ring[i] = v_piece<SANE>(vt, vx, i / kOut, i % kOut);
#pragma unroll
    for (int i = 0; i < kSlots; ++i) {
      const int st = i / kOut, o = i % kOut;
      if (o == 0) {
#pragma unroll
        for (int e = 0; e < 8; ++e) {
          const float x = s[st >> 1][8 * (st & 1) + e], top = REST ? __uint_as_float(__float_as_uint(x) & 0xffff0000u) : x;
          p[e] = (__bf16)top;
          if (REST) rest[e] = (__bf16)fmaf(x, 1.0f + 0x1p-20f, -top);
        }
      }
      if (FULL || 32 * o < dim) {
        acc[o] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(ring[i % kAhead], p, acc[o], 0, 0, 0);
        if (REST) acc[o] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(ring[i % kAhead], rest, acc[o], 0, 0, 0);
      }
      if (i + kAhead < kSlots) ring[i % kAhead] = v_piece<SANE>(vt, vx, (i + kAhead) / kOut, (i + kAhead) % kOut);
#pragma unroll
      for (int e = i * 32 / kSlots; NEXT && e < (i + 1) * 32 / kSlots; ++e) t = fmaxf(t, sn[e >> 4][e & 15]);
    }
    if (NEXT) *top = t;
  }
  // ... and the infinities and NaN that it left out, where a row sees them (the block's keys from j0
  // on, of which `there` are seen by some row of the tile).
  __device__ __forceinline__ void add_odd(const AttendArgs &a, uint64_t there, int64_t j0, const f32x16_t (&s)[2],
                                          const uint8_t *vt) {
    const int lane = threadIdx.x & 63, hf = lane >> 5;
    const Sight sight = sight_of(a, place, j0);
#pragma unroll 1
    for (int k = 0; k < kTileKeys; ++k) {
      const bool seen = ((there >> k & 1) != 0) & sight.sees(k);  // (its weight may have underflowed to 0)
      float p = 0.0f;
#pragma unroll
      for (int x = 0; x < 2; ++x)
#pragma unroll
        for (int i = 0; i < 16; ++i)
          if ((k >> 5) == x && ((k >> 3) & 3) == i >> 2 && (k & 3) == (i & 3)) p = s[x][i];
      p = __shfl(p, (lane & 31) + 32 * ((k >> 2) & 1));
#pragma unroll
      for (int o = 0; o < kOut; ++o)
#pragma unroll
        for (int e = 0; e < 16; ++e) {
          const int d = 32 * o + 8 * (e >> 2) + 4 * hf + (e & 3);
          const uint16_t v = reinterpret_cast<const uint16_t *>(vt + k * kRow + v_place(k, d >> 3) * 16)[d & 7];
          if (seen && odd_bits(v)) acc[o][e] += p * bf16_to_f32(v);
        }
    }
  }
};

// x: tile and cache head; z: split; k0 .. v1: kTileKeys rows each, in arrays of their own, so that reads of one
// do not wait for loads into another.
template <int DT, bool FULL, bool PHASED>
__device__ __forceinline__ void attend_tile(const AttendArgs &a, int x, int z, uint8_t *k0, uint8_t *k1, uint8_t *v0, uint8_t *v1) {
  using Wave = TileWave<DT, FULL>;
  constexpr int kRow = Wave::kRow, kChunks = Wave::kChunks, kLoads = kTileKeys * kChunks / 256;

  const int kvh = x % a.pool.n_kv;
  const RowTile t = find_tile<kTileRows, PHASED>(a, x / a.pool.n_kv);
  if (t.seq < 0) return;
  RowPlaces<kTileRows> places;
  if constexpr (PHASED) places.find(a, t);
  KeyBlocks kb;
  if constexpr (PHASED) kb = key_blocks<kTileKeys>(a, t, places);
  else kb = key_blocks<kTileKeys>(a, t);
  const int parts = kb.n > a.per_split ? (kb.n + a.per_split - 1) / a.per_split : 1;
  if (z >= parts) {
    if constexpr (PHASED) put_nothing<kTileRows>(a, t, x, z);
    return;
  }
  const int b0 = z * a.per_split, b_end = kb.n < b0 + a.per_split ? kb.n : b0 + a.per_split;
  const int lane = threadIdx.x & 63, w = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), col = lane & 31, hf = lane >> 5;
  const int row = 32 * w + col, r_in = row < t.count ? row : t.count - 1;  // (rows past the last repeat it)

  Wave wave;
  if constexpr (PHASED) wave.take_places(places, w, col);
  else wave.take_places(a, t, w, r_in);
  wave.take_rows(a, t, kvh, r_in);
  const char *zeros = reinterpret_cast<const char *>(attend_zeros);
  const int64_t head_bytes = ((int64_t)kvh << a.pool.shift) * a.dim * 2;
  const int64_t page_bytes = ((int64_t)a.pool.n_kv << a.pool.shift) * a.dim * 2;
  const char *kp = (const char *)a.k + head_bytes, *vp = (const char *)a.v + head_bytes;
  const int row_bytes = a.dim * 2;
  const int32_t *table = PHASED ? t.pages : a.batch.table + t.seq * a.batch.max_pages;

  HeldPages held;
  // page of key `lane` of a block where some row of the tile sees it, else -1
  auto page_of = [&](int b) {
    if (b >= b_end) return -1;
    const int64_t j0 = block_key(kb, b, kTileKeys), p0 = j0 >> a.pool.shift, p1 = (j0 + kTileKeys - 1) >> a.pool.shift;
    if (held.first < 0 || p0 < held.first || p1 >= held.first + 64) {
      held.first = p0;
      const int p = p0 + lane < a.batch.max_pages ? table[p0 + lane] : -1;
      held.page = p >= 0 && p < a.pool.n_pages ? p : -1;
    }
    const int p = __shfl(held.page, (int)(((j0 + lane) >> a.pool.shift) - held.first));
    const bool inside = j0 + kTileKeys <= t.len && (!PHASED || j0 >= kb.lo) && j0 + kTileKeys - 1 <= kb.high &&
                        (!a.window || kb.low - j0 < a.window || j0 + kTileKeys <= a.sinks);
    return inside || any_sees<PHASED>(a, kb, t.len, j0 + lane) ? p : -1;
  };
  // wave w loads rows 16 w .. 16 w + 15 of a block of K or V; where all of them are there, in
  // one page and whole, from one address and fixed offsets
  auto issue = [&](int b, int page, uint64_t there, const char *pool, uint8_t *to, auto place) {
    const int j0 = (int)(block_key(kb, b, kTileKeys) & (a.pool.page - 1));
    to += w * kLoads * 1024;
    constexpr int kStep = 64 / kChunks;  // rows of a load
    const int r0 = lane / kChunks, x = lane % kChunks;
    if (a.pool.shift >= 4 && (there >> (16 * w) & 0xffffu) == 0xffffu) {
      const int64_t p = __builtin_amdgcn_readlane(page, 16 * w);
      const char *from = pool + p * page_bytes + ((j0 + 16 * w) & (a.pool.page - 1)) * row_bytes;
      uint32_t off = r0 * kRow + place(r0, x) * 16;  // (a load's rows begin at multiples of kStep: their exchange is in other bits)
      asm volatile("" : "+v"(off));
      // load i; of a head of fewer dims the rows are closer, and pieces past its end read zeros
      auto load = [&](auto i_) {
        constexpr int i = decltype(i_)::value;
        if constexpr (FULL) {
          load_to_lds<i % 4 * 1024>(from + i / 4 * 4096, off ^ (place(i * kStep, 0) * 16), to + i / 4 * 4096);
        } else {
          const int c = place(i * kStep + r0, x);
          load_to_lds<0>(from, c * 8 < a.dim ? (uint32_t)((i * kStep + r0) * row_bytes + c * 16) : kNoRow, to + i * 1024);
        }
      };
      load(Const<0>{}), load(Const<1>{});
      if constexpr (kLoads > 2) load(Const<2>{}), load(Const<3>{});
      if constexpr (kLoads > 4) load(Const<4>{}), load(Const<5>{}), load(Const<6>{}), load(Const<7>{});
      return;
    }
#pragma unroll 1
    for (int i = 0; i < kLoads; ++i) {
      const int r = i * kStep + r0, c = place(r, x), p = __shfl(page, 16 * w + r);
      const int64_t off = p * page_bytes + ((j0 + 16 * w + r) & (a.pool.page - 1)) * row_bytes;
      load_to_lds<0>(p >= 0 && c * 8 < a.dim ? pool + off + c * 16 : zeros, to + i * 1024);
    }
  };
  auto issue_k = [&](int b, int page, uint64_t there, uint8_t *to) { issue(b, page, there, kp, to, Wave::k_place); };
  auto issue_v = [&](int b, int page, uint64_t there, uint8_t *to) { issue(b, page, there, vp, to, Wave::v_place); };

  // The tile's blocks.  K of block b is in buffer (b - b0) % 2, V likewise.  At the barrier of
  // step b every wave's loads (K of b + 1, V of b) have landed, and K of b and V of
  // b - 1 have been read by all.  Returns whether the blocks have to be taken again.
  auto run = [&](auto kind) {
    constexpr bool kOdd = decltype(kind)::kOdd;
    wave.clear();
    bool again = false;
    if (b0 >= b_end) return again;
    f32x16_t sa[2], sb[2];
    held.first = -1;
    int page = page_of(b0), next = page_of(b0 + 1);
    uint64_t there = __ballot(page >= 0), there_next = __ballot(next >= 0), here = there;  // (here: of the block at hand)
    issue_k(b0, page, there, k0);
    issue_v(b0, page, there, v0);
    if (b0 + 1 < b_end) issue_k(b0 + 1, next, there_next, k1);
    stage_barrier();
    wave.scores(k0, sa);
    bool some = !wave.whole(a, there, block_key(kb, b0, kTileKeys));  // rows disagree on a key of the block at hand
    if (some) wave.mask(a, there, block_key(kb, b0, kTileKeys), sa);
    float top = sa[0][0];
#pragma unroll
    for (int i = 1; i < 32; ++i) top = fmaxf(top, sa[i >> 4][i & 15]);
    wave.rescale(top);
    // block b, of scores s, whose K was in kt, and the scores sn of block b + 1
    auto step = [&](int b, f32x16_t (&s)[2], f32x16_t (&sn)[2], uint8_t *kt, uint8_t *kn, uint8_t *vt, uint8_t *vn) {
      stage_barrier();
      page = page_of(b + 2);
      there = __ballot(page >= 0);
      if (b + 2 < b_end) issue_k(b + 2, page, there, kt);
      issue_v(b + 1, next, there_next, vn);
      const bool odd = some && Wave::odd_block(vt);
      wave.template weights<true>(s, kn, sn);
      const int64_t j1 = block_key(kb, b + 1, kTileKeys);
      some = !wave.whole(a, there_next, j1);
      if (some) wave.mask(a, there_next, j1, sn);
      if (kOdd && odd) {
        wave.template product<true, true, PHASED>(s, vt, sn, &top);
        wave.add_odd(a, here, block_key(kb, b, kTileKeys), s, vt);
      } else {
        wave.template product<false, true, PHASED>(s, vt, sn, &top);
        again |= odd;
      }
      wave.rescale(top);
      next = page, here = there_next, there_next = there;
    };
    auto last = [&](int b, f32x16_t (&s)[2], uint8_t *vt) {
      stage_barrier();
      const bool odd = some && Wave::odd_block(vt);
      wave.template weights<false>(s, vt, s);
      if (kOdd && odd) {
        wave.template product<true, false, PHASED>(s, vt, s, &top);
        wave.add_odd(a, here, block_key(kb, b, kTileKeys), s, vt);
      } else {
        wave.template product<false, false, PHASED>(s, vt, s, &top);
        again |= odd;
      }
    };
    int b = b0;
    for (; b + 2 < b_end; b += 2) {
      step(b, sa, sb, k0, k1, v0, v1);
      step(b + 1, sb, sa, k1, k0, v1, v0);
    }
    if (b + 1 < b_end) {
      step(b, sa, sb, k0, k1, v0, v1);
      last(b + 1, sb, v1);
    } else {
      last(b, sa, v0);
    }
    return again;
  };
  if (__syncthreads_or(run(Plain{}))) run(Odd{});

  wave.put(a, t, x, row, z, parts > 1 || PHASED);
}

template <int DT, bool FULL>
__global__ __launch_bounds__(256, DT > 128 ? 1 : 2) void attend_tile_kernel(AttendArgs a) {
  constexpr int kBytes = kTileKeys * TileWave<DT, FULL>::kRow;
  __shared__ __align__(16) uint8_t k0[kBytes], k1[kBytes], v0[kBytes], v1[kBytes];
  attend_tile<DT, FULL, false>(a, blockIdx.x, blockIdx.y, k0, k1, v0, v1);
}
// In phases, of tiles of 16 rows and of 128.  The rows of all sequences of a group share a tile, so that the
// prefix is read once for 128 of them: 64 sequences of 32 heads of 128 on 8 with 32000 keys in common and 100 to 2000 of
// their own (bf16) have 299 MB to read instead of 8.7 GB (the 256 rows of a cache head are two tiles), 103 us with the join (traced
// 9.9), where attention sequence after sequence takes 1460.  Both phases are in one launch, since the prefix's tiles are bound by products and the sequences' own by
// memory.  A workgroup's registers and LDS are those of the larger tile for both, so two of them a compute unit are all
// the loads that decode has in flight here; that, and parts of unlike lengths (about 5 us of each before its first
// product), is what is left above the 62 us of the bytes.  The compiler spills 78 of a wave's registers at 128 dims, 120 at
// 256 (attend_tile_kernel 52 and 115).
template <int DT, bool FULL>
__global__ __launch_bounds__(256, DT > 128 ? 1 : 2) void attend_phases_kernel(AttendArgs a, PhaseArgs p) {
  constexpr int kBytes = kTileKeys * TileWave<DT, FULL>::kRow;
  static_assert(kBytes >= RowsPart<uint16_t, DT>::kBytes, "");
  __shared__ __align__(16) uint8_t k0[kBytes], k1[kBytes], v0[kBytes], v1[kBytes];
  __shared__ float ml[4][16][2];
  int x, z;
  if (take_set(a, p, blockIdx.x, &x, &z) & 1) {
    attend_tile<DT, FULL, true>(a, x, z, k0, k1, v0, v1);
    put_row_parts<kTileRows>(a, p, x, z);
  } else {
    uint8_t *const part[4] = {k0, k1, v0, v1};
    attend_rows<uint16_t, DT, FULL, true>(a, x, z, part, ml);
    put_row_parts<16>(a, p, x, z);
  }
}

// ------------------------------------------------------------------ join

// Joins the parts of a tile's rows where it was split (into blocks of KEYS keys): W waves per row, each part of a row
// held by `lanes` lanes, so that a wave adds 64 / lanes parts at a time and the W waves'
// loads are all in flight.  The order of a row's sum depends on the batch's bounds alone.
// Latency: two dependent loads and the launch, 5.7 us for 64 sequences in 4 parts each, 8.2 us
// for one sequence in 61.
template <typename T, int R, int W, int KEYS>
__global__ __launch_bounds__(256) void attend_join_kernel(AttendArgs a) {
  __shared__ float ls[W > 1 ? W : 1];
  __shared__ f32x4 os[W > 1 ? W : 1][64];
  const RowTile t = find_tile<R>(a, blockIdx.x / a.pool.n_kv);
  const int wave = threadIdx.x >> 6, r = blockIdx.y * (4 / W) + wave / W, w = wave % W, lane = threadIdx.x & 63;
  if (t.seq < 0 || (W > 1 ? (int)blockIdx.y : r) >= t.count) return;  // (W > 1: a row a workgroup)
  const KeyBlocks kb = key_blocks<KEYS>(a, t);
  const int parts = kb.n > a.per_split ? (kb.n + a.per_split - 1) / a.per_split : 1;
  if (parts == 1) return;
  const int64_t at = (int64_t)blockIdx.x * a.splits * R + r;  // part z's row is at + z * R
  float top = -INFINITY;
  for (int z = lane; z < parts; z += 64) top = fmaxf(top, a.part_ml[(at + (int64_t)z * R) * 2]);
#pragma unroll
  for (int d = 32; d; d >>= 1) top = fmaxf(top, __shfl_xor(top, d));
  const float at0 = top == -INFINITY ? 0.0f : top;
  const int lanes = a.dim <= 64 ? 16 : a.dim <= 128 ? 32 : 64, sub = lane / lanes, per = 64 / lanes;
  const int d = lane % lanes * 4, dd = d < a.dim ? d : 0;
  float l = 0.0f;
  f32x4 o = f32x4{0, 0, 0, 0};
#pragma unroll 4
  for (int z0 = w * per; z0 < parts; z0 += W * per) {
    const int z = z0 + sub < parts ? z0 + sub : parts - 1;
    const float *ml = a.part_ml + (at + (int64_t)z * R) * 2;
    const float lz = z0 + sub < parts ? ml[1] : 0.0f, f = exp2_fast(ml[0] - at0);
    const f32x4 x = *reinterpret_cast<const f32x4 *>(a.part + (at + (int64_t)z * R) * a.dim + dd);
    // (a part that saw nothing has 0; one whose scores are NaN has no maximum, but NaN here)
    if (lz != 0.0f) l += lz * f, o += x * f;
  }
  for (int m = lanes; m < 64; m <<= 1) {
    l += __shfl_xor(l, m);
#pragma unroll
    for (int i = 0; i < 4; ++i) o[i] += __shfl_xor(o[i], m);
  }
  if constexpr (W > 1) {
    os[w][lane] = o;
    if (lane == 0) ls[w] = l;
    __syncthreads();
    if (w) return;
    o = f32x4{0, 0, 0, 0}, l = 0.0f;
#pragma unroll
    for (int i = 0; i < W; ++i) o += os[i][lane], l += ls[i];
  }
  if (lane < lanes && d < a.dim) put_row<T>(a, t, r, blockIdx.x % a.pool.n_kv, d, o, top, l);
}

// The same where sequences share prefixes: W waves a row, whose parts are where the launch before wrote that
// they are (put_row_parts).  Every split has left a part, an empty one too, whose sums are loaded as well.  What is read there is used only
// within its set: a row that no tile was launched for holds anything.
// Latency: three dependent loads, and the parts' bytes: 5.0 us for 128 rows of up to 11 parts, 9.9 for 2048 of up to 36,
// 13.4 for 12000 of up to 20 (of which a wave a row where rows are many: kJoinRows).
template <typename T, int W>
__global__ __launch_bounds__(256) void attend_join_phases_kernel(AttendArgs a, PhaseArgs p) {
  __shared__ float ls[W > 1 ? W : 1];
  __shared__ f32x4 os[W > 1 ? W : 1][64];
  const int wave = threadIdx.x >> 6, w = wave % W, lane = threadIdx.x & 63;
  const int64_t row = (int64_t)blockIdx.x * (4 / W) + wave / W, tok = row / a.n_q;
  bool live = tok < a.batch.n_tokens;
  if (W == 1 && !live) return;
  const RowParts at = p.parts[live ? row : 0];
  // a row of some sequence?
  bool in = false;
  auto within = [&](int s) {
    const SeqView v = seq_view(a.batch, a.pool, s);
    return tok >= v.start && tok < v.start + v.n_new;
  };
  if (a.batch.n_seqs <= 256) {  // (at once, or one after another's half)
    for (int s = lane; s < a.batch.n_seqs; s += 64) in |= within(s);
  } else {
    int s;
    token_place(a.batch, tok, &s);
    in = within(s);
  }
  live = live && __any(in);
  const int set = at.own >= p.set[kOwnLarge].row0 ? kOwnLarge : kOwnSmall;
  const int pre = at.shared >= p.set[kSharedLarge].row0 && p.set[kSharedLarge].tiles ? kSharedLarge : kSharedSmall;
  int n[2], tall[2], first[2] = {at.own, at.shared};
#pragma unroll
  for (int x = 0; x < 2; ++x) {
    const PhaseSet &s = p.set[x ? pre : set];
    tall[x] = (x ? pre : set) & 1 ? kTileRows : 16;
    n[x] = s.splits;
    if (!s.tiles || first[x] < s.row0 || first[x] - s.row0 > s.rows - 1 - (s.splits - 1) * tall[x]) n[x] = 0, first[x] = 0;
  }
  const int all = n[0] + n[1];
  auto part_row = [&](int z) { return (int64_t)(z < n[0] ? first[0] + z * tall[0] : first[1] + (z - n[0]) * tall[1]); };
  // the largest maximum; each lane has a part's of every 64
  float top = -INFINITY;
  for (int z = lane; z < all; z += 64) top = fmaxf(top, p.part_ml[part_row(z) * 2]);
#pragma unroll
  for (int d = 32; d; d >>= 1) top = fmaxf(top, __shfl_xor(top, d));
  const float at0 = top == -INFINITY ? 0.0f : top;
  const int lanes = a.dim <= 64 ? 16 : a.dim <= 128 ? 32 : 64, sub = lane / lanes, per = 64 / lanes;
  const int d = lane % lanes * 4, dd = d < a.dim ? d : 0;
  float l = 0.0f;
  f32x4 o = f32x4{0, 0, 0, 0};
#pragma unroll 8
  for (int z0 = w * per; z0 < all; z0 += W * per) {
    const int z = z0 + sub;
    const int64_t r = part_row(z < all ? z : z0);
    const float *ml = p.part_ml + r * 2;
    const float lz = z < all ? ml[1] : 0.0f, f = exp2_fast(ml[0] - at0);
    // (an empty part holds no sums)
    const f32x4 v = *reinterpret_cast<const f32x4 *>(p.part + r * a.dim + dd);
    if (lz != 0.0f) l += lz * f, o += v * f;
  }
  for (int m = lanes; m < 64; m <<= 1) {
    l += __shfl_xor(l, m);
#pragma unroll
    for (int i = 0; i < 4; ++i) o[i] += __shfl_xor(o[i], m);
  }
  if constexpr (W > 1) {
    os[w][lane] = o;
    if (lane == 0) ls[w] = l;
    __syncthreads();
    if (w) return;
    o = f32x4{0, 0, 0, 0}, l = 0.0f;
#pragma unroll
    for (int i = 0; i < W; ++i) o += os[i][lane], l += ls[i];
  }
  if (!live || !n[0] || lane >= lanes || d >= a.dim) return;
  RowTile t;  // (the row as one of a tile of its own)
  t.start = tok, t.first = 0;
  const int h = (int)(row - tok * a.n_q);
  put_row<T>(a, t, h % a.group, h / a.group, d, o, top, l);
}

}  // namespace sats

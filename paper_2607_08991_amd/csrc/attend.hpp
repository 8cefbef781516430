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
#pragma once

#include "paged.hpp"

namespace sats {

typedef __bf16 bf16x8_t __attribute__((ext_vector_type(8)));
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
};

__device__ u32x4 attend_zeros[64];  // a row of zeros
constexpr uint32_t kNoRow = 0x80000000u;  // an offset past every buffer: the load returns zeros
__device__ __forceinline__ __amdgpu_buffer_rsrc_t rows_rsrc(const char *base) {
  return __builtin_amdgcn_make_buffer_rsrc(const_cast<char *>(base), (short)0, 0x7fffffff, 0x00020000);
}

constexpr float kLog2e = 1.44269504088896340736f, kLn2 = 0.69314718055994530942f;
__device__ __forceinline__ float exp2_fast(float x) { return __builtin_amdgcn_exp2f(x); }

// A tile of rows: rows first .. first + count - 1 of (token, group) pairs of a sequence.
struct RowTile {
  int seq;          // -1: none
  int first, count;
  int64_t start, place0, len;  // sequence's first token; place of its first new token; length
};

__device__ __forceinline__ bool takes(const AttendArgs &a, int rows) { return rows <= 16 ? a.small : a.large; }

// Tile `t` of the batch (rows in tiles of R; a sequence's last rows, which see most keys, first).
template <int R>
__device__ __forceinline__ RowTile find_tile(const AttendArgs &a, int t) {
  RowTile o;
  o.seq = -1;
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
  return o;
}

// The blocks of B keys that a tile's rows see.
struct KeyBlocks {
  int64_t low, high;  // places of the first and last row
  int n_sink;         // blocks of sinks before the window
  int64_t first;      // first block of the window
  int n;              // all
};
template <int B> __device__ __forceinline__ KeyBlocks key_blocks(const AttendArgs &a, const RowTile &t) {
  KeyBlocks k;
  k.low = t.place0 + t.first / a.group;
  k.high = t.place0 + (t.first + t.count - 1) / a.group;
  const int64_t end = k.high + 1 < t.len ? k.high + 1 : t.len;
  int64_t from = a.window ? k.low - a.window + 1 : 0;
  from = from < 0 ? 0 : from;
  k.first = from / B;
  const int64_t last = end > 0 ? (end + B - 1) / B : 0, sink = a.window ? (a.sinks + B - 1) / B : 0;
  k.n_sink = (int)(sink < k.first ? sink : k.first);
  if (k.n_sink > last) k.n_sink = (int)last;
  k.n = k.n_sink + (int)(last > k.first ? last - k.first : 0);
  return k;
}
__device__ __forceinline__ int64_t block_key(const KeyBlocks &k, int b, int keys) {
  return (b < k.n_sink ? b : k.first + (b - k.n_sink)) * keys;
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
__device__ __forceinline__ bool any_sees(const AttendArgs &a, const KeyBlocks &k, int64_t len, int64_t j) {
  return j < len && j <= k.high && (!a.window || k.low - j < a.window || j < a.sinks);
}

// Page of key j where some row sees it, else -1.
__device__ __forceinline__ int key_page(const AttendArgs &a, const RowTile &t, const KeyBlocks &k, int64_t j) {
  if (!any_sees(a, k, t.len, j)) return -1;
  const int p = a.batch.table[t.seq * a.batch.max_pages + (j >> a.pool.shift)];
  return p >= 0 && p < a.pool.n_pages ? p : -1;
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
// bf16, 711 MB) take 151 us with the join, 4.7 TB/s (counters: 712 MB fetched, no bank
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

// FULL: heads of DT dims.  Else every load leaves out the dims that a head has not (they are the
// next slot's, or lie behind the cache), and up to DT = 128 the products do too.  Of 256 they
// multiply zeros there: leaving them out spills 989 registers (bf16; 683 float32), all of them none.
template <typename T, int DT, bool FULL>
__global__ __launch_bounds__(256, DT > 128 ? 1 : DT > 96 ? 2 : 3) void attend_rows_kernel(AttendArgs a) {
  constexpr int kKeys = RowsOf<T>::kKeys, kVec = Elem<T>::kVec, kRow = DT * (int)sizeof(T), kChunks = kRow / 16;
  constexpr bool kSkip = !FULL && DT <= 128;
  constexpr int kTiles = kKeys / 16, kSteps = kChunks / 4, kLoads = kKeys * kChunks / 64, kOut = DT / 16;
  // V's rows lie a little apart, so that the rows that are read together (bf16: 32 bytes of 8
  // rows; float32: 64 bytes of 4 rows, 4 apart) are in different banks
  constexpr int kPitch = kRow + (sizeof(T) == 2 ? 32 : 16);
  constexpr int kPart = kKeys * kPitch > 16 * DT * 4 ? kKeys * kPitch : 16 * DT * 4;  // (the waves' sums are joined there)
  __shared__ __align__(16) uint8_t lds[4][kPart];
  __shared__ float ml[4][16][2];

  const int kvh = blockIdx.x % a.pool.n_kv, z = blockIdx.y;
  const RowTile t = find_tile<16>(a, blockIdx.x / a.pool.n_kv);
  if (t.seq < 0) return;
  const KeyBlocks kb = key_blocks<kKeys>(a, t);
  const int parts = kb.n > a.per_split ? (kb.n + a.per_split - 1) / a.per_split : 1;
  if (z >= parts) return;
  const int b_end = kb.n < (z + 1) * a.per_split ? kb.n : (z + 1) * a.per_split;
  const int lane = threadIdx.x & 63, w = threadIdx.x >> 6, row = lane & 15, g = lane >> 4;
  const int64_t place = t.place0 + (t.first + (row < t.count ? row : t.count - 1)) / a.group;
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
  auto page_of = [&](int b) {  // of key lane % kKeys of a block
    return b < b_end ? key_page(a, t, kb, block_key(kb, b, kKeys) + (lane & (kKeys - 1))) : -1;
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
  uint8_t *mine = lds[w];

  int b = z * a.per_split + w;
  int page = page_of(b);
  uint32_t there = (uint32_t)__ballot(page >= 0);
  if (b < b_end) load(b, page, there);
  int page_next = page_of(b + 4);
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
    page = page_next;
    there = (uint32_t)__ballot(page >= 0);
    if (b + 4 < b_end) {
      load(b + 4, page, there);
      page_next = page_of(b + 8);
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
  // each wave's sums, scaled to the common maximum: [wave][dim / 4][row][4]
  float *sums = reinterpret_cast<float *>(lds);
#pragma unroll
  for (int o = 0; o < kOut; ++o)
    *reinterpret_cast<f32x4 *>(sums + ((w * (DT / 4) + 4 * o + g) * 16 + row) * 4) = acc[o] * fw[w];
  __syncthreads();
  const bool split = parts > 1;
  for (int i = threadIdx.x >> 4; i < DT / 4; i += 16) {
    f32x4 o = f32x4{0, 0, 0, 0};
#pragma unroll
    for (int x = 0; x < 4; ++x) o += *reinterpret_cast<const f32x4 *>(sums + ((x * (DT / 4) + i) * 16 + row) * 4);
    if (row >= t.count) continue;
    if (split) put_part(a, ((int64_t)blockIdx.x * a.splits + z) * 16 + row, 4 * i, o, top, total);
    else put_row<T>(a, t, row, kvh, 4 * i, o, top, total);
  }
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
  template <bool SANE, bool NEXT>
  __device__ __forceinline__ void product(const f32x16_t (&s)[2], const uint8_t *vt, const f32x16_t (&sn)[2], float *top) {
    constexpr int kSlots = 4 * kOut, kAhead = 4;
    bf16x8_t ring[kAhead], p;
    float t = sn[0][0];
    const int vx = v_base();
#pragma unroll
    for (int i = 0; i < kAhead; ++i) ring[i] = v_piece<SANE>(vt, vx, i / kOut, i % kOut);
#pragma unroll
    for (int i = 0; i < kSlots; ++i) {
      const int st = i / kOut, o = i % kOut;
      if (o == 0) {
#pragma unroll
        for (int e = 0; e < 8; ++e) p[e] = (__bf16)s[st >> 1][8 * (st & 1) + e];
      }
      if (FULL || 32 * o < dim) acc[o] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(ring[i % kAhead], p, acc[o], 0, 0, 0);
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

template <int DT, bool FULL>
__global__ __launch_bounds__(256, DT > 128 ? 1 : 2) void attend_tile_kernel(AttendArgs a) {
  using Wave = TileWave<DT, FULL>;
  constexpr int kRow = Wave::kRow, kChunks = Wave::kChunks, kLoads = kTileKeys * kChunks / 256;
  // (arrays of their own, so that reads of one do not wait for loads into another)
  __shared__ __align__(16) uint8_t k0[kTileKeys * kRow], k1[kTileKeys * kRow], v0[kTileKeys * kRow], v1[kTileKeys * kRow];

  const int kvh = blockIdx.x % a.pool.n_kv, z = blockIdx.y;
  const RowTile t = find_tile<kTileRows>(a, blockIdx.x / a.pool.n_kv);
  if (t.seq < 0) return;
  const KeyBlocks kb = key_blocks<kTileKeys>(a, t);
  const int parts = kb.n > a.per_split ? (kb.n + a.per_split - 1) / a.per_split : 1;
  if (z >= parts) return;
  const int b0 = z * a.per_split, b_end = kb.n < b0 + a.per_split ? kb.n : b0 + a.per_split;
  const int lane = threadIdx.x & 63, w = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), col = lane & 31, hf = lane >> 5;
  const int row = 32 * w + col, r_in = row < t.count ? row : t.count - 1;  // (rows past the last repeat it)

  Wave wave;
  wave.dim = a.dim;
  wave.place = t.place0 + (t.first + r_in) / a.group;
  wave.low = t.place0 + (t.first + (32 * w < t.count ? 32 * w : t.count - 1)) / a.group;
  wave.high = t.place0 + (t.first + (32 * w + 31 < t.count ? 32 * w + 31 : t.count - 1)) / a.group;
  wave.scale2 = a.scale == 0.0f ? 1.0f : fabsf(a.scale) * kLog2e;
  {  // q with the scale's sign (zeros for a scale of 0), so that the largest product is the largest score
    const int r = t.first + r_in;
    const uint16_t *q = (const uint16_t *)a.q + (t.start + r / a.group) * a.q_stride +
                        (int64_t)(kvh * a.group + r % a.group) * a.dim;
#pragma unroll
    for (int s = 0; s < Wave::kSteps; ++s) {
      const int c = 2 * s + hf;
      u32x4 x = c * 8 < a.dim && a.scale != 0.0f ? *reinterpret_cast<const u32x4 *>(q + c * 8) : u32x4{0, 0, 0, 0};
      if (a.scale < 0.0f) x ^= 0x80008000u;
      wave.q[s] = __builtin_bit_cast(bf16x8_t, x);
    }
  }
  const char *zeros = reinterpret_cast<const char *>(attend_zeros);
  const int64_t head_bytes = ((int64_t)kvh << a.pool.shift) * a.dim * 2;
  const int64_t page_bytes = ((int64_t)a.pool.n_kv << a.pool.shift) * a.dim * 2;
  const char *kp = (const char *)a.k + head_bytes, *vp = (const char *)a.v + head_bytes;
  const int row_bytes = a.dim * 2;
  const int32_t *table = a.batch.table + t.seq * a.batch.max_pages;

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
    const bool inside = j0 + kTileKeys <= t.len && j0 + kTileKeys - 1 <= kb.high &&
                        (!a.window || kb.low - j0 < a.window || j0 + kTileKeys <= a.sinks);
    return inside || any_sees(a, kb, t.len, j0 + lane) ? p : -1;
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
        wave.template product<true, true>(s, vt, sn, &top);
        wave.add_odd(a, here, block_key(kb, b, kTileKeys), s, vt);
      } else {
        wave.template product<false, true>(s, vt, sn, &top);
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
        wave.template product<true, false>(s, vt, s, &top);
        wave.add_odd(a, here, block_key(kb, b, kTileKeys), s, vt);
      } else {
        wave.template product<false, false>(s, vt, s, &top);
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

  float l = wave.l;
  l += __shfl_xor(l, 32);
  if (row >= t.count) return;
  const float m = wave.m * wave.scale2;
#pragma unroll
  for (int o = 0; o < Wave::kOut; ++o)
#pragma unroll
    for (int e = 0; e < 4; ++e) {
      const f32x4 v = {wave.acc[o][4 * e], wave.acc[o][4 * e + 1], wave.acc[o][4 * e + 2], wave.acc[o][4 * e + 3]};
      const int d = 32 * o + 8 * e + 4 * hf;
      if (parts > 1) put_part(a, ((int64_t)blockIdx.x * a.splits + z) * kTileRows + row, d, v, m, l);
      else put_row<uint16_t>(a, t, row, kvh, d, v, m, l);
    }
}

// ------------------------------------------------------------------ join

// Joins the parts of a tile's rows where it was split: W waves per row, each part of a row
// held by `lanes` lanes, so that a wave adds 64 / lanes parts at a time and the W waves'
// loads are all in flight.  The order of a row's sum depends on the batch's bounds alone.
// Latency: two dependent loads and the launch, 5.7 us for 64 sequences in 4 parts each, 8.2 us
// for one sequence in 61.
template <typename T, int R, int W>
__global__ __launch_bounds__(256) void attend_join_kernel(AttendArgs a) {
  constexpr int kKeys = R == 16 ? RowsOf<T>::kKeys : kTileKeys;
  __shared__ float ls[W > 1 ? W : 1];
  __shared__ f32x4 os[W > 1 ? W : 1][64];
  const RowTile t = find_tile<R>(a, blockIdx.x / a.pool.n_kv);
  const int wave = threadIdx.x >> 6, r = blockIdx.y * (4 / W) + wave / W, w = wave % W, lane = threadIdx.x & 63;
  if (t.seq < 0 || (W > 1 ? (int)blockIdx.y : r) >= t.count) return;  // (W > 1: a row a workgroup)
  const KeyBlocks kb = key_blocks<kKeys>(a, t);
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

}  // namespace sats

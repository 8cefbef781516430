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
  int tiles;          // upper bound of the row tiles of the batch
  int splits;         // workgroups a tile's blocks are split over, at most
  int per_split;      // key blocks of a split
  int small, large;   // which sequences the launch takes: at most 16 rows a head, more
  float *part;        // [tiles * n_kv][splits][rows of a tile][dim]
  float *part_ml;     // [tiles * n_kv][splits][rows of a tile][2]
};

__device__ u32x4 attend_zeros[64];  // a row of zeros

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

struct Plain { static constexpr bool kOdd = false; };
struct Odd { static constexpr bool kOdd = true; };

// ------------------------------------------------------------------ tiles of 16 rows

// Decode and short chunks (and float32 of any length): each of the four waves takes
// every fourth block of a tile's keys with a softmax of its own, joined in LDS at the end.
// K goes from memory straight to the lanes that multiply it; V through LDS, a wave's
// own part, for the transposing reads.  The next block's loads are in flight while
// one is worked on.
template <typename T> struct RowsOf {
  static constexpr int kKeys = sizeof(T) == 2 ? 32 : 16;  // keys of a block
};

template <typename T, int DT>
__global__ __launch_bounds__(256, DT > 128 ? 1 : 2) void attend_rows_kernel(AttendArgs a) {
  constexpr int kKeys = RowsOf<T>::kKeys, kVec = Elem<T>::kVec, kRow = DT * (int)sizeof(T), kChunks = kRow / 16;
  constexpr int kTiles = kKeys / 16, kSteps = kChunks / 4, kLoads = kKeys * kChunks / 64, kOut = DT / 16;
  // 16-byte pieces of V's rows are exchanged so that the rows of a transposing read
  // (bf16: 8 rows of 32 bytes; float32: 4 rows, 4 apart, of 64) lie in different banks
  constexpr int kLine = kRow < 256 ? 256 / kRow : 1, kMask = (kRow / 32 < 8 ? kRow / 32 : 8) - 1;
  auto place_of = [](int r, int c) {
    if constexpr (sizeof(T) == 2) return c ^ (2 * ((r / kLine) & kMask));
    else return c ^ (4 * ((r >> 2) & 3));
  };
  __shared__ __align__(16) uint8_t lds[4][kKeys * kRow];
  __shared__ float ml[4][16][2];
  static_assert(sizeof lds >= 4 * 16 * DT * 4, "the waves' sums are joined there");

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
  auto load = [&](int b, int page) {
    const int j0 = (int)(block_key(kb, b, kKeys) & (a.pool.page - 1));  // (blocks and pages are powers of two)
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
  if (b < b_end) load(b, page);
  int page_next = page_of(b + 4);
  for (; b < b_end; b += 4) {
    const int64_t j0 = block_key(kb, b, kKeys);
    const uint64_t there = __ballot(page >= 0);
    const bool whole = (uint32_t)there == (uint32_t)((1ull << kKeys) - 1) && j0 + kKeys - 1 <= kb.low &&
                       (!a.window || kb.high - j0 < a.window || j0 + kKeys <= a.sinks);
    // scores: lane (row, keys 16 kt + 4 g + i)
    f32x4 s[kTiles];
#pragma unroll
    for (int kt = 0; kt < kTiles; ++kt) {
      s[kt] = f32x4{0, 0, 0, 0};
#pragma unroll
      for (int st = 0; st < kSteps; ++st) {
        if constexpr (sizeof(T) == 2) {
          s[kt] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(__builtin_bit_cast(bf16x8_t, kr[kt * kSteps + st]),
                                                          __builtin_bit_cast(bf16x8_t, qv[st]), s[kt], 0, 0, 0);
        } else {
#pragma unroll
          for (int e = 0; e < 4; ++e)
            s[kt] = __builtin_amdgcn_mfma_f32_16x16x4f32(__uint_as_float(kr[kt * kSteps + st][e]),
                                                         __uint_as_float(qv[st][e]), s[kt], 0, 0, 0);
        }
      }
    }
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
      *reinterpret_cast<u32x4 *>(mine + r * kRow + place_of(r, at % kChunks) * 16) = vr[i];
    }
    page = page_next;
    if (b + 4 < b_end) {
      load(b + 4, page);
      page_next = page_of(b + 8);
    }
#pragma unroll
    for (int kt = 0; kt < kTiles; ++kt) s[kt] *= scale2;
    if (!whole) {
      const Sight sight = sight_of(a, place, j0);
      const uint32_t here = (uint32_t)there >> (4 * g);
#pragma unroll
      for (int kt = 0; kt < kTiles; ++kt)
#pragma unroll
        for (int i = 0; i < 4; ++i)
          s[kt][i] = ((here >> (16 * kt + i) & 1) != 0) & sight.sees(16 * kt + 4 * g + i) ? s[kt][i] : -INFINITY;
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
        bf16x8_t p;  // contraction slot (g, e): key 4 g + e of tile 0, then of tile 1
#pragma unroll
        for (int e = 0; e < 8; ++e) p[e] = (__bf16)s[e >> 2][e & 3];
#pragma unroll
        for (int o = 0; o < kOut; ++o) {
          i16x4_t v2[2];
#pragma unroll
          for (int kt = 0; kt < 2; ++kt) {
            const int r = 16 * kt + 4 * g + (row >> 2), c = 2 * o + ((row & 3) >> 1);
            v2[kt] = __builtin_amdgcn_ds_read_tr16_b64_v4i16(
                (lds_i16x4 *)(mine + r * kRow + place_of(r, c) * 16 + (row & 1) * 8));
            if (kOdd) v2[kt] = sane(v2[kt]);
          }
          bf16x8_t v8;
          __builtin_memcpy(&v8, v2, 16);
          acc[o] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(v8, p, acc[o], 0, 0, 0);
        }
      } else {
#pragma unroll
        for (int o = 0; o < kOut; ++o)
#pragma unroll
          for (int i = 0; i < 4; ++i) {
            const int r = 4 * g + i, c = 4 * o + (row >> 2);
            float v = *reinterpret_cast<const float *>(mine + r * kRow + place_of(r, c) * 16 + (row & 3) * 4);
            if (kOdd) v = odd_of(v) ? 0.0f : v;
            acc[o] = __builtin_amdgcn_mfma_f32_16x16x4f32(v, s[0][i], acc[o], 0, 0, 0);
          }
      }
    };
    if (!odd) {
      product(Plain{});
    } else {
      product(Odd{});
#pragma unroll 1
      for (int k = 0; k < kKeys; ++k) {
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
            const float v = Elem<T>::get(reinterpret_cast<const T *>(mine + k * kRow + place_of(k, d / kVec) * 16) + d % kVec);
            if (p != 0.0f && odd_of(v)) acc[o][e] += p * v;
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
// with their 16-byte pieces exchanged, so that the 8 lanes that a cycle serves (K: the
// same piece of 8 rows; V: two pieces of 4 rows) read different banks.
constexpr int kTileRows = 128, kTileKeys = 64;

// 16 bytes of each lane into LDS at dst + 16 * lane (dst the same for the whole wave).
__device__ __forceinline__ void load_to_lds(const void *src, uint8_t *dst) {
  __builtin_amdgcn_global_load_lds((const __attribute__((address_space(1))) void *)src,
                                   (__attribute__((address_space(3))) void *)dst, 16, 0, 0);
}

// Every load of this wave has landed, and every wave is here.
__device__ __forceinline__ void stage_barrier() {
  asm volatile("" ::: "memory");
  __builtin_amdgcn_s_waitcnt(0);
  __builtin_amdgcn_s_barrier();
  asm volatile("" ::: "memory");
}

// The state of a wave's 32 rows: O^T, and of this lane's row the running maximum (of the
// scores before the scale) and the sum.
template <int DT> struct TileSums {
  f32x16_t acc[DT / 32];
  float m, l;
};

// One block for one wave: scores, softmax step, product.  `there`: the block's keys that
// some row of the tile sees.  Returns whether values of keys on which the rows disagree
// hold infinities or NaN (ODD false: the product then has to be made again with ODD).
template <int DT, bool ODD>
__device__ __forceinline__ bool tile_step(const AttendArgs &a, TileSums<DT> &t, const bf16x8_t (&qv)[DT / 16], float scale2,
                                          const uint8_t *kt, const uint8_t *vt, uint64_t there, int64_t j0, int64_t place,
                                          int64_t low, int64_t high) {
  constexpr int kRow = DT * 2, kChunks = kRow / 16, kOut = DT / 32, kSteps = DT / 16;
  constexpr int kLine = kRow < 256 ? 256 / kRow : 1, kMask = (kRow / 32 < 8 ? kRow / 32 : 8) - 1;
  const int lane = threadIdx.x & 63, col = lane & 31, hf = lane >> 5;
  f32x16_t s[2];
#pragma unroll
  for (int x = 0; x < 2; ++x) {
#pragma unroll
    for (int i = 0; i < 16; ++i) s[x][i] = 0.0f;
#pragma unroll
    for (int st = 0; st < kSteps; ++st) {
      const int r = 32 * x + col;
      const u32x4 kv = *reinterpret_cast<const u32x4 *>(kt + r * kRow + ((2 * st + hf) ^ ((r / kLine) & (2 * kMask + 1))) * 16);
      s[x] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(__builtin_bit_cast(bf16x8_t, kv), qv[st], s[x], 0, 0, 0);
    }
  }
  bool odd = false;
  const bool whole = there == ~0ull && j0 + kTileKeys - 1 <= low &&
                     (!a.window || high - j0 < a.window || j0 + kTileKeys <= a.sinks);
  if (!whole) {
    const Sight sight = sight_of(a, place, j0);
    const uint64_t here = there >> (4 * hf);
#pragma unroll
    for (int x = 0; x < 2; ++x)
#pragma unroll
      for (int i = 0; i < 16; ++i) {
        const int k = 32 * x + 8 * (i >> 2) + (i & 3);  // (and 4 hf)
        s[x][i] = ((here >> k & 1) != 0) & sight.sees(k + 4 * hf) ? s[x][i] : -INFINITY;
      }
    for (int c = lane; c < kTileKeys * kChunks; c += 64) odd |= odd_value<uint16_t>(*reinterpret_cast<const u32x4 *>(vt + c * 16));
    odd = __any(odd);
    if (odd && !ODD) return true;
  }
  float top = s[0][0];
#pragma unroll
  for (int i = 1; i < 32; ++i) top = fmaxf(top, s[i >> 4][i & 15]);
  top = fmaxf(top, __shfl_xor(top, 32));
  // the maximum moves, and the sums are scaled to it, only where a weight would pass 2^8
  if (__any(!((top - t.m) * scale2 <= 8.0f))) {
    const float mn = fmaxf(t.m, top), f = mn == t.m ? 1.0f : exp2_fast((t.m - mn) * scale2);
    t.m = mn;
    t.l *= f;
#pragma unroll
    for (int o = 0; o < kOut; ++o)
#pragma unroll
      for (int i = 0; i < 16; ++i) t.acc[o][i] *= f;
  }
  const float base = t.m == -INFINITY ? 0.0f : -t.m * scale2;
  float sum = 0.0f;
#pragma unroll
  for (int x = 0; x < 2; ++x)
#pragma unroll
    for (int i = 0; i < 16; ++i) {
      s[x][i] = exp2_fast(fmaf(s[x][i], scale2, base));
      sum += s[x][i];
    }
  t.l += sum;
#pragma unroll
  for (int st = 0; st < 4; ++st) {
    bf16x8_t p;  // contraction slot (hf, e): key 16 st + 8 (e / 4) + 4 hf + e % 4
#pragma unroll
    for (int e = 0; e < 8; ++e) p[e] = (__bf16)s[st >> 1][8 * (st & 1) + e];
#pragma unroll
    for (int o = 0; o < kOut; ++o) {
      i16x4_t v2[2];
#pragma unroll
      for (int y = 0; y < 2; ++y) {
        const int r = 16 * st + 8 * y + 4 * hf + ((lane & 15) >> 2);
        const int c = (4 * o + 2 * ((lane >> 4) & 1) + ((lane & 3) >> 1)) ^ (2 * ((r / kLine) & kMask));
        v2[y] = __builtin_amdgcn_ds_read_tr16_b64_v4i16((lds_i16x4 *)(vt + r * kRow + c * 16 + (lane & 1) * 8));
        if (ODD && odd) v2[y] = sane(v2[y]);
      }
      bf16x8_t v8;
      __builtin_memcpy(&v8, v2, 16);
      t.acc[o] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(v8, p, t.acc[o], 0, 0, 0);
    }
  }
  if (ODD && odd) {
#pragma unroll 1
    for (int k = 0; k < kTileKeys; ++k) {
      float p = 0.0f;
#pragma unroll
      for (int x = 0; x < 2; ++x)
#pragma unroll
        for (int i = 0; i < 16; ++i)
          if ((k >> 5) == x && ((k >> 3) & 3) == i >> 2 && (k & 3) == (i & 3)) p = s[x][i];
      p = __shfl(p, col + 32 * ((k >> 2) & 1));
#pragma unroll
      for (int o = 0; o < kOut; ++o)
#pragma unroll
        for (int e = 0; e < 16; ++e) {
          const int d = 32 * o + 8 * (e >> 2) + 4 * hf + (e & 3);
          const uint16_t *v = reinterpret_cast<const uint16_t *>(vt + k * kRow + ((d >> 3) ^ (2 * ((k / kLine) & kMask))) * 16);
          if (p != 0.0f && odd_bits(v[d & 7])) t.acc[o][e] += p * bf16_to_f32(v[d & 7]);
        }
    }
  }
  return false;
}

template <int DT>
__global__ __launch_bounds__(256, DT > 128 ? 1 : 2) void attend_tile_kernel(AttendArgs a) {
  constexpr int kRow = DT * 2, kChunks = kRow / 16, kLoads = kTileKeys * kChunks / 256, kOut = DT / 32, kSteps = DT / 16;
  constexpr int kLine = kRow < 256 ? 256 / kRow : 1, kMask = (kRow / 32 < 8 ? kRow / 32 : 8) - 1;
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
  const int64_t place = t.place0 + (t.first + r_in) / a.group;
  // places of this wave's first and last row
  const int w_lo = 32 * w < t.count ? 32 * w : t.count - 1, w_hi = 32 * w + 31 < t.count ? 32 * w + 31 : t.count - 1;
  const int64_t low = t.place0 + (t.first + w_lo) / a.group, high = t.place0 + (t.first + w_hi) / a.group;

  // q with the scale's sign (zeros for a scale of 0), so that the largest product is the largest score
  bf16x8_t qv[kSteps];
  {
    const int r = t.first + r_in;
    const uint16_t *q = (const uint16_t *)a.q + (t.start + r / a.group) * a.q_stride +
                        (int64_t)(kvh * a.group + r % a.group) * a.dim;
#pragma unroll
    for (int s = 0; s < kSteps; ++s) {
      const int c = 2 * s + hf;
      u32x4 x = c * 8 < a.dim && a.scale != 0.0f ? *reinterpret_cast<const u32x4 *>(q + c * 8) : u32x4{0, 0, 0, 0};
      if (a.scale < 0.0f) x ^= 0x80008000u;
      qv[s] = __builtin_bit_cast(bf16x8_t, x);
    }
  }
  const float scale2 = a.scale == 0.0f ? 1.0f : fabsf(a.scale) * kLog2e;
  const char *zeros = reinterpret_cast<const char *>(attend_zeros);
  const int64_t head_bytes = ((int64_t)kvh << a.pool.shift) * a.dim * 2;
  const int64_t page_bytes = ((int64_t)a.pool.n_kv << a.pool.shift) * a.dim * 2;
  const char *kp = (const char *)a.k + head_bytes, *vp = (const char *)a.v + head_bytes;
  const int row_bytes = a.dim * 2;

  auto page_of = [&](int b) { return b < b_end ? key_page(a, t, kb, block_key(kb, b, kTileKeys) + lane) : -1; };
  // wave w loads rows 16 w .. 16 w + 15 of the block (K and V); where all of them are there, in
  // one page and whole, from one address and fixed offsets
  auto issue = [&](int b, int page, uint64_t there, uint8_t *kd, uint8_t *vd) {
    const int j0 = (int)(block_key(kb, b, kTileKeys) & (a.pool.page - 1));
    uint8_t *kw = kd + w * kLoads * 1024, *vw = vd + w * kLoads * 1024;
    if (a.pool.shift >= 4 && (there >> (16 * w) & 0xffffu) == 0xffffu && a.dim == DT) {
      const int64_t p = __builtin_amdgcn_readlane(page, 16 * w);
      const int64_t off = p * page_bytes + ((j0 + 16 * w) & (a.pool.page - 1)) * kRow;
      const char *ks = kp + off, *vs = vp + off;
#pragma unroll
      for (int i = 0; i < kLoads; ++i) {
        const int r = (i * 64 + lane) / kChunks, x = lane % kChunks;
        load_to_lds(ks + (uint32_t)(r * kRow + (x ^ ((r / kLine) & (2 * kMask + 1))) * 16), kw + i * 1024);
        load_to_lds(vs + (uint32_t)(r * kRow + (x ^ (2 * ((r / kLine) & kMask))) * 16), vw + i * 1024);
      }
      return;
    }
#pragma unroll 1
    for (int i = 0; i < kLoads; ++i) {
      const int r = (i * 64 + lane) / kChunks, x = lane % kChunks, p = __shfl(page, 16 * w + r);
      const int64_t off = p * page_bytes + ((j0 + 16 * w + r) & (a.pool.page - 1)) * row_bytes;
      const int kc = x ^ ((r / kLine) & (2 * kMask + 1)), vc = x ^ (2 * ((r / kLine) & kMask));
      load_to_lds(p >= 0 && kc * 8 < a.dim ? kp + off + kc * 16 : zeros, kw + i * 1024);
      load_to_lds(p >= 0 && vc * 8 < a.dim ? vp + off + vc * 16 : zeros, vw + i * 1024);
    }
  };

  TileSums<DT> sums;
  // The tile's blocks; block b lives in buffer (b - b0) % 2: it has landed when every load is
  // done, and the other buffer is free when every wave is past the barrier.  Returns
  // whether a product has to be made again.
  auto run = [&](auto kind) {
    constexpr bool kOdd = decltype(kind)::kOdd;
#pragma unroll
    for (int o = 0; o < kOut; ++o)
#pragma unroll
      for (int i = 0; i < 16; ++i) sums.acc[o][i] = 0.0f;
    sums.m = -INFINITY, sums.l = 0.0f;
    bool again = false;
    int next = page_of(b0), after = page_of(b0 + 1);
    uint64_t there = 0, there_next = __ballot(next >= 0);
    if (b0 < b_end) issue(b0, next, there_next, k0, v0);
    auto step = [&](int b, uint8_t *kt, uint8_t *vt, uint8_t *kn, uint8_t *vn) {
      stage_barrier();
      there = there_next, next = after;
      there_next = __ballot(next >= 0);
      if (b + 1 < b_end) issue(b + 1, next, there_next, kn, vn);
      after = page_of(b + 2);
      if (!again)
        again = tile_step<DT, kOdd>(a, sums, qv, scale2, kt, vt, there, block_key(kb, b, kTileKeys), place, low, high);
    };
    for (int b = b0; b < b_end; b += 2) {
      step(b, k0, v0, k1, v1);
      if (b + 1 < b_end) step(b + 1, k1, v1, k0, v0);
    }
    return again;
  };
  if (__syncthreads_or(run(Plain{}))) run(Odd{});

  float l = sums.l;
  l += __shfl_xor(l, 32);
  if (row >= t.count) return;
  const float m = sums.m * scale2;
#pragma unroll
  for (int o = 0; o < kOut; ++o)
#pragma unroll
    for (int e = 0; e < 4; ++e) {
      const f32x4 v = {sums.acc[o][4 * e], sums.acc[o][4 * e + 1], sums.acc[o][4 * e + 2], sums.acc[o][4 * e + 3]};
      const int d = 32 * o + 8 * e + 4 * hf;
      if (parts > 1) put_part(a, ((int64_t)blockIdx.x * a.splits + z) * kTileRows + row, d, v, m, l);
      else put_row<uint16_t>(a, t, row, kvh, d, v, m, l);
    }
}

// ------------------------------------------------------------------ join

// Joins the parts of a tile's rows where it was split: W waves per row, each part of a row
// held by `lanes` lanes, so that a wave adds 64 / lanes parts at a time and the W waves'
// loads are all in flight.  The order of a row's sum depends on the batch's bounds alone.
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
    const float f = z0 + sub < parts ? exp2_fast(ml[0] - at0) : 0.0f;
    const f32x4 x = *reinterpret_cast<const f32x4 *>(a.part + (at + (int64_t)z * R) * a.dim + dd);
    if (f != 0.0f) l += ml[1] * f, o += x * f;  // (f is NaN where the row's maximum is an infinity)
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

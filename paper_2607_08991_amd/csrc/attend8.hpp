// Attention over a cache of 8 bits (gfx950): the tiles, masks, softmax and parts of attend.hpp with
// other loads.  Codes become bf16 numbers in registers (exactly: their scales are powers of two), those
// of E4M3 with the scale in the converting instruction, and multiply as those of a bf16 cache do.
// Queries of float32 go in as three bf16 pieces (24 bits), weights for them too, so that float32
// callers lose nothing but what the cache has lost.
//
// Pages have 16 tokens or more here, so that 16 keys have one address.
#pragma once

#include "attend.hpp"

namespace sats {

typedef int i32x2_t __attribute__((ext_vector_type(2)));
typedef __attribute__((address_space(3))) i32x2_t lds_i32x2;

// ------------------------------------------------------------------ tiles of 16 rows

// As attend_rows, with two blocks of a wave on their way: K's codes in registers, V's straight into LDS (as
// codes: its transposing reads give a lane eight keys of a dim, which it converts then).  V's scales belong to the keys,
// so they go into the weights.
//
// Bound by the cache's bytes and by their conversion (two numbers an instruction for E4M3, five instructions for two of
// INT8): 64 sequences of 500 to 8000 keys (8 heads of 128, four rows each, 359 MB of E4M3) take 95.5 us with the join, 3.75
// TB/s, where a bf16 cache takes 146 us for 711 MB; INT8 99.6.  Two blocks ahead because one of 8 bits is half the bytes: with one, and
// three workgroups a compute unit, 139.  Heads of 64, 80, 96, 256 (half as many of the last): 61, 100, 103, 156.
// One sequence of 32768 keys: 21.9 us and 8.3 in the join (67.6 MB, 14 us).  float32 over the same 64
// sequences (INT8): 107 us, three products for one with queries and three for two with values.
//
// Rows of V lie in LDS as in the cache, their 16-byte pieces exchanged so that the eight rows of a read
// (keys 4 g .. and 16 + 4 g ..) are in different banks.
template <int DT> struct Rows8 {
  static constexpr int kKeys = 32, kChunks = DT / 16, kBytes = kKeys * DT;  // of a wave's buffer
  __device__ __forceinline__ static int piece(int r, int c) {
    return c ^ (DT > 64 ? (r & 3) | (r >> 2 & 4) : r >> 4 & 1);
  }
};
// Waits until at most N loads are on their way, or for LDS.
template <int N> __device__ __forceinline__ void wait_loads() {
  asm volatile("" ::: "memory");
  __builtin_amdgcn_s_waitcnt((N & 15) | (N >> 4) << 14 | 0xf70);
  asm volatile("" ::: "memory");
}
__device__ __forceinline__ void wait_lds() {
  asm volatile("" ::: "memory");
  __builtin_amdgcn_s_waitcnt(0xc07f);
  asm volatile("" ::: "memory");
}

// x: tile and cache head; z: split.  v0, v1: a buffer for each wave; lds: 16 x DT floats for each wave, over the same.
template <typename T, int F, int DT, bool FULL, bool PHASED>
__device__ __forceinline__ void attend_rows8(const AttendArgs &a, int x, int z, uint8_t *v0, uint8_t *v1, uint8_t *const (&lds)[4],
                                             float (&ml)[4][16][2]) {
  using R8 = Rows8<DT>;
  constexpr int kKeys = R8::kKeys, kTiles = 2, kOut = DT / 16, kChunks = R8::kChunks, kSteps = DT / 64;
  constexpr int kLoads = kKeys * kChunks / 64, kPer = kLoads / kTiles, kPieces = sizeof(T) == 2 ? 1 : 3;
  constexpr bool kSkip = !FULL && DT <= 128;

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
  const int lane = threadIdx.x & 63, w = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), row = lane & 15, g = lane >> 4;
  int64_t place;
  if constexpr (PHASED) place = places.of(row);
  else place = t.place0 + (t.first + (row < t.count ? row : t.count - 1)) / a.group;
  const bool several = kb.low != kb.high;

  // Q as the second operand: of this lane's row the dims 16 (g + 4 s) .. + 15, as a lane has a key's codes
  u32x4 qv[kPieces][kSteps][2];
  {
    const int r = t.first + (row < t.count ? row : t.count - 1);
    const T *q = (const T *)a.q + (t.start + r / a.group) * a.q_stride + (int64_t)(kvh * a.group + r % a.group) * a.dim;
#pragma unroll
    for (int s = 0; s < kSteps; ++s)
#pragma unroll
      for (int y = 0; y < 2; ++y) {
        const int d = 16 * (g + 4 * s) + 8 * y;
        if constexpr (sizeof(T) == 2) {
          qv[0][s][y] = d < a.dim ? *reinterpret_cast<const u32x4 *>(q + d) : u32x4{0, 0, 0, 0};
        } else {
          float x[8];
#pragma unroll
          for (int i = 0; i < 8; i += 4) {
            const f32x4 v = d < a.dim ? *reinterpret_cast<const f32x4 *>(q + d + i) : f32x4{0, 0, 0, 0};
#pragma unroll
            for (int j = 0; j < 4; ++j) x[i + j] = v[j];
          }
#pragma unroll
          for (int p = 0; p < kPieces; ++p) {
            bf16x8_t piece;
#pragma unroll
            for (int i = 0; i < 8; ++i) {
              const float top = odd_of(x[i]) ? x[i] : __uint_as_float(__float_as_uint(x[i]) & 0xffff0000u);
              piece[i] = (__bf16)top;
              x[i] = odd_of(x[i]) ? 0.0f : x[i] - top;  // (what is infinite or NaN is so in its first piece)
            }
            qv[p][s][y] = __builtin_bit_cast(u32x4, piece);
          }
        }
      }
  }
  const float scale2 = a.scale * kLog2e;
  const int64_t head_bytes = ((int64_t)kvh << a.pool.shift) * a.dim, head_rows = (int64_t)kvh << a.pool.shift;
  const int64_t page_bytes = ((int64_t)a.pool.n_kv << a.pool.shift) * a.dim, page_rows = (int64_t)a.pool.n_kv << a.pool.shift;
  const char *kp = (const char *)a.k + head_bytes, *vp = (const char *)a.v + head_bytes;
  const char *ksp = (const char *)a.k_scale + head_rows, *vsp = (const char *)a.v_scale + head_rows;

  // A block on its way: K's codes and scales (of key 16 kt + row), V's scales (of keys 16 kt + 4 g ..), which of its keys
  // some row sees.
  struct Held {
    u32x4 k[kTiles][kSteps];
    uint32_t vs[kTiles];
    uint8_t ks[kTiles];
    uint32_t there;
    int page;  // of key lane % 32
  };
  constexpr int kHeldLoads = kTiles * (kSteps + 2);
  auto entry_of = [&](int b) {
    return b < b_end ? key_entry<PHASED>(a, t, kb, block_key(kb, b, kKeys) + (lane & (kKeys - 1))) : -1;
  };
  // the pages and first slot of 16 keys of a block
  auto page_at = [&](const Held &h, int kt) {
    const uint32_t here = h.there >> (16 * kt) & 0xffffu;
    return here ? (int64_t)__builtin_amdgcn_readlane(h.page, 16 * kt + __builtin_ctz(here)) : 0;
  };
  auto slot_at = [&](int b, int kt) {
    return ((int)(block_key(kb, b, kKeys) & (a.pool.page - 1)) + 16 * kt) & (a.pool.page - 1);
  };
  // (Of a block past the last no key is there: every load reads zeros.  No load is under a condition, so that the
  // waits count them.)
  auto load = [&](Held &h, int b, int entry) {
    h.page = page_or_none(a, entry);
    h.there = (uint32_t)__ballot(h.page >= 0);
#pragma unroll
    for (int kt = 0; kt < kTiles; ++kt) {
      const uint32_t here = h.there >> (16 * kt) & 0xffffu;
      const int64_t p = page_at(h, kt);
      const int slot = slot_at(b, kt);
      const __amdgpu_buffer_rsrc_t rk = rows_rsrc(kp + p * page_bytes + slot * a.dim);
      const __amdgpu_buffer_rsrc_t rks = rows_rsrc(ksp + p * page_rows + slot), rvs = rows_rsrc(vsp + p * page_rows + slot);
      const bool k_here = here >> row & 1;
      const uint32_t k_off = k_here ? row * a.dim + g * 16 : kNoRow;
      h.ks[kt] = __builtin_amdgcn_raw_buffer_load_b8(rks, k_here ? row : kNoRow, 0, 0);
      h.vs[kt] = __builtin_amdgcn_raw_buffer_load_b32(rvs, here ? 4 * g : kNoRow, 0, 0);
#pragma unroll
      for (int s = 0; s < kSteps; ++s)
        h.k[kt][s] = __builtin_bit_cast(u32x4, __builtin_amdgcn_raw_buffer_load_b128(
                                                   rk, FULL || (4 * s + g) * 16 < a.dim ? k_off + 64 * s : kNoRow, 0, 0));
    }
  };
  auto load_v = [&](const Held &h, int b, uint8_t *to) {
#pragma unroll
    for (int kt = 0; kt < kTiles; ++kt) {
      const uint32_t here = h.there >> (16 * kt) & 0xffffu;
      const char *from = vp + page_at(h, kt) * page_bytes + slot_at(b, kt) * a.dim;
#pragma unroll
      for (int i = 0; i < kPer; ++i) {
        const int r = (i * 64 + lane) / kChunks, c = R8::piece(16 * kt + r, lane % kChunks);
        load_to_lds<0>(from, (here >> r & 1) && (FULL || c * 16 < a.dim) ? (uint32_t)(r * a.dim + c * 16) : kNoRow,
                       to + (kt * kPer + i) * 1024);
      }
    }
  };

  f32x4 acc[kOut];
#pragma unroll
  for (int i = 0; i < kOut; ++i) acc[i] = f32x4{0, 0, 0, 0};
  float m = -INFINITY, l = 0.0f;

  int entry;  // the table's, of the block after the next
  auto step = [&](Held &h, int b, uint8_t *mine) {
    const int64_t j0 = block_key(kb, b, kKeys);
    const uint32_t here = h.there;
    const bool whole = here == ~0u && j0 + kKeys - 1 <= kb.low &&
                       (!a.window || kb.high - j0 < a.window || j0 + kKeys <= a.sinks);
    // scores: lane (row, keys 16 kt + 4 g + i)
    f32x4 s[kTiles];
#pragma unroll
    for (int kt = 0; kt < kTiles; ++kt) {
      s[kt] = f32x4{0, 0, 0, 0};
      const float f = scale_of<F>(h.ks[kt]);
#pragma unroll
      for (int st = 0; st < kSteps; ++st) {
        if (kSkip && st * 64 >= a.dim) break;
#pragma unroll
        for (int y = 0; y < 2; ++y) {
          const bf16x8_t k8 = __builtin_bit_cast(bf16x8_t, decode8<F>(h.k[kt][st][2 * y], h.k[kt][st][2 * y + 1], f));
#pragma unroll
          for (int p = kPieces - 1; p >= 0; --p)
            s[kt] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(k8, __builtin_bit_cast(bf16x8_t, qv[p][st][y]), s[kt], 0, 0, 0);
        }
      }
    }
    uint32_t vs[kTiles];
#pragma unroll
    for (int kt = 0; kt < kTiles; ++kt) vs[kt] = h.vs[kt];
    asm volatile("" ::: "memory");
    const int after = entry_of(b + 12);
    load(h, b + 8, entry);
    entry = after;
    asm volatile("" ::: "memory");
#pragma unroll
    for (int kt = 0; kt < kTiles; ++kt) s[kt] *= scale2;
    uint32_t seen = ~0u;  // which of its eight keys this lane's row sees: bit 4 kt + i
    if (!whole) {
      const Sight sight = sight_of(a, place, j0);
      const uint32_t mask = here >> (4 * g);
      seen = 0;
#pragma unroll
      for (int kt = 0; kt < kTiles; ++kt)
#pragma unroll
        for (int i = 0; i < 4; ++i) {
          const bool sees = ((mask >> (16 * kt + i) & 1) != 0) & sight.sees(16 * kt + 4 * g + i);
          s[kt][i] = sees ? s[kt][i] : -INFINITY;
          seen |= (uint32_t)sees << (4 * kt + i);
        }
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
        s[kt][i] = exp2_fast(s[kt][i] - at0);
        sum += s[kt][i];
        // the weight of the key's codes (255, NaN, goes in as infinity: its codes are zeros)
        const uint32_t byte = vs[kt] >> (8 * i) & 0xffu;
        s[kt][i] *= __uint_as_float(byte ? byte << 23 : 0x00400000u);
      }
    if (!whole) {
#pragma unroll
      for (int kt = 0; kt < kTiles; ++kt)
#pragma unroll
        for (int i = 0; i < 4; ++i) s[kt][i] = seen >> (4 * kt + i) & 1 ? s[kt][i] : 0.0f;
    }
    l = l * f + sum;
#pragma unroll
    for (int i = 0; i < kOut; ++i) acc[i] *= f;
    // V of this block is there: what was issued since is the next one's and half of the one after
    wait_loads<kLoads + 2 * kHeldLoads>();
    bool odd = false;  // codes that are NaN, in a block in which rows disagree on a key
    if (F == kE4m3 && several && !whole) {
      for (int i = lane; i < R8::kBytes / 4; i += 64) {
        const uint32_t c = reinterpret_cast<const uint32_t *>(mine)[i];
        odd |= ((c & 0x7f7f7f7fu) + 0x01010101u & 0x80808080u) != 0;
      }
      odd = __any(odd);
    }
    auto product = [&](auto kind) {
      constexpr bool kOdd = decltype(kind)::kOdd;
      // a weight in two pieces of 8 bits (the second as attend_rows has it), for float32 in three
      constexpr int kWeights = kPieces == 1 ? 2 : 3;
      bf16x8_t p[kWeights];
#pragma unroll
      for (int e = 0; e < 8; ++e) {
        float x = s[e >> 2][e & 3];
#pragma unroll
        for (int i = 0; i < kWeights - 1; ++i) {
          const float top = __uint_as_float(__float_as_uint(x) & 0xffff0000u);
          p[i][e] = (__bf16)top;
          x = kWeights == 2 ? fmaf(x, 1.0f + 0x1p-20f, -top) : x - top;
        }
        p[kWeights - 1][e] = (__bf16)x;
      }
      // contraction slot (g, e): key 4 g + e of tile 0, then of tile 1
      const int j = row >> 1, r = (j < 4 ? 0 : 12) + 4 * g + j;
      int at = r * DT + R8::piece(r, 0) * 16 + (row & 1) * 8;
#pragma unroll
      for (int o = 0; o < kOut; ++o) {
        if (kSkip && 16 * o >= a.dim) break;
        i32x2_t c = __builtin_amdgcn_ds_read_tr8_b64_v2i32((lds_i32x2 *)(mine + (at ^ (16 * o))));
        if (kOdd) {
#pragma unroll
          for (int y = 0; y < 2; ++y) {
            const uint32_t nan = ((uint32_t)c[y] & 0x7f7f7f7fu) + 0x01010101u & 0x80808080u;
            c[y] &= ~((nan >> 7) * 0xffu);
          }
        }
        const bf16x8_t v8 = __builtin_bit_cast(bf16x8_t, decode8<F>((uint32_t)c[0], (uint32_t)c[1], 1.0f));
#pragma unroll
        for (int i = kWeights - 1; i >= 0; --i) acc[o] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(v8, p[i], acc[o], 0, 0, 0);
      }
    };
    if (!odd) {
      product(Plain{});
    } else {
      product(Odd{});
      const Sight sight = sight_of(a, place, j0);
#pragma unroll 1
      for (int k = 0; k < kKeys; ++k) {
        if (!(((here >> k & 1) != 0) & sight.sees(k))) continue;
#pragma unroll
        for (int o = 0; o < kOut; ++o)
#pragma unroll
          for (int e = 0; e < 4; ++e)
            if ((mine[k * DT + R8::piece(k, o) * 16 + 4 * g + e] & 0x7f) == 0x7f) acc[o][e] = __uint_as_float(0x7fc00000u);
      }
    }
    wait_lds();  // (its buffer is the one of the block after the next)
    load_v(h, b + 8, mine);
    asm volatile("" ::: "memory");
  };
  int b = z * a.per_split + w;
  uint8_t *const mine0 = v0 + w * R8::kBytes, *const mine1 = v1 + w * R8::kBytes;
  Held h0, h1;
  const int p0 = entry_of(b), p1 = entry_of(b + 4);
  entry = entry_of(b + 8);
  asm volatile("" ::: "memory");
  load(h0, b, p0);
  asm volatile("" ::: "memory");
  load_v(h0, b, mine0);
  asm volatile("" ::: "memory");
  load(h1, b + 4, p1);
  asm volatile("" ::: "memory");
  load_v(h1, b + 4, mine1);
  asm volatile("" ::: "memory");
  while (b < b_end) {
    step(h0, b, mine0);
    if ((b += 4) >= b_end) break;
    step(h1, b, mine1);
    b += 4;
  }
  wait_loads<0>();  // (before others write their sums where these loads go)
  uint8_t *mine = w == 0 ? lds[0] : w == 1 ? lds[1] : w == 2 ? lds[2] : lds[3];
  finish_rows<T, DT>(a, t, x, z, parts > 1 || PHASED, m, l, acc, mine, lds, ml);
}

template <typename T, int F, int DT, bool FULL>
__global__ __launch_bounds__(256, DT > 128 ? 1 : DT > 64 ? 2 : 3) void attend_rows8_kernel(AttendArgs a) {
  __shared__ __align__(16) uint8_t v0[4 * Rows8<DT>::kBytes], v1[4 * Rows8<DT>::kBytes];
  __shared__ float ml[4][16][2];
  uint8_t *const part[4] = {v0, v0 + 64 * DT, v1, v1 + 64 * DT};
  attend_rows8<T, F, DT, FULL, false>(a, blockIdx.x, blockIdx.y, v0, v1, part, ml);
}
template <typename T, int F, int DT, bool FULL>
__global__ __launch_bounds__(256, DT > 128 ? 1 : DT > 64 ? 2 : 3) void attend_rows8_phases_kernel(AttendArgs a, PhaseArgs p) {
  __shared__ __align__(16) uint8_t v0[4 * Rows8<DT>::kBytes], v1[4 * Rows8<DT>::kBytes];
  __shared__ float ml[4][16][2];
  uint8_t *const part[4] = {v0, v0 + 64 * DT, v1, v1 + 64 * DT};
  int x, z;
  take_set(a, p, blockIdx.x, &x, &z);
  attend_rows8<T, F, DT, FULL, true>(a, x, z, v0, v1, part, ml);
  put_row_parts<16>(a, p, x, z);
}

// ------------------------------------------------------------------ tiles of 128 rows

// As attend_tile, whose blocks come from memory straight into LDS: here a wave's codes of a block
// are in registers for the length of a step, and become bf16 rows in LDS at the start of the next.
//
// Bound by instruction issue: a step converts 2 x 8 pieces a wave and stores them, which a bf16 cache leaves to
// its loads, and INT8 takes more instructions for it (2750 for two blocks, E4M3 2240).  2048 tokens on 4096 (32 heads of 128 on
// 8, 172 Gflop): E4M3 241 us (713 TFLOP/s), INT8 313 to 343, bf16 200.  K's and V's codes, their scales and pages live through a step
// in a kernel that has no registers left: the compiler spills 90 (E4M3, 128 dims) and 273 (INT8), 253 and 543 at 256 dims,
// where attend_tile_kernel spills 52 and 115; in phases 136 and 289, 171 and 521.  At 128 dims 8 and 19 of the accesses are
// in the loop of two blocks, the others around it and in the loop for infinities and NaN (73 and 185).  The places of a row's pieces in LDS differ in fixed bits, so that a step has one address for its stores (276 us
// with an address for each).  Heads of 64 and 256 (half and twice as many dims): 282 and 398 of E4M3, 354 and 560 of INT8.
template <int F, int DT, bool FULL, bool PHASED>
__device__ __forceinline__ void attend_tile8(const AttendArgs &a, int x, int z, uint8_t *k0, uint8_t *k1, uint8_t *v0, uint8_t *v1) {
  using Wave = TileWave<DT, FULL>;
  constexpr int kRow = Wave::kRow, kCodes = DT / 16, kLoads = 16 * kCodes / 64;  // (a wave's 16 rows of a block)

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
  const int lane = threadIdx.x & 63, w = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), col = lane & 31;
  const int row = 32 * w + col, r_in = row < t.count ? row : t.count - 1;  // (rows past the last repeat it)

  Wave wave;
  if constexpr (PHASED) wave.take_places(places, w, col);
  else wave.take_places(a, t, w, r_in);
  wave.take_rows(a, t, kvh, r_in);
  const int64_t head_rows = (int64_t)kvh << a.pool.shift, page_rows = (int64_t)a.pool.n_kv << a.pool.shift;
  const char *kp = (const char *)a.k + head_rows * a.dim, *vp = (const char *)a.v + head_rows * a.dim;
  const char *ksp = (const char *)a.k_scale + head_rows, *vsp = (const char *)a.v_scale + head_rows;
  const int32_t *table = PHASED ? t.pages : a.batch.table + t.seq * a.batch.max_pages;

  HeldPages held;
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
  // wave w's 16 rows of a block: load i holds rows i * (64 / kCodes) .., piece lane % kCodes
  struct Codes {
    u32x4 c[kLoads];
    uint8_t s[kLoads];
  };
  Codes kc, vc;
  const int r0 = lane / kCodes, c0 = lane % kCodes;
  auto fetch = [&](int b, int page, uint64_t there, const char *pool, const char *scales, Codes &to) {
    const int slot = ((int)(block_key(kb, b, kTileKeys) & (a.pool.page - 1)) + 16 * w) & (a.pool.page - 1);
    const uint32_t here = (uint32_t)(there >> (16 * w)) & 0xffffu;
    const int64_t p = here ? __builtin_amdgcn_readlane(page, 16 * w + __builtin_ctz(here)) : 0;
    const __amdgpu_buffer_rsrc_t rc = rows_rsrc(pool + (p * page_rows + slot) * a.dim), rs = rows_rsrc(scales + p * page_rows + slot);
#pragma unroll
    for (int i = 0; i < kLoads; ++i) {
      const int r = i * (64 / kCodes) + r0;
      const bool in = here >> r & 1;
      to.c[i] = __builtin_bit_cast(u32x4, __builtin_amdgcn_raw_buffer_load_b128(
                                              rc, in && (FULL || c0 * 16 < a.dim) ? r * a.dim + c0 * 16 : kNoRow, 0, 0));
      to.s[i] = __builtin_amdgcn_raw_buffer_load_b8(rs, in ? r : kNoRow, 0, 0);
    }
  };
  // (the places of a row's pieces are exchanged by bits of its number, and i and y are bits of their own: places
  // differ from the first one in fixed bits, and in whole rows)
  auto put = [&](const Codes &from, uint8_t *to, auto place) {
    int at = r0 * kRow + place(r0, 2 * c0) * 16;
    asm volatile("" : "+v"(at));
    to += 16 * w * kRow;
#pragma unroll
    for (int i = 0; i < kLoads; ++i) {
      const int r = i * (64 / kCodes);
      const float f = scale_of<F>(from.s[i]);
#pragma unroll
      for (int y = 0; y < 2; ++y)
        *reinterpret_cast<u32x4 *>(to + (at ^ (place(r, y) * 16)) + r * kRow) = decode8<F>(from.c[i][2 * y], from.c[i][2 * y + 1], f);
    }
  };
  auto put_k = [&](uint8_t *to) { put(kc, to, Wave::k_place); };
  auto put_v = [&](uint8_t *to) { put(vc, to, Wave::v_place); };

  // K of block b is in buffer (b - b0) % 2, V likewise.  At the barrier of step b every wave's rows (K of
  // b + 1, V of b) are in LDS, and K of b and V of b - 1 have been read by all; the codes of K of
  // b + 2 and V of b + 1 are in registers, or on their way.
  auto run = [&](auto kind) {
    constexpr bool kOdd = decltype(kind)::kOdd;
    wave.clear();
    bool again = false;
    if (b0 >= b_end) return again;
    f32x16_t sa[2], sb[2];
    held.first = -1;
    int page = page_of(b0);
    uint64_t here = __ballot(page >= 0), there_next, there;  // (of the block at hand, of the next, of the one after)
    fetch(b0, page, here, kp, ksp, kc);
    fetch(b0, page, here, vp, vsp, vc);
    put_k(k0);
    put_v(v0);
    int next = page_of(b0 + 1);
    there_next = __ballot(next >= 0);
    if (b0 + 1 < b_end) {
      fetch(b0 + 1, next, there_next, kp, ksp, kc);
      fetch(b0 + 1, next, there_next, vp, vsp, vc);
      put_k(k1);
    }
    page = page_of(b0 + 2);
    there = __ballot(page >= 0);
    if (b0 + 2 < b_end) fetch(b0 + 2, page, there, kp, ksp, kc);
    stage_barrier();
    wave.scores(k0, sa);
    bool some = !wave.whole(a, here, block_key(kb, b0, kTileKeys));  // rows disagree on a key of the block at hand
    if (some) wave.mask(a, here, block_key(kb, b0, kTileKeys), sa);
    float top = sa[0][0];
#pragma unroll
    for (int i = 1; i < 32; ++i) top = fmaxf(top, sa[i >> 4][i & 15]);
    wave.rescale(top);
    auto step = [&](int b, f32x16_t (&s)[2], f32x16_t (&sn)[2], uint8_t *kt, uint8_t *kn, uint8_t *vt, uint8_t *vn) {
      stage_barrier();
      if (b + 2 < b_end) put_k(kt);
      put_v(vn);
      if (b + 2 < b_end) fetch(b + 2, page, there, vp, vsp, vc);
      const int after = page_of(b + 3);
      const uint64_t there_after = __ballot(after >= 0);
      if (b + 3 < b_end) fetch(b + 3, after, there_after, kp, ksp, kc);
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
      here = there_next, there_next = there, there = there_after, page = after;
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

template <int F, int DT, bool FULL>
__global__ __launch_bounds__(256, DT > 128 ? 1 : 2) void attend_tile8_kernel(AttendArgs a) {
  constexpr int kBytes = kTileKeys * TileWave<DT, FULL>::kRow;
  __shared__ __align__(16) uint8_t k0[kBytes], k1[kBytes], v0[kBytes], v1[kBytes];
  attend_tile8<F, DT, FULL, false>(a, blockIdx.x, blockIdx.y, k0, k1, v0, v1);
}
template <int F, int DT, bool FULL>
__global__ __launch_bounds__(256, DT > 128 ? 1 : 2) void attend8_phases_kernel(AttendArgs a, PhaseArgs p) {
  constexpr int kBytes = kTileKeys * TileWave<DT, FULL>::kRow;
  __shared__ __align__(16) uint8_t k0[kBytes], k1[kBytes], v0[kBytes], v1[kBytes];
  __shared__ float ml[4][16][2];
  int x, z;
  if (take_set(a, p, blockIdx.x, &x, &z) & 1) {
    attend_tile8<F, DT, FULL, true>(a, x, z, k0, k1, v0, v1);
    put_row_parts<kTileRows>(a, p, x, z);
  } else {
    static_assert(kBytes == 4 * Rows8<DT>::kBytes, "");
    uint8_t *const part[4] = {k0, k0 + 64 * DT, k1, k1 + 64 * DT};
    attend_rows8<uint16_t, F, DT, FULL, true>(a, x, z, k0, k1, part, ml);
    put_row_parts<16>(a, p, x, z);
  }
}

}  // namespace sats

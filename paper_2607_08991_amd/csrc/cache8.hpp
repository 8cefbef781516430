// Keys and values in 8 bits: the formats of a cache's rows, and reading a cache back (gfx950).
//
// A row (a token's head) is head_dim codes and a scale byte b; code c stands for c 2^(b - 127),
// c being an E4M3 number (448 at most) or a whole number from -127 to 127, and b = 255 for NaN.
// b is the smallest from 1 to 254 at which the row's largest magnitude is within the codes, and a
// value goes to the nearest code, ties to even.  A row with infinities or NaN is zeros under 255.
//
// The scales are powers of two, so that a value read back is exactly a bf16 number (above 2^-126:
// a code has at most 7 significant bits): what multiplies it needs no scale of its own, the
// conversion of E4M3 takes it in the same instruction, and attention over such a cache is attention
// over a bf16 one.  An E4M3 number is no less exact for it; a step of INT8 is up to twice as wide as
// with max |x| / 127.
#pragma once

#include "paged.hpp"

namespace sats {

enum : int { kPlain = 0, kE4m3 = 1, kInt8 = 2 };  // formats of a cache's rows (kPlain: its elements as they are)

typedef __bf16 bf16x2_t __attribute__((ext_vector_type(2)));
typedef __bf16 bf16x8_t __attribute__((ext_vector_type(8)));

// The scale of byte b, as decode4 takes it: the conversion of E4M3 looks at the exponent alone, of
// which 0 is 2^-127 and 255 NaN.
template <int F> __device__ __forceinline__ float scale_of(uint32_t b) {
  return __uint_as_float(F == kE4m3 ? b << 23 : b == 0 ? 0x00400000u : b == 255 ? 0x7fc00000u : b << 23);
}

// Four codes as bf16 numbers, two a word.
template <int F> __device__ __forceinline__ void decode4(uint32_t codes, float scale, uint32_t (&w)[2]) {
  if constexpr (F == kE4m3) {
    const bf16x2_t lo = __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(codes, scale, false);
    const bf16x2_t hi = __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(codes, scale, true);
    __builtin_memcpy(&w[0], &lo, 4);
    __builtin_memcpy(&w[1], &hi, 4);
  } else {
    float f[4];  // (the upper halves of such products are all of them)
#pragma unroll
    for (int i = 0; i < 4; ++i) f[i] = (float)(int8_t)(codes >> (8 * i)) * scale;
    w[0] = __builtin_amdgcn_perm(__float_as_uint(f[1]), __float_as_uint(f[0]), 0x07060302);
    w[1] = __builtin_amdgcn_perm(__float_as_uint(f[3]), __float_as_uint(f[2]), 0x07060302);
  }
}
// Eight codes of words i and i + 1.
template <int F> __device__ __forceinline__ u32x4 decode8(uint32_t c0, uint32_t c1, float scale) {
  uint32_t a[2], b[2];
  decode4<F>(c0, scale, a);
  decode4<F>(c1, scale, b);
  return u32x4{a[0], a[1], b[0], b[1]};
}

// The scale byte of a row whose largest magnitude has the bits `top`, and the factor and limit of
// its codes.  (The limit cuts off what would round past the largest float32 when it is read.)
struct RowScale {
  uint32_t byte;
  float factor, limit;
};
template <int F> __device__ __forceinline__ RowScale row_scale(uint32_t top) {
  if (top >= 0x7f800000u) return {255u, 0.0f, 0.0f};
  constexpr int kTop = F == kE4m3 ? 8 : 6;                          // 448 = 1.75 * 2^8, 127 = 1.984375 * 2^6
  constexpr uint32_t kPart = F == kE4m3 ? 0x600000u : 0x7e0000u;
  const int e = (int)(top >> 23) - 127 - kTop + ((top & 0x7fffffu) > kPart);
  const int k = e < -126 ? -126 : e;
  const float most = F == kE4m3 ? 448.0f : 127.0f, last = F == kE4m3 ? 240.0f : 63.0f;
  return {(uint32_t)(k + 127), __uint_as_float((uint32_t)(127 - k) << 23), k == 128 - kTop ? last : most};
}
// Codes of N numbers (N: 1 or 4) in a word's bytes.
template <int F, int N> __device__ __forceinline__ uint32_t encode(const float *x, const RowScale &s) {
  if (s.byte == 255) return 0;
  float y[4] = {0.0f, 0.0f, 0.0f, 0.0f};
#pragma unroll
  for (int i = 0; i < N; ++i) y[i] = fminf(fmaxf(x[i] * s.factor, -s.limit), s.limit);
  if constexpr (F == kE4m3) {
    const int lo = __builtin_amdgcn_cvt_pk_fp8_f32(y[0], y[1], 0, false);
    return (uint32_t)(N > 1 ? __builtin_amdgcn_cvt_pk_fp8_f32(y[2], y[3], lo, true) : lo);
  } else {
    uint32_t w = 0;
#pragma unroll
    for (int i = 0; i < N; ++i) w |= ((uint32_t)(int)rintf(y[i]) & 0xffu) << (8 * i);
    return w;
  }
}

// V codes at p (V > 1: on 4 bytes).
template <int F, int V> __device__ __forceinline__ void store_codes(uint8_t *p, const float (&x)[V], const RowScale &s) {
  if constexpr (V == 1) {
    *p = (uint8_t)encode<F, 1>(x, s);
  } else {
#pragma unroll
    for (int i = 0; i < V; i += 4) *reinterpret_cast<uint32_t *>(p + i) = encode<F, 4>(x + i, s);
  }
}

// ------------------------------------------------------------------ reading back

struct ReadArgs {
  const void *k, *v;                // of the layer
  const uint8_t *k_scale, *v_scale; // of the layer, 8-bit caches
  void *k_out, *v_out;              // or null
  int64_t k_stride, v_stride;       // elements between tokens
  BatchView batch;
  PoolView pool;
  int dim, chunks;                  // chunks: pieces of 8 dims of a row
};

// Eight dims a thread; zeros for a token without a page, nothing for one of no sequence.
// Bound by memory where there are tokens: 4096 of 8 heads of 128 (INT8 into bf16, 25.4 MB) take 8.0 us, 3.2 TB/s of
// which the codes have just been written; one token is the launch, 4.6 us.
template <typename C, int F, typename T, bool WIDE>
__global__ __launch_bounds__(kThreads) void cache_read_kernel(ReadArgs a) {
  const int64_t u = (int64_t)blockIdx.x * kThreads + threadIdx.x;
  const int per = a.pool.n_kv * a.chunks;
  const int64_t t = u / per;
  if (t >= a.batch.n_tokens) return;
  const int x = (int)(u - t * per), h = x / a.chunks, d = (x - h * a.chunks) * 8;
  int seq;
  const int64_t place = token_place(a.batch, t, &seq);
  if (t < a.batch.q_start[seq] || t >= a.batch.q_start[seq + 1]) return;
  int64_t row = pool_row(a.batch, a.pool, seq, place);
  if (row >= 0) row += (int64_t)h << a.pool.shift;
#pragma unroll
  for (int kv = 0; kv < 2; ++kv) {
    T *out = (T *)(kv ? a.v_out : a.k_out);
    if (!out) continue;
    out += t * (kv ? a.v_stride : a.k_stride) + (int64_t)h * a.dim + d;
    float v[8];
#pragma unroll
    for (int i = 0; i < 8; ++i) v[i] = 0.0f;
    if (row >= 0) {
      const C *src = (const C *)(kv ? a.v : a.k) + row * a.dim + d;
      if constexpr (F == kPlain) {
        constexpr int V = Elem<C>::kVec;
#pragma unroll
        for (int i = 0; i < 8; i += V) {
          float w[V];
          load_vec<C, V>(src + i, w);
#pragma unroll
          for (int j = 0; j < V; ++j) v[i + j] = w[j];
        }
      } else {
        const uint2 c = *reinterpret_cast<const uint2 *>(src);
        const u32x4 w = decode8<F>(c.x, c.y, scale_of<F>((kv ? a.v_scale : a.k_scale)[row]));
#pragma unroll
        for (int i = 0; i < 8; ++i) v[i] = unpack<uint16_t>(w, i);
      }
    }
    T o[8];
#pragma unroll
    for (int i = 0; i < 8; ++i) o[i] = Elem<T>::round(v[i]);
    if constexpr (WIDE) {
#pragma unroll
      for (int i = 0; i < (int)sizeof(T) / 2; ++i) {
        u32x4 w;
        __builtin_memcpy(&w, reinterpret_cast<const char *>(o) + 16 * i, 16);
        reinterpret_cast<u32x4 *>(out)[i] = w;
      }
    } else {
#pragma unroll
      for (int i = 0; i < 8; ++i) out[i] = o[i];
    }
  }
}

}  // namespace sats

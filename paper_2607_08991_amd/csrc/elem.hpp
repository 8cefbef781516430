// Elements, vector loads and the hand-off between workgroups that every kernel of the
// library shares (gfx950).
#pragma once

#include <hip/hip_runtime.h>
#include <stdint.h>

namespace sats {

constexpr int kThreads = 256;

// ------------------------------------------------------------------ elements

__device__ __forceinline__ float bf16_to_f32(uint32_t b) { return __uint_as_float(b << 16); }

// float -> bfloat16 bits, round to nearest even (from the bit layout: add half
// an ulp of the kept part, plus one when the kept part is odd, then truncate)
__device__ __forceinline__ uint16_t f32_to_bf16(float f) {
  uint32_t u = __float_as_uint(f);
  if ((u & 0x7fffffffu) > 0x7f800000u) return (uint16_t)((u >> 16) | 0x40u);  // quiet NaN
  u += 0x7fffu + ((u >> 16) & 1u);
  return (uint16_t)(u >> 16);
}

typedef unsigned int u32x4 __attribute__((ext_vector_type(4)));
typedef float f32x4 __attribute__((ext_vector_type(4)));

template <typename T> struct Elem;
template <> struct Elem<uint16_t> {  // bfloat16 storage
  static constexpr int kVec = 8;     // elements per 16-byte load
  __device__ __forceinline__ static float get(const uint16_t *p) { return bf16_to_f32(*p); }
  __device__ __forceinline__ static uint16_t round(float f) { return f32_to_bf16(f); }
  __device__ __forceinline__ static float value(uint16_t s) { return bf16_to_f32(s); }
};
template <> struct Elem<float> {
  static constexpr int kVec = 4;
  __device__ __forceinline__ static float get(const float *p) { return *p; }
  __device__ __forceinline__ static float round(float f) { return f; }
  __device__ __forceinline__ static float value(float s) { return s; }
};

// VEC consecutive elements starting at p as float32.  VEC > 1 requires p to be
// 16-byte aligned (the host only selects the vector path when it is).
template <typename T, int VEC>
__device__ __forceinline__ void load_vec(const T *__restrict__ p, float (&w)[VEC]) {
  if constexpr (VEC == 1) {
    w[0] = Elem<T>::get(p);
  } else if constexpr (sizeof(T) == 2) {
    static_assert(VEC == 8, "bf16 vector width");
    const u32x4 v = __builtin_nontemporal_load(reinterpret_cast<const u32x4 *>(p));
    const uint32_t q[4] = {v.x, v.y, v.z, v.w};
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      w[2 * i] = __uint_as_float(q[i] << 16);
      w[2 * i + 1] = __uint_as_float(q[i] & 0xffff0000u);
    }
  } else {
    static_assert(VEC == 4, "f32 vector width");
    const f32x4 v = __builtin_nontemporal_load(reinterpret_cast<const f32x4 *>(p));
    w[0] = v.x; w[1] = v.y; w[2] = v.z; w[3] = v.w;
  }
}

// Raw 16-byte loads, unpacked element by element where they are used (keeps
// bf16 data packed in registers).
template <typename T>
__device__ __forceinline__ u32x4 load_raw(const T *__restrict__ p) {
  return __builtin_nontemporal_load(reinterpret_cast<const u32x4 *>(p));
}
template <typename T>
__device__ __forceinline__ float unpack(const u32x4 &q, int v) {
  if constexpr (sizeof(T) == 2) {
    const uint32_t w = q[v >> 1];
    return __uint_as_float((v & 1) ? (w & 0xffff0000u) : (w << 16));
  } else {
    return __uint_as_float(q[v]);
  }
}

// Same for small, reused operands (cached load).
template <typename T, int VEC>
__device__ __forceinline__ void load_vec_cached(const T *__restrict__ p, float (&w)[VEC]) {
  if constexpr (VEC == 1) {
    w[0] = Elem<T>::get(p);
  } else if constexpr (sizeof(T) == 2) {
    const u32x4 v = *reinterpret_cast<const u32x4 *>(p);
    const uint32_t q[4] = {v.x, v.y, v.z, v.w};
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      w[2 * i] = __uint_as_float(q[i] << 16);
      w[2 * i + 1] = __uint_as_float(q[i] & 0xffff0000u);
    }
  } else {
    const f32x4 v = *reinterpret_cast<const f32x4 *>(p);
    w[0] = v.x; w[1] = v.y; w[2] = v.z; w[3] = v.w;
  }
}

__device__ __forceinline__ float silu(float a) { return a / (1.0f + __expf(-a)); }

__device__ __forceinline__ float wave_sum(float v) {
#pragma unroll
  for (int o = 32; o > 0; o >>= 1) v += __shfl_xor(v, o, 64);
  return v;
}

// Cross-workgroup hand-off without cache-wide maintenance.  Partials that
// another workgroup will read are written with device-coherent stores
// (agent-scope atomic stores: written through to the device-coherent level)
// and read back with device-coherent loads, so no L2 writeback or invalidate
// is needed.  arrive_last() waits for this thread's stores to complete,
// counts one arrival of the workgroup and reports whether it was the last of
// `expected`; the last arrival resets the counter for the next launch.
__device__ __forceinline__ void store_coherent(float *p, float v) {
  __hip_atomic_store(p, v, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT);
}
__device__ __forceinline__ float load_coherent(const float *p) {
  return __hip_atomic_load(const_cast<float *>(p), __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT);
}

// sum_{q < n} p[q * stride], added in index order.  The loads are issued 16 at
// a time before any is used (one memory latency per 16 terms instead of one
// per term); addresses past n are clamped in bounds and their values dropped.
__device__ __forceinline__ float sum_coherent(const float *p, size_t stride, int n) {
  float s = 0.0f;
  for (int q0 = 0; q0 < n; q0 += 16) {
    float v[16];
#pragma unroll
    for (int q = 0; q < 16; ++q) v[q] = load_coherent(p + (size_t)min(q0 + q, n - 1) * stride);
#pragma unroll
    for (int q = 0; q < 16; ++q)
      if (q0 + q < n) s += v[q];
  }
  return s;
}

__device__ __forceinline__ bool arrive_last(unsigned *counter, unsigned expected, int *flag_lds) {
  __builtin_amdgcn_s_waitcnt(0);  // this thread's coherent stores have completed
  __atomic_signal_fence(__ATOMIC_SEQ_CST);
  __syncthreads();
  if (threadIdx.x == 0) {
    const unsigned prev = __hip_atomic_fetch_add(counter, 1u, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT);
    const int last = (prev == expected - 1);
    if (last) __hip_atomic_store(counter, 0u, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT);
    *flag_lds = last;
  }
  __syncthreads();
  __atomic_signal_fence(__ATOMIC_SEQ_CST);
  return *flag_lds != 0;
}

}  // namespace sats

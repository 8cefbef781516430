// Norms of queries and keys for each head, the position rotation and the append of
// keys and values to their cache, in one pass over the projections' output (gfx950).
//
//   y = x / sqrt(mean(x^2) + eps) * w                       (where a weight is given)
//   (a, b) -> (a cos - b sin, b cos + a sin)                the pairs of the first rot dims
//
// Both in float32 on registers, rounded once.  A row (a token's head) is held by
// `lanes` lanes, each with V elements and the V that they are rotated with, so that the
// rotation moves nothing between lanes and the mean square is a sum over `lanes` lanes.
//
// Bound by memory where there are tokens: 4096 of 32 + 8 + 8 heads of 128 with norms (bf16,
// 102.8 MB in and out) take 23.2 us, 4.4 TB/s, where a large copy reaches 4.9.  One token is
// the launch: 3.8 us of kernel in 11.2 us of a call from Python.
#pragma once

#include "elem.hpp"
#include "paged.hpp"

namespace sats {

struct RopeArgs {
  const void *q, *k, *v;             // rows of a token at its stride
  int64_t q_stride, k_stride, v_stride;  // elements between tokens
  const void *q_norm, *k_norm;       // [head_dim] or null
  float eps;
  const float *rope;                 // [n_pos][rot]: rot / 2 cosines, rot / 2 sines
  int64_t n_pos;
  const int32_t *positions;          // [n_tokens] or null: the place in the sequence
  void *q_out, *k_out;
  int64_t q_out_stride, k_out_stride;
  int n_q, n_kv, dim, rot, pairs;
  int64_t n_tokens;
  int lanes;                         // lanes of a row, a power of two
  int rows;                          // rows of a token: n_q + n_kv, with a cache + n_kv
  int per;                           // rows of a token that a row of lanes takes
  // the cache (null k_pool: keys go to k_out)
  void *k_pool, *v_pool;             // of the layer
  BatchView batch;
  PoolView pool;
};

// NU: units of 2 V elements that a lane holds (1, or 2 for scalar loads of long rows).
template <typename T, int V, int NU>
__global__ __launch_bounds__(kThreads) void rope_kernel(RopeArgs a) {
  const int lane = threadIdx.x & (a.lanes - 1);
  const int groups = (a.rows + a.per - 1) / a.per;  // rows of lanes per token
  const int64_t slot = ((int64_t)blockIdx.x * kThreads + threadIdx.x) / a.lanes;
  const int64_t t = slot / groups;
  const int first = (int)(slot - t * groups);
  const bool live = t < a.n_tokens;
  // the token's sequence and place (all lanes of a row alike; a wave may hold several tokens)
  int64_t pos = 0, place = 0;
  int seq = 0;
  if (live) {
    if (a.k_pool) place = token_place(a.batch, t, &seq);  // (without a cache there is no batch)
    pos = a.positions ? a.positions[t] : place;
    pos = pos < 0 ? 0 : pos >= a.n_pos ? a.n_pos - 1 : pos;
  }
  int64_t dst_row = -1;  // row of (page, head 0, slot) in the pool
  if (live && a.k_pool) dst_row = pool_row(a.batch, a.pool, seq, place);

  const int units = a.dim / (2 * V), half = a.rot / 2;
  float c[NU][V], s[NU][V];
  int e0[NU], e1[NU];  // first element of each half of a unit
  bool on[NU], turn[NU];
#pragma unroll
  for (int u = 0; u < NU; ++u) {
    const int unit = lane + u * a.lanes;
    on[u] = live && unit < units;
    turn[u] = on[u] && unit * 2 * V < a.rot;
    e0[u] = unit * 2 * V;
    e1[u] = e0[u] + V;
    if (turn[u] && !a.pairs) e0[u] = unit * V, e1[u] = half + unit * V;
    if (turn[u]) {
      const float *row = a.rope + pos * a.rot + unit * V;
      if constexpr (V == 1) {
        c[u][0] = row[0], s[u][0] = row[half];
      } else {
        // V angles of the unit (rot is a multiple of 2 V, so both halves are on 16 bytes)
#pragma unroll
        for (int i = 0; i < V; i += 4) {
          const f32x4 x = *reinterpret_cast<const f32x4 *>(row + i), y = *reinterpret_cast<const f32x4 *>(row + half + i);
#pragma unroll
          for (int j = 0; j < 4; ++j) c[u][i + j] = x[j], s[u][i + j] = y[j];
        }
      }
    }
  }

  for (int r = first; r < a.rows; r += groups) {
    const bool is_q = r < a.n_q, is_v = r >= a.n_q + a.n_kv;
    const int h = is_q ? r : is_v ? r - a.n_q - a.n_kv : r - a.n_q;
    const T *src = is_q ? (const T *)a.q + t * a.q_stride : is_v ? (const T *)a.v + t * a.v_stride
                                                                 : (const T *)a.k + t * a.k_stride;
    src += (int64_t)h * a.dim;
    const T *norm = (const T *)(is_q ? a.q_norm : is_v ? nullptr : a.k_norm);
    float x[NU][V], y[NU][V], wx[NU][V], wy[NU][V];
#pragma unroll
    for (int u = 0; u < NU; ++u) {
#pragma unroll
      for (int i = 0; i < V; ++i) x[u][i] = y[u][i] = 0.0f;
      if (on[u]) {
        load_vec_cached<T, V>(src + e0[u], x[u]);
        load_vec_cached<T, V>(src + e1[u], y[u]);
        if (norm) {
          load_vec_cached<T, V>(norm + e0[u], wx[u]);
          load_vec_cached<T, V>(norm + e1[u], wy[u]);
        }
      }
    }
    if (norm) {
      float ss = 0.0f;
#pragma unroll
      for (int u = 0; u < NU; ++u)
#pragma unroll
        for (int i = 0; i < V; ++i) ss += x[u][i] * x[u][i] + y[u][i] * y[u][i];
      for (int m = a.lanes >> 1; m; m >>= 1) ss += __shfl_xor(ss, m);
      const float f = 1.0f / sqrtf(ss / (float)a.dim + a.eps);
#pragma unroll
      for (int u = 0; u < NU; ++u)
#pragma unroll
        for (int i = 0; i < V; ++i)
          if (on[u]) x[u][i] *= f * wx[u][i], y[u][i] *= f * wy[u][i];
    }
    T *dst = nullptr;
    if (live) {
      if (is_q) dst = (T *)a.q_out + t * a.q_out_stride + (int64_t)h * a.dim;
      else if (!a.k_pool) dst = (T *)a.k_out + t * a.k_out_stride + (int64_t)h * a.dim;
      else if (dst_row >= 0) dst = (T *)(is_v ? a.v_pool : a.k_pool) + (dst_row + (int64_t)h * a.pool.page) * a.dim;
    }
#pragma unroll
    for (int u = 0; u < NU; ++u) {
      if (!on[u] || !dst) continue;
      T o0[V], o1[V];
      if (turn[u] && !is_v) {
        if (!a.pairs) {
#pragma unroll
          for (int i = 0; i < V; ++i) {
            const float p = x[u][i], q = y[u][i];
            x[u][i] = p * c[u][i] - q * s[u][i];
            y[u][i] = q * c[u][i] + p * s[u][i];
          }
        } else if constexpr (V == 1) {
          const float p = x[u][0], q = y[u][0];
          x[u][0] = p * c[u][0] - q * s[u][0];
          y[u][0] = q * c[u][0] + p * s[u][0];
        } else {
#pragma unroll
          for (int i = 0; i < V / 2; ++i) {
            const float p = x[u][2 * i], q = x[u][2 * i + 1];
            x[u][2 * i] = p * c[u][i] - q * s[u][i];
            x[u][2 * i + 1] = q * c[u][i] + p * s[u][i];
            const float p2 = y[u][2 * i], q2 = y[u][2 * i + 1];
            y[u][2 * i] = p2 * c[u][V / 2 + i] - q2 * s[u][V / 2 + i];
            y[u][2 * i + 1] = q2 * c[u][V / 2 + i] + p2 * s[u][V / 2 + i];
          }
        }
      }
#pragma unroll
      for (int i = 0; i < V; ++i) o0[i] = Elem<T>::round(x[u][i]), o1[i] = Elem<T>::round(y[u][i]);
      store_vec<T, V>(dst + e0[u], o0);
      store_vec<T, V>(dst + e1[u], o1);
    }
  }
}

}  // namespace sats

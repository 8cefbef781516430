// Attention of new tokens over the paged cache (gfx950).
//
//   o = sum_j p_j v_j,  p = softmax over the visible keys of scale (q . k_j)
//
// A token at place i of its sequence sees the keys j <= i with i - j < window or
// j < sinks (window 0: all of them); keys whose page is absent are not seen.
// Running maximum and sum over one pass of the keys, float32.
#pragma once

#include "paged.hpp"

namespace sats {

struct AttendArgs {
  const void *q;
  int64_t q_stride;
  const void *k, *v;  // of the layer
  void *out;
  float *lse;         // or null
  BatchView batch;
  PoolView pool;
  int n_q, dim;
  float scale;
  int64_t window, sinks;
};

// One wave per (token, head).
template <typename T>
__global__ __launch_bounds__(64) void attend_simple_kernel(AttendArgs a) {
  const int64_t t = blockIdx.x;
  const int h = blockIdx.y, lane = threadIdx.x, kvh = h / (a.n_q / a.pool.n_kv);
  int seq;
  const int64_t place = token_place(a.batch, t, &seq);
  const SeqView sv = seq_view(a.batch, a.pool, seq);
  const T *q = (const T *)a.q + t * a.q_stride + (int64_t)h * a.dim;
  const int64_t last = place < sv.len - 1 ? place : sv.len - 1;
  float m = -INFINITY, l = 0.0f, acc[4] = {};
  for (int64_t j = 0; j <= last; ++j) {
    if (a.window && place - j >= a.window && j >= a.sinks) continue;
    const int64_t row = pool_row(a.batch, a.pool, seq, j);
    if (row < 0) continue;
    const int64_t at = (row + (int64_t)kvh * a.pool.page) * a.dim;
    float s = 0.0f;
    for (int d = lane; d < a.dim; d += 64) s += Elem<T>::get(q + d) * Elem<T>::get((const T *)a.k + at + d);
    for (int x = 32; x; x >>= 1) s += __shfl_xor(s, x);
    s *= a.scale;
    const float mn = fmaxf(m, s), at0 = mn == -INFINITY ? 0.0f : mn, f = expf(m - at0), p = expf(s - at0);
    l = l * f + p;
    m = mn;
    for (int d = lane, i = 0; d < a.dim; d += 64, ++i) acc[i] = acc[i] * f + p * Elem<T>::get((const T *)a.v + at + d);
  }
  T *o = (T *)a.out + (t * a.n_q + h) * a.dim;
  for (int d = lane, i = 0; d < a.dim; d += 64, ++i) o[d] = Elem<T>::round(l == 0.0f ? 0.0f : acc[i] / l);
  if (a.lse && lane == 0) a.lse[t * a.n_q + h] = l == 0.0f ? -INFINITY : m + logf(l);
}

}  // namespace sats

// Rules on logits ahead of sampling (gfx950): penalties for the ids so far, biases, grammar masks.
//
//   l <- l / r or l r (l > 0 or not)           where the id has come so far (prompt or answer)
//   l <- l - f count - p [count > 0]           count: how often it has come in the answer
//   l <- l + sum of the id's biases            in their order
//   l <- -inf                                  where the row's mask has no bit for it
//
// A workgroup takes kLogitChunk ids of a row: it counts, in LDS, those of the ids so far that are its
// own, adds up its biases there, and then passes once over its logits.  The counts are whole numbers,
// so the order of the atomic additions does not show; biases are added a batch at a time, of several for
// one id the earliest first.  Every workgroup of a row reads all of its ids so far (32 times at 128256 ids): 4 bytes
// each from the caches, where sorting them into chunks would be a launch of its own.  Penalties alone on 64 x 128256 (float32),
// us by the ids so far of each row: 1 16.1, 1000 17.2, 8000 26.4, 32000 44.6, 128000 129 (1 GB of reads); on one row 4.7, 5.2, 8.7,
// 15.5, 44.9.
//
// 64 rows of 128256 (float32, 66 MB in and out) with histories of up to 8000, up to 300 biases and masks take 23.6 us,
// 2.8 TB/s, where a copy's rate would be 13.6; without any rule 16.5, with histories and masks 18.9: a workgroup's
// steps (lengths, ids, counts, biases) wait for each other.  Listing the ids that are met, and writing these anew
// after a pass of the mask alone, takes 30.5; chunks of 2048 ids or 512 threads take as long.
// In place the same rules take 26.9: what is changed is read after its rule is known, not ahead of it.  Where few logits are
// changed that pays: penalties of one id a row 8.4 instead of 16.1, of histories as above alone 14.5 instead of 18.6.
#pragma once

#include "elem.hpp"

namespace sats {

constexpr int kLogitChunk = 4096, kLogitThreads = 256, kLogitOwners = 1024;
constexpr uint32_t kToldBit = 0x80000000u;  // of a count: the id has come

struct LogitArgs {
  const void *logits;
  void *out;
  int64_t stride, out_stride, vocab;
  const int32_t *seqs, *history, *history_len, *prompt_len;
  int64_t n_seqs, history_stride, max_history;
  const float *repetition, *frequency, *presence;
  const int32_t *bias_start, *bias_ids;
  const float *bias;
  int64_t n_bias;
  const uint32_t *masks;
  const int32_t *mask_of;
  int64_t n_masks, mask_stride;
  int in_place;  // out is logits: a step (of V) that no rule changes is neither read nor written
};

// Adds this thread's bias (live: it has one, of id `at` of the chunk) to those of the chunk: in rounds, in
// each of which the lowest thread of each owner slot adds its own.
__device__ __forceinline__ void add_biases(float *bias, unsigned *owner, bool live, int at, float v) {
  const int slot = at & (kLogitOwners - 1);
  while (__syncthreads_or(live)) {
    if (live) atomicMin(owner + slot, threadIdx.x);
    __syncthreads();
    if (live && owner[slot] == threadIdx.x) {
      bias[at] += v;
      owner[slot] = 0xffffffffu;  // (a slot's other threads see that they are not it either way)
      live = false;
    }
  }
}

// The first `left` of V logits from p on (V > 1: on 16 bytes where all are there).
template <typename T, int V> __device__ __forceinline__ void load_logits(const T *p, int left, float (&x)[V]) {
  constexpr int kAtOnce = V == 1 ? 1 : 16 / (int)sizeof(T);
  if (V == 1 || left >= V) {
#pragma unroll
    for (int j = 0; j < V; j += kAtOnce) {
      float w[kAtOnce];
      load_vec<T, kAtOnce>(p + j, w);
#pragma unroll
      for (int k = 0; k < kAtOnce; ++k) x[j + k] = w[k];
    }
  } else {
#pragma unroll
    for (int j = 0; j < V; ++j) x[j] = j < left ? Elem<T>::get(p + j) : 0.0f;
  }
}

// V: logits of a thread's step (8, rows on 16 bytes; or 1).
template <typename T, typename O, int V>
__global__ __launch_bounds__(kLogitThreads) void logits_kernel(LogitArgs a) {
  extern __shared__ __align__(16) uint32_t lds[];
  __shared__ unsigned owner[kLogitOwners];
  const int64_t row = blockIdx.y, c0 = (int64_t)blockIdx.x * kLogitChunk;
  const int n = (int)(a.vocab - c0 < kLogitChunk ? a.vocab - c0 : kLogitChunk), tid = threadIdx.x;
  uint32_t *count = lds;
  float *bias = reinterpret_cast<float *>(lds + (a.history ? kLogitChunk : 0));

  const T *src = (const T *)a.logits + row * a.stride + c0;
  // the logits of this thread's steps, on their way while the rules are gathered (in place few are read)
  constexpr int kSteps = kLogitChunk / (kLogitThreads * V);
  float held[V > 1 ? kSteps : 1][V];
  if constexpr (V > 1) {
    if (!a.in_place)
#pragma unroll
      for (int s = 0; s < kSteps; ++s) {
        const int i = (s * kLogitThreads + tid) * V;
        if (i < n) load_logits<T, V>(src + i, n - i, held[s]);
      }
  }

  const int64_t seq = a.seqs ? a.seqs[row] : row;
  const bool known = a.history && seq >= 0 && seq < a.n_seqs;
  int64_t told = known ? a.history_len[seq] : 0;
  told = told < 0 ? 0 : told > a.max_history ? a.max_history : told;
  int64_t b0 = 0, b1 = 0;
  if (a.bias) {
    b0 = a.bias_start[row], b1 = a.bias_start[row + 1];
    b0 = b0 < 0 ? 0 : b0;
    b1 = b1 > a.n_bias ? a.n_bias : b1;
  }
  const uint32_t *mask = nullptr;
  if (a.masks) {
    const int64_t m = a.mask_of ? a.mask_of[row] : row;
    if (m >= 0 && m < a.n_masks) mask = a.masks + m * a.mask_stride;
  }
  if (told > 0)
    for (int i = tid * 4; i < kLogitChunk; i += kLogitThreads * 4) *reinterpret_cast<u32x4 *>(count + i) = u32x4{0, 0, 0, 0};
  if (b1 > b0) {
    for (int i = tid * 4; i < kLogitChunk; i += kLogitThreads * 4) *reinterpret_cast<u32x4 *>(bias + i) = u32x4{0, 0, 0, 0};
    for (int i = tid; i < kLogitOwners; i += kLogitThreads) owner[i] = 0xffffffffu;
  }
  __syncthreads();
  if (told > 0) {
    const int32_t *ids = a.history + seq * a.history_stride;
    const int64_t prompt = a.prompt_len ? a.prompt_len[seq] : 0;
    auto tell = [&](int id, int64_t at) {
      const int64_t x = (int64_t)id - c0;
      if (x < 0 || x >= n) return;
      if (at < prompt) atomicOr(count + x, kToldBit);
      else atomicAdd(count + x, 1u);
    };
    const int64_t whole = ((uintptr_t)ids & 15) == 0 ? told & ~(int64_t)3 : 0;
#pragma unroll 4
    for (int64_t i = tid * 4; i < whole; i += kLogitThreads * 4) {
      const u32x4 v = *reinterpret_cast<const u32x4 *>(ids + i);
#pragma unroll
      for (int j = 0; j < 4; ++j) tell((int)v[j], i + j);
    }
    for (int64_t i = whole + tid; i < told; i += kLogitThreads) tell(ids[i], i);
  }
  for (int64_t b = b0; b < b1; b += kLogitThreads) {
    const int64_t i = b + tid, x = i < b1 ? a.bias_ids[i] - c0 : -1;
    const bool live = x >= 0 && x < n;
    add_biases(bias, owner, live, live ? (int)x : 0, live ? a.bias[i] : 0.0f);
  }
  __syncthreads();

  const float r = a.repetition ? a.repetition[row] : 1.0f, f = a.frequency ? a.frequency[row] : 0.0f;
  const float p = a.presence ? a.presence[row] : 0.0f;
  O *dst = (O *)a.out + row * a.out_stride + c0;
#pragma unroll(V > 1 ? kSteps : 1)
  for (int s = 0; s < kSteps; ++s) {
    const int i = (s * kLogitThreads + tid) * V;
    if (i >= n) break;
    const int m = V > 1 && n - i < V ? n - i : V;
    uint32_t c[V], on = (1u << V) - 1;
    float add[V];
    bool same = true;
#pragma unroll
    for (int j = 0; j < V; ++j) c[j] = told > 0 ? count[i + j] : 0, add[j] = b1 > b0 ? bias[i + j] : 0.0f;
    if (mask) on &= mask[(c0 + i) >> 5] >> (i & 31);
    if (a.in_place) {
#pragma unroll
      for (int j = 0; j < V; ++j) same &= j >= m || (!c[j] && add[j] == 0.0f && (on >> j & 1));
      if (same) continue;
    }
    float x[V];
    if (V > 1 && !a.in_place) {
#pragma unroll
      for (int j = 0; j < V; ++j) x[j] = held[V > 1 ? s : 0][j];
    } else {
      load_logits<T, V>(src + i, n - i, x);
    }
#pragma unroll
    for (int j = 0; j < V; ++j) {
      if (c[j]) {
        x[j] = x[j] > 0.0f ? x[j] / r : x[j] * r;
        const uint32_t k = c[j] & ~kToldBit;
        if (k) x[j] = x[j] - f * (float)k - p;
      }
      if (add[j] != 0.0f) x[j] += add[j];
      if (!(on >> j & 1)) x[j] = -INFINITY;
    }
    O o[V];
#pragma unroll
    for (int j = 0; j < V; ++j) o[j] = Elem<O>::round(x[j]);
    if (V > 1 && m == V) {
#pragma unroll
      for (int j = 0; j < V * (int)sizeof(O) / 16; ++j) {
        u32x4 w;
        __builtin_memcpy(&w, reinterpret_cast<const char *>(o) + 16 * j, 16);
        reinterpret_cast<u32x4 *>(dst + i)[j] = w;
      }
    } else {
#pragma unroll
      for (int j = 0; j < V; ++j)
        if (j < m) dst[i + j] = o[j];
    }
  }
}

}  // namespace sats

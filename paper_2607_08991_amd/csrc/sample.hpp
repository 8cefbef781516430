// Sampling of the next id from logits (gfx950): temperature, then the top k, then the top
// p of what is left, then a least share of the largest probability, and a draw from
// what remains with one given number of [0, 1) a row.
//
// The weight of id i is the integer w_i = round(2^40 exp((l_i - max) / T)) (the
// difference, its product with 1 / T and the exponential in float32).  Sums of these are
// exact in 64 bits whatever their order, so which ids are kept and which one is drawn do
// not depend on how a row is split; ids of weight 0 are never kept.  In the order of
// falling logit, the lower id first where two are equal, an id is kept while
//   its rank is below k, the weights before it are below p times those of the top k
//   (in float64), and exp(..) >= min_p,
// and the first one always; the id drawn is the first, in the order of ids, whose
// running sum of kept weights exceeds u times their total.
//
// Nothing is sorted.  Four launches, each over chunks of the rows but the last:
//   max     the row's largest logit;
//   hist    weights and counts by bins of (max - l) / T, where k or p ask for it;
//   cut     the bins in which k and p can end: their ids go to a list, the weights of
//           the bins before them to a sum per chunk;
//   pick    a workgroup per row: k and p end at an element of the list, found by its
//           (logit, id) key 8 bits at a time; then the chunk, then the id, of the draw.
#pragma once

#include "elem.hpp"
#include "paged.hpp"

namespace sats {

constexpr int kSampChunk = 4096;  // ids of a chunk
constexpr int kSampBins = 2048;
constexpr float kSampScale = 70.0f;   // bins per unit of (max - l) / T: weights past bin 2047 round to 0
constexpr int kPickThreads = 1024;
typedef unsigned long long u64;

struct SampleArgs {
  const void *logits;
  int64_t stride, vocab;
  int n, chunks;
  const float *temperature, *top_p, *min_p, *u;
  const int32_t *top_k;
  int32_t *tokens, *n_kept;
  float *prob;
  // scratch, per row
  float *cmax;        // [n][chunks] largest logit
  int32_t *cid;       // [n][chunks] its lowest id
  u64 *hsum;          // [n][kSampBins]
  uint32_t *hcnt;     // [n][kSampBins]
  u64 *csum;          // [n][chunks] weights kept for certain
  uint32_t *ccnt;     // [n][chunks] ... and how many
  u64 *list;          // [n][vocab] keys of the ids to look at
  uint32_t *n_list;   // [n]
};

// What a row asks for.
struct RowRule {
  bool first;     // the largest logit alone
  bool cut;       // k or p may end the kept ids
  float inv_t, min_p;
  int64_t k;
  double p;
};
__device__ __forceinline__ RowRule row_rule(const SampleArgs &a, int r) {
  RowRule q;
  const float t = a.temperature ? a.temperature[r] : 1.0f;
  const int32_t k = a.top_k ? a.top_k[r] : 0;
  const float p = a.top_p ? a.top_p[r] : 1.0f;
  q.min_p = a.min_p ? a.min_p[r] : 0.0f;
  q.first = !(t > 0.0f) || k == 1 || !(p > 0.0f) || !(q.min_p <= 1.0f);
  q.inv_t = 1.0f / t;
  q.k = k > 0 && k < a.vocab ? k : a.vocab;
  q.p = p < 1.0f ? (double)p : 1.0;
  q.cut = !q.first && (q.k < a.vocab || q.p < 1.0);
  return q;
}

__device__ __forceinline__ float logit_of(const SampleArgs &a, float v) { return v == v ? v : -INFINITY; }

// exp((x - max) / T), 0 for what can have no weight.
__device__ __forceinline__ float share_of(float x, float top, float inv_t, float *z) {
  const float d = x == top ? 0.0f : (x - top) * inv_t;
  *z = d;
  return d > -30.0f ? expf(d) : 0.0f;
}
__device__ __forceinline__ u64 weight_of(float share) { return (u64)rintf(share * 1099511627776.0f); }
__device__ __forceinline__ int bin_of(float z) {
  const int b = (int)(-z * kSampScale);
  return b < kSampBins - 1 ? b : kSampBins - 1;
}
// Ascending keys: falling logit, then rising id.
__device__ __forceinline__ u64 key_of(float x, uint32_t id) {
  const uint32_t b = __float_as_uint(x + 0.0f);  // (-0 and 0 are equal)
  const uint32_t up = b & 0x80000000u ? ~b : b | 0x80000000u;
  return (u64)~up << 32 | id;
}

__device__ __forceinline__ u64 wave_sum(u64 v) {
#pragma unroll
  for (int d = 32; d; d >>= 1) v += __shfl_xor(v, d);
  return v;
}

// Largest logit of a row from its chunks, and its lowest id (any wave, all lanes).
__device__ __forceinline__ float row_max(const SampleArgs &a, int r, int32_t *id) {
  float m = -INFINITY;
  int32_t at = 0x7fffffff;
  for (int c = threadIdx.x & 63; c < a.chunks; c += 64) {
    const float x = a.cmax[(int64_t)r * a.chunks + c];
    if (x > m) m = x, at = a.cid[(int64_t)r * a.chunks + c];
  }
#pragma unroll
  for (int d = 32; d; d >>= 1) {
    const float x = __shfl_xor(m, d);
    const int32_t y = __shfl_xor(at, d);
    if (x > m || (x == m && y < at)) m = x, at = y;
  }
  *id = at;
  return m;
}

// Calls f(logit, id) for this thread's ids of a chunk, 256 threads, V consecutive ids at a time.
template <typename T, int V, typename F>
__device__ __forceinline__ void for_chunk(const SampleArgs &a, int r, int chunk, F f) {
  const T *row = (const T *)a.logits + (int64_t)r * a.stride;
  const int64_t lo = (int64_t)chunk * kSampChunk, hi = lo + kSampChunk < a.vocab ? lo + kSampChunk : a.vocab;
#pragma unroll
  for (int step = 0; step < kSampChunk / (kThreads * V); ++step) {
    const int64_t i = lo + (step * kThreads + (int)threadIdx.x) * V;
    if (i + V <= hi) {
      float x[V];
      load_vec_cached<T, V>(row + i, x);
#pragma unroll
      for (int j = 0; j < V; ++j) f(logit_of(a, x[j]), (uint32_t)(i + j));
    } else {
      for (int j = 0; j < V; ++j)
        if (i + j < hi) f(logit_of(a, Elem<T>::get(row + i + j)), (uint32_t)(i + j));
    }
  }
}

template <typename T, int V>
__global__ __launch_bounds__(kThreads) void sample_max_kernel(SampleArgs a) {
  __shared__ float sm[4];
  __shared__ int32_t si[4];
  const int chunk = blockIdx.x, r = blockIdx.y;
  for (int b = chunk * kThreads + threadIdx.x; b < kSampBins; b += a.chunks * kThreads)
    a.hsum[(int64_t)r * kSampBins + b] = 0, a.hcnt[(int64_t)r * kSampBins + b] = 0;
  if (chunk == 0 && threadIdx.x == 0) a.n_list[r] = 0;
  float m = -INFINITY;
  uint32_t at = 0x7fffffff;
  for_chunk<T, V>(a, r, chunk, [&](float x, uint32_t i) {
    if (x > m) m = x, at = i;  // (a thread's ids rise)
  });
#pragma unroll
  for (int d = 32; d; d >>= 1) {
    const float x = __shfl_xor(m, d);
    const uint32_t y = __shfl_xor(at, d);
    if (x > m || (x == m && y < at)) m = x, at = y;
  }
  if ((threadIdx.x & 63) == 0) sm[threadIdx.x >> 6] = m, si[threadIdx.x >> 6] = (int32_t)at;
  __syncthreads();
  if (threadIdx.x == 0) {
    for (int w = 1; w < 4; ++w)
      if (sm[w] > m || (sm[w] == m && (uint32_t)si[w] < at)) m = sm[w], at = (uint32_t)si[w];
    a.cmax[(int64_t)r * a.chunks + chunk] = m;
    a.cid[(int64_t)r * a.chunks + chunk] = (int32_t)at;
  }
}

template <typename T, int V>
__global__ __launch_bounds__(kThreads) void sample_hist_kernel(SampleArgs a) {
  __shared__ u64 hs[kSampBins];
  __shared__ uint32_t hc[kSampBins];
  const int chunk = blockIdx.x, r = blockIdx.y;
  const RowRule q = row_rule(a, r);
  if (!q.cut) return;
  int32_t id;
  const float top = row_max(a, r, &id);
  for (int b = threadIdx.x; b < kSampBins; b += kThreads) hs[b] = 0, hc[b] = 0;
  __syncthreads();
  for_chunk<T, V>(a, r, chunk, [&](float x, uint32_t) {
    float z;
    const u64 w = weight_of(share_of(x, top, q.inv_t, &z));
    if (w) {
      const int b = bin_of(z);
      atomicAdd(&hs[b], w);
      atomicAdd(&hc[b], 1u);
    }
  });
  __syncthreads();
  for (int b = threadIdx.x; b < kSampBins; b += kThreads)
    if (hc[b]) {
      atomicAdd(&a.hsum[(int64_t)r * kSampBins + b], hs[b]);
      atomicAdd(&a.hcnt[(int64_t)r * kSampBins + b], hc[b]);
    }
}

// Where k and p can end, from a row's bins.
struct RowCut {
  int k_bin;          // bin that holds the last of the top k (kSampBins: all are in)
  u64 k_before;       // weights of the bins before it
  int64_t k_left;     // ids of that bin that are among the top k
  int p_lo, p_hi;     // bins in which p can end
  u64 p_before;       // weights of the bins before p_lo
};

// Prefix sums of the bins by 256 threads (8 bins each); lds: 8 words.
__device__ __forceinline__ RowCut row_cut(const SampleArgs &a, int r, const RowRule &q, u64 *lds_s, uint32_t *lds_c,
                                          RowCut *out) {
  constexpr int kPer = kSampBins / kThreads;
  const u64 *hs = a.hsum + (int64_t)r * kSampBins;
  const uint32_t *hc = a.hcnt + (int64_t)r * kSampBins;
  u64 s[kPer], inc_s = 0;
  uint32_t c[kPer], inc_c = 0;
  const int tid = threadIdx.x, lane = tid & 63, wave = tid >> 6;
  if (tid < kThreads) {
#pragma unroll
    for (int i = 0; i < kPer; ++i) s[i] = hs[tid * kPer + i], c[i] = hc[tid * kPer + i], inc_s += s[i], inc_c += c[i];
  }
  const u64 own_s = inc_s;
  const uint32_t own_c = inc_c;
#pragma unroll
  for (int d = 1; d < 64; d <<= 1) {
    const u64 o = __shfl_up(inc_s, d);
    const uint32_t oc = __shfl_up(inc_c, d);
    if (lane >= d) inc_s += o, inc_c += oc;
  }
  if (tid < kThreads && lane == 63) lds_s[wave] = inc_s, lds_c[wave] = inc_c;
  if (tid == 0) out->k_bin = kSampBins, out->k_left = 0, out->p_lo = out->p_hi = kSampBins - 1;
  __syncthreads();
  u64 bs = 0, total = 0;
  uint32_t bc = 0, count = 0;
#pragma unroll
  for (int w = 0; w < kThreads / 64; ++w) {
    if (w < wave) bs += lds_s[w], bc += lds_c[w];
    total += lds_s[w], count += lds_c[w];
  }
  const u64 s0 = bs + inc_s - own_s;
  const uint32_t c0 = bc + inc_c - own_c;
  if (tid == 0) out->k_before = total;
  __syncthreads();
  if (tid < kThreads && q.k < (int64_t)count) {
    u64 x = s0;
    int64_t y = c0;
#pragma unroll
    for (int i = 0; i < kPer; ++i) {
      if (y < q.k && q.k <= y + c[i]) out->k_bin = tid * kPer + i, out->k_before = x, out->k_left = q.k - y;
      x += s[i], y += c[i];
    }
  }
  __syncthreads();
  const int kb = out->k_bin;
  const u64 low = out->k_before;  // the top k weigh at least this much, at most that of their last bin more
  u64 high = low;
  if (kb < kSampBins) high += hs[kb];
  if (tid < kThreads) {
    // p ends in the last bin with ids whose weights before are below p * (weight of the top k):
    // the first candidates are in that bin for `low` (or later), the last in that for `high`
    u64 x = s0;
    const double dl = q.p * (double)low, dh = q.p * (double)high;
#pragma unroll
    for (int i = 0; i < kPer; ++i) {
      if (c[i]) {
        const double before = (double)x, after = (double)(x + s[i]);
        if (before < dl && !(after < dl)) out->p_lo = tid * kPer + i;
        if (before < dh && !(after < dh)) out->p_hi = tid * kPer + i;
      }
      if (tid == 0 && i == 0 && !(dl > 0.0)) out->p_lo = 0;
      x += s[i];
    }
  }
  __syncthreads();
  {
    u64 x = s0;
    if (tid < kThreads) {
#pragma unroll
      for (int i = 0; i < kPer; ++i) {
        if (tid * kPer + i == out->p_lo) out->p_before = x;
        x += s[i];
      }
    }
  }
  __syncthreads();
  return *out;
}

template <typename T, int V>
__global__ __launch_bounds__(kThreads) void sample_cut_kernel(SampleArgs a) {
  __shared__ u64 ls[4];
  __shared__ uint32_t lc[4];
  __shared__ RowCut cut_lds;
  const int chunk = blockIdx.x, r = blockIdx.y;
  const RowRule q = row_rule(a, r);
  if (q.first) return;
  int32_t id;
  const float top = row_max(a, r, &id);
  RowCut cut;
  cut.p_lo = kSampBins, cut.p_hi = -1, cut.k_bin = -1;
  if (q.cut) cut = row_cut(a, r, q, ls, lc, &cut_lds);
  u64 sum = 0;
  uint32_t cnt = 0;
  u64 *list = a.list + (int64_t)r * a.vocab;
  for_chunk<T, V>(a, r, chunk, [&](float x, uint32_t i) {
    float z;
    const float share = share_of(x, top, q.inv_t, &z);
    const u64 w = weight_of(share);
    if (!w) return;
    const int b = bin_of(z);
    if (b < cut.p_lo && b != cut.k_bin) {
      if (share >= q.min_p) sum += w, ++cnt;
    } else if (b <= cut.p_hi || b == cut.k_bin) {
      list[atomicAdd(&a.n_list[r], 1u)] = key_of(x, i);
    }
  });
  sum = wave_sum(sum);
  const u64 c = wave_sum((u64)cnt);
  __syncthreads();
  if ((threadIdx.x & 63) == 0) ls[threadIdx.x >> 6] = sum, lc[threadIdx.x >> 6] = (uint32_t)c;
  __syncthreads();
  if (threadIdx.x == 0) {
    a.csum[(int64_t)r * a.chunks + chunk] = ls[0] + ls[1] + ls[2] + ls[3];
    a.ccnt[(int64_t)r * a.chunks + chunk] = lc[0] + lc[1] + lc[2] + lc[3];
  }
}

constexpr int kPickList = 4096;  // keys of the list that are held in LDS

struct PickLds {
  u64 sum[256];
  uint32_t cnt[256];
  u64 key_and, key_or, base, weight, found;
  int64_t left;
  uint32_t one;
  u64 scan_s[kPickThreads / 64];
  uint32_t scan_c[kPickThreads / 64];
  u64 chunk[kPickThreads];
  RowCut cut;
  u64 keys[kPickList];
};

// Exclusive prefix of one u64 per thread over the workgroup; *total its sum.
__device__ __forceinline__ u64 pick_scan(u64 v, u64 *lds, u64 *total) {
  const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
  u64 inc = v;
#pragma unroll
  for (int d = 1; d < 64; d <<= 1) {
    const u64 o = __shfl_up(inc, d);
    if (lane >= d) inc += o;
  }
  __syncthreads();
  if (lane == 63) lds[wave] = inc;
  __syncthreads();
  u64 base = 0, sum = 0;
  for (int w = 0; w < kPickThreads / 64; ++w) {
    if (w < wave) base += lds[w];
    sum += lds[w];
  }
  *total = sum;
  return base + inc - v;
}

// The key, among those of the list in bins [lo, hi], at which the kept ids end: the
// `left`-th smallest (BY_COUNT), or the last one whose weights before it, from `base` on,
// are below `limit`.  Each step splits the keys that are left by the 8 highest bits in
// which they differ and goes on with one part.  *upto: base and the weights up to it.
template <bool BY_COUNT>
__device__ u64 pick_end(const u64 *list, uint32_t n, int lo, int hi, float top, float inv_t, int64_t left, u64 base,
                        double limit, PickLds &l, u64 *upto) {
  u64 fixed = 0, value = 0;  // bits that are decided, and what they are
  const int tid = threadIdx.x;
  for (;;) {
    __syncthreads();
    if (tid < 256) l.sum[tid] = 0, l.cnt[tid] = 0;
    if (tid == 0) l.key_and = ~0ull, l.key_or = 0;
    __syncthreads();
    u64 ka = ~0ull, ko = 0;
    auto each = [&](auto f) {
      for (uint32_t i = tid; i < n; i += kPickThreads) {
        const u64 key = list[i];
        if ((key & fixed) != value) continue;
        const uint32_t up = ~(uint32_t)(key >> 32);
        const float x = __uint_as_float(up & 0x80000000u ? up & 0x7fffffffu : ~up);
        float z;
        const u64 w = weight_of(share_of(x, top, inv_t, &z));
        const int b = bin_of(z);
        if (b >= lo && b <= hi) f(key, w);
      }
    };
    each([&](u64 key, u64) { ka &= key, ko |= key; });
#pragma unroll
    for (int d = 32; d; d >>= 1) ka &= __shfl_xor(ka, d), ko |= __shfl_xor(ko, d);
    if ((tid & 63) == 0 && ko) atomicAnd(&l.key_and, ka), atomicOr(&l.key_or, ko);
    __syncthreads();
    const u64 diff = l.key_and ^ l.key_or;
    const int high = diff ? 63 - __clzll((long long)diff) : 7, shift = high > 7 ? high - 7 : 0;
    each([&](u64 key, u64 w) {
      const int b = (int)(key >> shift) & 255;
      atomicAdd(&l.sum[b], w);
      atomicAdd(&l.cnt[b], 1u);
    });
    __syncthreads();
    if (tid < 64) {  // four parts a lane
      u64 s[4], inc = 0;
      uint32_t c[4], incc = 0;
#pragma unroll
      for (int i = 0; i < 4; ++i) s[i] = l.sum[4 * tid + i], c[i] = l.cnt[4 * tid + i], inc += s[i], incc += c[i];
      const u64 own = inc;
      const uint32_t ownc = incc;
#pragma unroll
      for (int d = 1; d < 64; d <<= 1) {
        const u64 o = __shfl_up(inc, d);
        const uint32_t oc = __shfl_up(incc, d);
        if (tid >= d) inc += o, incc += oc;
      }
      u64 before = base + inc - own, at = 0;
      int64_t cb = (int64_t)(incc - ownc), cat = 0;
      int part = -1;
      uint32_t size = 0;
#pragma unroll
      for (int i = 0; i < 4; ++i) {
        if (c[i] && (BY_COUNT ? cb < left : (double)before < limit)) part = 4 * tid + i, at = before, cat = cb, size = c[i];
        before += s[i], cb += c[i];
      }
      const u64 any = __ballot(part >= 0);
      const int winner = any ? 63 - __clzll((long long)any) : -1;
      if (tid == winner) l.found = (u64)part, l.base = at, l.left = cat, l.one = size;
      if (winner < 0 && tid == 0) l.found = 0, l.base = base, l.left = 0, l.one = 0;
    }
    __syncthreads();
    const u64 mask = 255ull << shift;
    // (bits above `high` are common to the keys that are left)
    const u64 above = shift + 8 < 64 ? ~0ull << (shift + 8) : 0;
    fixed = above | mask;
    value = (l.key_and & above) | l.found << shift;
    base = l.base;
    left -= l.left;
    const uint32_t size = l.one;
    if (size <= 1 || shift == 0) break;
  }
  // the one key that is left (all bits are decided where shift reached 0)
  __syncthreads();
  if (tid == 0) l.found = 0, l.weight = 0;
  __syncthreads();
  for (uint32_t i = tid; i < n; i += kPickThreads) {
    const u64 key = list[i];
    if ((key & fixed) != value) continue;
    const uint32_t up = ~(uint32_t)(key >> 32);
    const float x = __uint_as_float(up & 0x80000000u ? up & 0x7fffffffu : ~up);
    float z;
    const u64 w = weight_of(share_of(x, top, inv_t, &z));
    const int b = bin_of(z);
    if (b >= lo && b <= hi) l.found = key, l.weight = w;
  }
  __syncthreads();
  *upto = base + l.weight;
  return l.found;
}

template <typename T>
__global__ __launch_bounds__(kPickThreads) void sample_pick_kernel(SampleArgs a) {
  __shared__ PickLds l;
  const int r = blockIdx.x, tid = threadIdx.x;
  const RowRule q = row_rule(a, r);
  int32_t id;
  const float top = row_max(a, r, &id);
  if (q.first || !(top > -INFINITY)) {
    const bool some = top > -INFINITY;
    if (tid == 0) {
      a.tokens[r] = some ? id : -1;
      if (a.prob) a.prob[r] = some ? 1.0f : 0.0f;
      if (a.n_kept) a.n_kept[r] = some;
    }
    return;
  }
  u64 last = ~0ull;
  const u64 *list = a.list + (int64_t)r * a.vocab;
  uint32_t n = 0;
  if (q.cut) {
    const RowCut cut = row_cut(a, r, q, l.scan_s, l.scan_c, &l.cut);
    n = a.n_list[r];
    if (n <= kPickList) {
      for (uint32_t i = tid; i < n; i += kPickThreads) l.keys[i] = list[i];
      list = l.keys;
    }
    u64 all = cut.k_before, unused;
    if (cut.k_bin < kSampBins)
      (void)pick_end<true>(list, n, cut.k_bin, cut.k_bin, top, q.inv_t, cut.k_left, cut.k_before, 0.0, l, &all);
    last = pick_end<false>(list, n, cut.p_lo, cut.p_hi, top, q.inv_t, 0, cut.p_before, q.p * (double)all, l, &unused);
  }
  // weights and counts of each chunk
  __syncthreads();
  u64 kept = 0;
  if (tid < a.chunks) l.chunk[tid] = a.csum[(int64_t)r * a.chunks + tid], kept = a.ccnt[(int64_t)r * a.chunks + tid];
  __syncthreads();
  for (uint32_t i = tid; i < n; i += kPickThreads) {
    const u64 key = list[i];
    if (key > last) continue;
    const uint32_t up = ~(uint32_t)(key >> 32);
    const float x = __uint_as_float(up & 0x80000000u ? up & 0x7fffffffu : ~up);
    float z;
    const float share = share_of(x, top, q.inv_t, &z);
    if (share >= q.min_p) atomicAdd(&l.chunk[(uint32_t)key / kSampChunk], weight_of(share)), ++kept;
  }
  __syncthreads();
  u64 total, count;
  const u64 mine = tid < a.chunks ? l.chunk[tid] : 0, before = pick_scan(mine, l.scan_s, &total);
  if (tid == 0) l.found = 0, l.base = 0;
  (void)pick_scan(kept, l.scan_s, &count);
  const double u = (double)fmaxf(a.u[r], 0.0f);
  u64 at = (u64)fmin(u * (double)total, 18014398509481984.0 * 512.0);
  at = at < total ? at : total - 1;
  if (at >= before && at < before + mine) l.found = (u64)tid, l.base = before;
  __syncthreads();
  // the id within its chunk
  constexpr int kPer = kSampChunk / kPickThreads;
  const int64_t lo = (int64_t)l.found * kSampChunk + tid * kPer;
  const u64 base = l.base;
  u64 w[kPer], sum = 0;
#pragma unroll
  for (int i = 0; i < kPer; ++i) {
    w[i] = 0;
    if (lo + i < a.vocab) {
      const float x = logit_of(a, Elem<T>::get((const T *)a.logits + (int64_t)r * a.stride + lo + i));
      float z;
      const float share = share_of(x, top, q.inv_t, &z);
      if (share >= q.min_p && key_of(x, (uint32_t)(lo + i)) <= last) w[i] = weight_of(share);
    }
    sum += w[i];
  }
  u64 chunk_total;
  u64 x = base + pick_scan(sum, l.scan_s, &chunk_total);
#pragma unroll
  for (int i = 0; i < kPer; ++i) {
    if (at >= x && at < x + w[i]) {
      a.tokens[r] = (int32_t)(lo + i);
      if (a.prob) a.prob[r] = (float)((double)w[i] / (double)total);
      if (a.n_kept) a.n_kept[r] = (int32_t)count;
    }
    x += w[i];
  }
}

}  // namespace sats

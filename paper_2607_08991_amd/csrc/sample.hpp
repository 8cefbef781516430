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
// Nothing is sorted.  Either one launch, a workgroup per row that does all of it
// (sample_row_kernel), or four, each over chunks of the rows but the last:
//   max     the row's largest logit;
//   hist    weights (for p) and counts (for k) by bins of (max - l) / T; the row's last
//           workgroup finds the bins in which k and p can end;
//   cut     the ids of those bins go to a list, the weights of the bins before them to a
//           sum per chunk;
//   pick    a workgroup per row: k and p end at an element of the list, found by its
//           (logit, id) key against the others, or 8 bits at a time where the list is long;
//           then the chunk, then the id, of the draw.
//
// The logits are read four times, from the caches after the first.  64 rows of 128256 float32
// (32.8 MB), each with its own limits, take 55.4 us: max 8.4 (3.9 TB/s), hist 17.6, cut 14.2, pick 17.
// max is bound by its bytes.  hist and pick are chains: with top-k and top-p, 16, 32, 64 and 128
// rows take 20.2, 19.6, 21.1 and 29.6 us in hist, 9.8, 9.9, 10.1 and 10.3 in pick.  hist's is the row's
// maximum, the bins in LDS, their addition to the row's in memory by every workgroup, and the cut
// by the last one; one row of 32 workgroups takes 9.5.  What it works on, 31 vector instructions an
// id, shows above 64 rows only (8.5 us for 8.2 million ids).  cut reads as max does where k leaves
// out most ids by their bin (8.1 us), and forms every id's weight where there is no limit
// (14.8) or p alone, which leaves most of the weight in (14.6).  pick's chain is longer where p
// ends among many ids: 8.4 us without limits, 10.4 with k, 12.5 with p.
// One row is latency and the fetch of code that runs once: 128256 bf16 in four launches 17.5 us
// with min-p, 18.5 without limits, 25.3 with k, 27.1 with k and p, 30.8 with p, 13.1 for
// the largest logit alone; 2000 10.9 in one.
#pragma once

#include "elem.hpp"
#include "paged.hpp"

namespace sats {

typedef unsigned long long u64;

constexpr int kSampChunk = 4096;  // ids of a chunk
constexpr int kSampThreads = 512; // (when chosen, with 512, 1024, 256: 1 x 128256 bf16 24.7, 27.1, 26.2 us; 64 float32 rows 59.3, 57.8, 64.4)
constexpr int kSampSpan = 8;      // chunks that a workgroup takes, at most (a power of two, no more than its waves)
constexpr int kSampBins = 2048;
constexpr float kSampScale = 70.0f;   // bins per unit of (max - l) / T: weights past bin 2047 round to 0
constexpr int kPickThreads = 1024;

// Where k and p can end in a row, from its bins.
struct RowCut {
  int k_bin;          // bin that holds the last of the top k (kSampBins: all are in)
  int p_lo, p_hi;     // bins in which p can end
  int64_t k_left;     // ids of k_bin that are among the top k
  u64 k_before;       // weights of the bins before k_bin
  u64 p_before;       // weights of the bins before p_lo
};

struct SampleArgs {
  const void *logits;
  int64_t stride, vocab;
  int n, chunks, span;  // span: chunks of a workgroup (of the launches over chunks)
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
  unsigned *arrived;  // [n] workgroups of the row that have added their bins
  RowCut *cuts;       // [n]
};

// What a row asks for.
struct RowRule {
  bool first;     // the largest logit alone
  bool by_k, by_p;  // k, p may end the kept ids
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
  q.by_k = !q.first && q.k < a.vocab;
  q.by_p = !q.first && q.p < 1.0;
  return q;
}

// (x - max) / T, and its exponential: 0 for what can have no weight (NaN among it).
__device__ __forceinline__ float below(float x, float top, float inv_t) { return x == top ? 0.0f : (x - top) * inv_t; }
__device__ __forceinline__ float share_of(float z) { return z > -30.0f ? expf(z) : 0.0f; }
__device__ __forceinline__ float share_of(float x, float top, float inv_t, float *z) {
  *z = below(x, top, inv_t);
  return share_of(*z);
}
__device__ __forceinline__ u64 weight_of(float share) {  // round(2^40 share): the low bits of 2^52 + it in float64
  return (u64)__double_as_longlong(fma((double)share, 0x1p40, 0x1p52)) & ((1ull << 52) - 1);
}
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

// Largest logit of a row from its chunks (any wave, all lanes), and its lowest id.
__device__ __forceinline__ float row_max(const SampleArgs &a, int r) {
  float m = -INFINITY;
  for (int c = threadIdx.x & 63; c < a.chunks; c += 64) m = fmaxf(m, a.cmax[(int64_t)r * a.chunks + c]);
#pragma unroll
  for (int d = 32; d; d >>= 1) m = fmaxf(m, __shfl_xor(m, d));
  return m;
}
__device__ __forceinline__ float row_max(const SampleArgs &a, int r, int32_t *id) {
  float m = -INFINITY;
  int32_t at = 0x7fffffff;
  for (int c = threadIdx.x & 63; c < a.chunks; c += 64) {
    const float x = a.cmax[(int64_t)r * a.chunks + c];
    const int32_t y = a.cid[(int64_t)r * a.chunks + c];
    if (x > m) m = x, at = y;
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

// Calls f(logit, id) for this lane's ids of lo .. hi - 1 (lo a multiple of V, hi the row's end
// or a multiple of V), rising, and for ids past the end with a logit of NaN.  The next kAhead loads are under way while those before are
// looked at.  One is enough where it brings eight ids: more of them cost the time to fetch the
// longer code (16 rows of 2000 bf16: 15.5 us with one, 17.4 with two, 21.2 with four;
// 256 of 128256 95.4, 93.6, 94.9; float32 13.7, 14.7, 16.5 and 117.1, 107.3, 106.1).
template <typename T, int V, typename F>
__device__ __forceinline__ void for_range(const T *row, int lo, int hi, F f) {
  constexpr int kAhead = V == 1 ? 8 : V == 4 ? 2 : 1, kStep = 64 * V;
  const int lane = threadIdx.x & 63;
  if (lo >= hi) return;
  if constexpr (V == 1) {
    float x[kAhead], y[kAhead];
    auto load = [&](float(&to)[kAhead], int from) {
#pragma unroll
      for (int s = 0; s < kAhead; ++s) {
        to[s] = NAN;
        if (from + s * kStep + lane < hi) to[s] = Elem<T>::get(row + from + s * kStep + lane);
      }
    };
    load(x, lo);
    for (int i = lo; i < hi; i += kAhead * kStep) {
      load(y, i + kAhead * kStep);
#pragma unroll
      for (int s = 0; s < kAhead; ++s) f(x[s], (uint32_t)(i + s * kStep + lane));
#pragma unroll
      for (int s = 0; s < kAhead; ++s) x[s] = y[s];
    }
  } else {
    const int end = hi - hi % V;
    const uint32_t none = sizeof(T) == 2 ? 0x7fc07fc0u : 0x7fc00000u;
    u32x4 x[kAhead], y[kAhead];
    auto load = [&](u32x4(&to)[kAhead], int from) {
#pragma unroll
      for (int s = 0; s < kAhead; ++s) {
        to[s] = u32x4{none, none, none, none};
        const int i = from + s * kStep + lane * V;
        if (i < end) to[s] = *reinterpret_cast<const u32x4 *>(row + i);
      }
    };
    load(x, lo);
    for (int i = lo; i < end; i += kAhead * kStep) {
      load(y, i + kAhead * kStep);
#pragma unroll
      for (int s = 0; s < kAhead; ++s) {
#pragma unroll
        for (int j = 0; j < V; ++j) f(unpack<T>(x[s], j), (uint32_t)(i + s * kStep + lane * V + j));
      }
#pragma unroll
      for (int s = 0; s < kAhead; ++s) x[s] = y[s];
    }
    if (end < hi) f(end + lane < hi ? Elem<T>::get(row + end + lane) : NAN, (uint32_t)(end + lane));
  }
}
// ... of a workgroup's span: a wave takes a share of consecutive ids, which are of one chunk.
template <typename T, int V, typename F>
__device__ __forceinline__ void for_span(const SampleArgs &a, int r, F f) {
  const int per = a.span * (kSampChunk / (kSampThreads / 64)), vocab = (int)a.vocab;
  const int lo = (int)(blockIdx.x * (kSampThreads / 64) + __builtin_amdgcn_readfirstlane(threadIdx.x >> 6)) * per;
  for_range<T, V>((const T *)a.logits + (int64_t)r * a.stride, lo, lo + per < vocab ? lo + per : vocab, f);
}

template <typename T, int V>
__global__ __launch_bounds__(kSampThreads) void sample_max_kernel(SampleArgs a) {
  constexpr int kWaves = kSampThreads / 64;
  __shared__ float sm[kWaves];
  __shared__ uint32_t si[kWaves];
  const int r = blockIdx.y, w = threadIdx.x >> 6;
  for (int b = blockIdx.x * kSampThreads + threadIdx.x; b < kSampBins; b += gridDim.x * kSampThreads)
    a.hsum[(int64_t)r * kSampBins + b] = 0, a.hcnt[(int64_t)r * kSampBins + b] = 0;
  if (blockIdx.x == 0 && threadIdx.x == 0) a.n_list[r] = 0, a.arrived[r] = 0;
  float m = -INFINITY;
  uint32_t at = 0x7fffffff;
  for_span<T, V>(a, r, [&](float x, uint32_t i) {
    if (x > m) m = x, at = i;  // (a thread's ids rise)
  });
#pragma unroll
  for (int d = 32; d; d >>= 1) {
    const float x = __shfl_xor(m, d);
    const uint32_t y = __shfl_xor(at, d);
    if (x > m || (x == m && y < at)) m = x, at = y;
  }
  if ((threadIdx.x & 63) == 0) sm[w] = m, si[w] = at;
  __syncthreads();
  const int per = kWaves / a.span, c = blockIdx.x * a.span + threadIdx.x;  // waves of a chunk
  if ((int)threadIdx.x < a.span && c < a.chunks) {
    m = -INFINITY, at = 0x7fffffff;
    for (int i = threadIdx.x * per; i < (int)(threadIdx.x + 1) * per; ++i)
      if (sm[i] > m || (sm[i] == m && si[i] < at)) m = sm[i], at = si[i];
    a.cmax[(int64_t)r * a.chunks + c] = m;
    a.cid[(int64_t)r * a.chunks + c] = (int32_t)at;
  }
}

// Finds a row's cut from its bins (sum(b), count(b)), by the first 256 threads of a
// workgroup (8 bins each).
template <typename Sum, typename Count>
__device__ __forceinline__ void row_cut(const RowRule &q, Sum sum, Count count_of, u64 *lds_s, uint32_t *lds_c, RowCut *out) {
  constexpr int kPer = kSampBins / kThreads;
  u64 s[kPer], inc_s = 0;
  uint32_t c[kPer], inc_c = 0;
  const int tid = threadIdx.x, lane = tid & 63, wave = tid >> 6;
  const bool on = tid < kThreads;
  if (on) {
#pragma unroll
    for (int i = 0; i < kPer; ++i) s[i] = sum(tid * kPer + i), c[i] = count_of(tid * kPer + i);
#pragma unroll
    for (int i = 0; i < kPer; ++i) inc_s += s[i], inc_c += c[i];
  }
  const u64 own_s = inc_s;
  const uint32_t own_c = inc_c;
#pragma unroll
  for (int d = 1; d < 64; d <<= 1) {
    const u64 o = __shfl_up(inc_s, d);
    const uint32_t oc = __shfl_up(inc_c, d);
    if (lane >= d) inc_s += o, inc_c += oc;
  }
  if (on && lane == 63) lds_s[wave] = inc_s, lds_c[wave] = inc_c;
  __syncthreads();
  u64 s0 = inc_s - own_s, total = 0;
  int64_t c0 = inc_c - own_c, count = 0;
#pragma unroll
  for (int w = 0; w < kThreads / 64; ++w) {
    if (w < wave) s0 += lds_s[w], c0 += lds_c[w];
    total += lds_s[w], count += lds_c[w];
  }
  // The counts are there where k is asked for, the weights where p is: what is not there is 0
  // and not looked at.
  if (tid == 0) {
    out->k_bin = kSampBins, out->k_left = 0, out->k_before = total;
    out->p_lo = kSampBins, out->p_hi = -1, out->p_before = 0;
  }
  __syncthreads();
  if (on && q.by_k && q.k < count) {
    u64 x = s0;
    int64_t y = c0;
#pragma unroll
    for (int i = 0; i < kPer; ++i) {
      if (y < q.k && q.k <= y + c[i]) out->k_bin = tid * kPer + i, out->k_before = x, out->k_left = q.k - y;
      x += s[i], y += c[i];
    }
  }
  __syncthreads();
  if (!q.by_p) return;
  // The top k weigh at least `low`, and at most the weight of their last bin more.  p ends in
  // the last bin with weights whose sum before it is below p times that.
  const int kb = out->k_bin;
  const u64 low = out->k_before;
  if (on && kb / kPer == tid) lds_s[4] = s[kb % kPer];
  if (kb == kSampBins && tid == 0) lds_s[4] = 0;
  __syncthreads();
  if (on) {
    u64 x = s0;
    const double dl = q.p * (double)low, dh = q.p * (double)(low + lds_s[4]);
    if (tid == 0 && !(dl > 0.0)) out->p_lo = 0;
#pragma unroll
    for (int i = 0; i < kPer; ++i) {
      const double before = (double)x, after = (double)(x + s[i]);
      if (before < dl && !(after < dl)) out->p_lo = tid * kPer + i, out->p_before = x;
      if (before < dh && !(after < dh)) out->p_hi = tid * kPer + i;
      x += s[i];
    }
  }
  __syncthreads();
}

// Calls go(f), f(logit, id) adding an id to the bins that the row's rule looks at: without a
// branch, so that the ids of a load overlap (what has no weight goes to a bin of the lane's
// past the last; from -29 on weights are 0).
constexpr int kSampBinsAll = kSampBins + 64;
template <typename Go>
__device__ __forceinline__ void with_bins(const RowRule &q, float top, u64 *hs, uint32_t *hc, Go go) {
  const int none = kSampBins + (threadIdx.x & 63);
  if (!q.by_p) {
    go([&](float x, uint32_t) {
      const float z = fmaxf(below(x, top, q.inv_t), -29.0f);
      atomicAdd(&hc[weight_of(expf(z)) ? (int)(-z * kSampScale) : none], 1u);
    });
  } else {
    const bool by_k = q.by_k;
    go([&](float x, uint32_t) {
      const float z = fmaxf(below(x, top, q.inv_t), -29.0f);
      const u64 w = weight_of(expf(z));
      const int b = z > -29.0f ? (int)(-z * kSampScale) : none;
      atomicAdd(&hs[b], w);
      if (by_k) atomicAdd(&hc[b], (uint32_t)(w != 0));
    });
  }
}

// Only ids whose (l - max) / T is above this can be kept or listed: those in bins below `reach`,
// where k or p set it, or above min_p where neither did.
__device__ __forceinline__ float least_z(const RowRule &q, int reach) {
  if (q.by_k || q.by_p) return reach < kSampBins ? -1.00001f / kSampScale * (float)reach : -30.0f;
  return q.min_p > 0.0f ? fmaxf(-30.0f, 1.00001f * logf(q.min_p) - 0.00001f) : -30.0f;
}

template <typename T, int V>
__global__ __launch_bounds__(kSampThreads) void sample_hist_kernel(SampleArgs a) {
  __shared__ u64 hs[kSampBinsAll];
  __shared__ uint32_t hc[kSampBinsAll];
  __shared__ u64 ls[8];
  __shared__ uint32_t lc[4];
  __shared__ RowCut cut;
  __shared__ int last;
  const int r = blockIdx.y;
  const RowRule q = row_rule(a, r);
  if (!q.by_k && !q.by_p) return;
  const float top = row_max(a, r);
  for (int b = threadIdx.x; b < kSampBins; b += kSampThreads) hs[b] = 0, hc[b] = 0;
  __syncthreads();
  with_bins(q, top, hs, hc, [&](auto f) { for_span<T, V>(a, r, f); });
  __syncthreads();
  for (int b = threadIdx.x; b < kSampBins; b += kSampThreads) {
    if (hs[b]) atomicAdd(&a.hsum[(int64_t)r * kSampBins + b], hs[b]);
    if (hc[b]) atomicAdd(&a.hcnt[(int64_t)r * kSampBins + b], hc[b]);
  }
  if (!arrive_last(a.arrived + r, gridDim.x, &last)) return;
  // (the bins were added by other workgroups of this launch)
  const u64 *hsum = a.hsum + (int64_t)r * kSampBins;
  const uint32_t *hcnt = a.hcnt + (int64_t)r * kSampBins;
  row_cut(
      q, [&](int b) { return __hip_atomic_load(hsum + b, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT); },
      [&](int b) { return __hip_atomic_load(hcnt + b, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT); }, ls, lc, &cut);
  if (threadIdx.x == 0) a.cuts[r] = cut;
}

constexpr uint32_t kCutList = 4096;

template <typename T, int V>
__global__ __launch_bounds__(kSampThreads) void sample_cut_kernel(SampleArgs a) {
  __shared__ u64 ls[kSampThreads / 64];
  __shared__ uint32_t lc[kSampThreads / 64];
  const int r = blockIdx.y;
  const RowRule q = row_rule(a, r);
  if (q.first) return;
  const float top = row_max(a, r);
  // bins below `sure` are kept whole (but for k_bin), those up to `maybe`, and k_bin, go to the list
  int sure = kSampBins, maybe = -1, k_bin = -1;
  if (q.by_k || q.by_p) {
    const RowCut cut = a.cuts[r];
    k_bin = cut.k_bin;
    if (q.by_p) sure = cut.p_lo, maybe = cut.p_hi;
    else sure = k_bin;  // (p 1: the top k, to the last)
  }
  // the list is gathered in LDS, so that a workgroup counts in the row's list once (what does
  // not fit is counted one by one)
  __shared__ u64 keys[kCutList];
  __shared__ uint32_t n_keys, first;
  if (threadIdx.x == 0) n_keys = 0;
  __syncthreads();
  u64 sum = 0;
  uint32_t cnt = 0;
  u64 *list = a.list + (int64_t)r * a.vocab;
  const float least = least_z(q, max(sure, max(maybe, k_bin) + 1));
  auto take = [&](float x, uint32_t i) {
    const float z = below(x, top, q.inv_t);
    if (!(z > least)) return;
    const int b = bin_of(z);
    const bool listed = ((b >= sure) & (b <= maybe)) | (b == k_bin);
    if (b < sure || listed) {
      const float share = share_of(z);
      const u64 w = weight_of(share);
      if (listed) {
        if (!w) return;
        const uint32_t at = atomicAdd(&n_keys, 1u);
        if (at < kCutList) keys[at] = key_of(x, i);
        else list[atomicAdd(&a.n_list[r], 1u)] = key_of(x, i);
      } else if (share >= q.min_p) {
        sum += w, cnt += w != 0;
      }
    }
  };
  for_span<T, V>(a, r, take);
  sum = wave_sum(sum);
  const u64 c = wave_sum((u64)cnt);
  if ((threadIdx.x & 63) == 0) ls[threadIdx.x >> 6] = sum, lc[threadIdx.x >> 6] = (uint32_t)c;
  __syncthreads();
  const int per = kSampThreads / 64 / a.span, chunk = blockIdx.x * a.span + threadIdx.x;
  if ((int)threadIdx.x < a.span && chunk < a.chunks) {
    sum = 0, cnt = 0;
    for (int i = threadIdx.x * per; i < (int)(threadIdx.x + 1) * per; ++i) sum += ls[i], cnt += lc[i];
    a.csum[(int64_t)r * a.chunks + chunk] = sum;
    a.ccnt[(int64_t)r * a.chunks + chunk] = cnt;
  }
  const uint32_t n = n_keys < kCutList ? n_keys : kCutList;
  if (threadIdx.x == 0 && n) first = atomicAdd(&a.n_list[r], n);
  __syncthreads();
  for (uint32_t i = threadIdx.x; i < n; i += kSampThreads) list[first + i] = keys[i];
}

constexpr int kPickList = 2048;  // keys of the list that are held in LDS
constexpr int kPickWave = 2048;  // ... that one wave looks through
constexpr int kPickFew = 256;    // ... whose ranks are counted

struct PickLds {
  u64 sum[256], rank[256];
  uint32_t cnt[256];
  u64 key_and, key_or, base, weight, found;
  int64_t left;
  uint32_t one;
  u64 scan[kPickThreads / 64];
  u64 chunk[kPickThreads];
  u64 few_p[256], few_k[256];
  u64 keys[kPickList], weights[kPickList];  // (weights: in the low 48 bits, the bin above)
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

__device__ __forceinline__ float key_logit(u64 key) {
  const uint32_t up = ~(uint32_t)(key >> 32);
  return __uint_as_float(up & 0x80000000u ? up & 0x7fffffffu : ~up);
}

// The keys of a row's list in bins [lo, hi], with their weights.
struct PickKeys {
  const u64 *list;
  const u64 *weights;  // with the bins, or null
  uint32_t n;
  float top, inv_t;
  int lo, hi;
  __device__ __forceinline__ u64 weigh(u64 key) const {
    float z;
    const u64 w = weight_of(share_of(key_logit(key), top, inv_t, &z));
    return (u64)bin_of(z) << 48 | w;
  }
  template <int THREADS, typename F> __device__ __forceinline__ void each(int tid, u64 fixed, u64 value, F f) const {
    for (uint32_t i = tid; i < n; i += THREADS) {
      const u64 key = list[i];
      if ((key & fixed) != value) continue;
      const u64 w = weights ? weights[i] : weigh(key);
      const int b = (int)(w >> 48);
      if (b >= lo && b <= hi) f(key, w & ((1ull << 48) - 1));
    }
  }
};

// The key at which the kept ids end: the `left`-th smallest (by_count), or the last one
// whose weights before it, from `base` on, are below `limit`.  Each step splits the keys
// that are left by the 8 highest bits in which they differ and goes on with one part.
// *upto: base and the weights up to it.  By the whole workgroup or by its first wave.
template <int THREADS>
__device__ __forceinline__ u64 pick_end(const PickKeys &k, bool by_count, int64_t left, u64 base, double limit, PickLds &l, u64 *upto) {
  u64 fixed = 0, value = 0;  // bits that are decided, and what they are
  const int tid = threadIdx.x;
  auto meet = [] {
    if constexpr (THREADS > 64) {
      __syncthreads();
    } else {
      __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront");
      __builtin_amdgcn_wave_barrier();
    }
  };
  for (;;) {
    meet();
    for (int b = tid; b < 256; b += THREADS) l.sum[b] = 0, l.cnt[b] = 0;
    if (tid == 0) l.key_and = ~0ull, l.key_or = 0;
    meet();
    u64 ka = ~0ull, ko = 0;
    k.template each<THREADS>(tid, fixed, value, [&](u64 key, u64) { ka &= key, ko |= key; });
#pragma unroll
    for (int d = 32; d; d >>= 1) ka &= __shfl_xor(ka, d), ko |= __shfl_xor(ko, d);
    if ((tid & 63) == 0 && ko) atomicAnd(&l.key_and, ka), atomicOr(&l.key_or, ko);
    meet();
    const u64 key_and = l.key_and, diff = key_and ^ l.key_or;
    const int high = diff ? 63 - __clzll((long long)diff) : 7, shift = high > 7 ? high - 7 : 0;
    k.template each<THREADS>(tid, fixed, value, [&](u64 key, u64 w) {
      const int b = (int)(key >> shift) & 255;
      atomicAdd(&l.sum[b], w);
      atomicAdd(&l.cnt[b], 1u);
    });
    meet();
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
        if (c[i] && (by_count ? cb < left : (double)before < limit)) part = 4 * tid + i, at = before, cat = cb, size = c[i];
        before += s[i], cb += c[i];
      }
      const u64 any = __ballot(part >= 0);
      const int winner = any ? 63 - __clzll((long long)any) : -1;
      if (tid == winner) l.found = (u64)part, l.base = at, l.left = cat, l.one = size;
      if (winner < 0 && tid == 0) l.found = 0, l.base = base, l.left = 0, l.one = 0;
    }
    meet();
    // (bits above `high` are common to the keys that are left)
    const u64 above = shift + 8 < 64 ? ~0ull << (shift + 8) : 0;
    fixed = above | 255ull << shift;
    value = (key_and & above) | l.found << shift;
    base = l.base;
    left -= l.left;
    if (l.one <= 1 || shift == 0) break;
  }
  // the one key that is left (all bits are decided where shift reached 0)
  meet();
  if (tid == 0) l.found = 0, l.weight = 0;
  meet();
  k.template each<THREADS>(tid, fixed, value, [&](u64 key, u64 w) { l.found = key, l.weight = w; });
  meet();
  *upto = base + l.weight;
  return l.found;
}

// The key at which a row's kept ids end.
template <int THREADS>
__device__ __forceinline__ u64 pick_last(const RowRule &q, const RowCut &cut, PickKeys k, PickLds &l) {
  u64 all = cut.k_before, end = ~0ull;
  // (one loop for k and for p: code that runs once costs its fetch)
#pragma unroll 1
  for (int step = 0; step < 2; ++step) {
    const bool by_k = step == 0;
    if (by_k ? cut.k_bin >= kSampBins : !q.by_p) continue;
    k.lo = by_k ? cut.k_bin : cut.p_lo, k.hi = by_k ? cut.k_bin : cut.p_hi;
    end = pick_end<THREADS>(k, by_k, cut.k_left, by_k ? cut.k_before : cut.p_before, q.p * (double)all, l, &all);
  }
  return end;
}

// The same where the keys are few: every key against every other.
__device__ __forceinline__ u64 pick_few(const RowRule &q, const RowCut &cut, const PickKeys &k, PickLds &l) {
  static_assert(kPickFew == 256 && kPickThreads % 256 == 0, "");
  constexpr u64 kOne = 1ull << 50;  // (256 weights sum to less)
  const int tid = threadIdx.x, i = tid & 255;
  const int n = (int)k.n;
  if (tid < 256) {
    u64 p = 0, of_k = 0;
    if (tid < n) {
      const u64 both = l.weights[tid], w = both & ((1ull << 48) - 1);
      const int b = (int)(both >> 48);
      p = b >= cut.p_lo && b <= cut.p_hi ? w : 0;
      of_k = b == cut.k_bin ? w | kOne : 0;
    }
    l.few_p[tid] = p, l.few_k[tid] = of_k, l.sum[tid] = 0, l.rank[tid] = 0;
  }
  if (tid == 0) l.base = cut.k_before, l.found = ~0ull, l.weight = 0;
  __syncthreads();
  const u64 key = i < n ? l.keys[i] : 0;
  const bool by_k = cut.k_bin < kSampBins;
  if (i < n) {
    u64 p = 0, of_k = 0;
    if (by_k) {
      for (int j = tid >> 8; j < n; j += kPickThreads / 256) {
        const bool less = l.keys[j] < key;
        p += less ? l.few_p[j] : 0, of_k += less ? l.few_k[j] : 0;
      }
      atomicAdd(&l.rank[i], of_k);
    } else {
      for (int j = tid >> 8; j < n; j += kPickThreads / 256) p += l.keys[j] < key ? l.few_p[j] : 0;
    }
    atomicAdd(&l.sum[i], p);
  }
  __syncthreads();
  if (by_k) {
    if (tid < n && l.few_k[tid] && (int64_t)(l.rank[tid] / kOne) == cut.k_left - 1)
      l.found = key, l.base = cut.k_before + ((l.rank[tid] + l.few_k[tid]) & (kOne - 1));
    __syncthreads();
  }
  if (!q.by_p) return l.found;
  const double limit = q.p * (double)l.base;
  if (tid < n && l.few_p[tid] && (double)(cut.p_before + l.sum[tid]) < limit) atomicMax(&l.weight, key);
  __syncthreads();
  return l.weight;
}

template <typename T>
__global__ __launch_bounds__(kPickThreads) void sample_pick_kernel(SampleArgs a) {
  __shared__ PickLds l;
  __shared__ u64 end_lds;
  const int r = blockIdx.x, tid = threadIdx.x;
  // everything that the row has so far, in one wait (what a row without a cut has not is not used)
  const bool mine_there = tid < a.chunks;
  const u64 csum = mine_there ? a.csum[(int64_t)r * a.chunks + tid] : 0;
  const uint32_t ccnt = mine_there ? a.ccnt[(int64_t)r * a.chunks + tid] : 0, n = a.n_list[r];
  const RowCut cut = a.cuts[r];
  const RowRule q = row_rule(a, r);
  const double u = (double)fmaxf(a.u[r], 0.0f);
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
  // weights and counts of each chunk
  u64 kept = ccnt;
  if (mine_there) l.chunk[tid] = csum;
  u64 last = ~0ull;
  if (q.by_k || q.by_p) {
    PickKeys k{a.list + (int64_t)r * a.vocab, nullptr, n, top, q.inv_t, 0, 0};
    if (n <= kPickList) {
      for (uint32_t i = tid; i < n; i += kPickThreads) {
        const u64 key = k.list[i];
        l.keys[i] = key;
        l.weights[i] = k.weigh(key);
      }
      k.list = l.keys, k.weights = l.weights;
    }
    __syncthreads();
    if (n <= kPickFew) {
      last = pick_few(q, cut, k, l);
    } else if (n <= kPickWave) {
      if (tid < 64) {
        const u64 end = pick_last<64>(q, cut, k, l);
        if (tid == 0) end_lds = end;
      }
      __syncthreads();
      last = end_lds;
    } else {
      last = pick_last<kPickThreads>(q, cut, k, l);
    }
    __syncthreads();
    for (uint32_t i = tid; i < n; i += kPickThreads) {
      const u64 key = k.list[i];
      if (key > last) continue;
      float z;
      const float share = share_of(key_logit(key), top, q.inv_t, &z);
      if (share >= q.min_p) atomicAdd(&l.chunk[(uint32_t)key / kSampChunk], weight_of(share)), ++kept;
    }
  }
  __syncthreads();
  u64 total, count;
  const u64 mine = tid < a.chunks ? l.chunk[tid] : 0, before = pick_scan(mine, l.scan, &total);
  if (tid == 0) l.found = 0, l.base = 0;
  (void)pick_scan(kept, l.scan, &count);
  u64 at = (u64)fmin(u * (double)total, 0x1p63);
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
      const float x = Elem<T>::get((const T *)a.logits + (int64_t)r * a.stride + lo + i);
      float z;
      const float share = share_of(x, top, q.inv_t, &z);
      if (share >= q.min_p && key_of(x, (uint32_t)(lo + i)) <= last) w[i] = weight_of(share);
    }
    sum += w[i];
  }
  u64 chunk_total;
  u64 x = base + pick_scan(sum, l.scan, &chunk_total);
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

// A row by one workgroup: the same steps, one after the other, bins and list in LDS.  A row
// of the four launches costs the chip less, but they are four, and pass through the caches:
// the host takes this one where its rounds over the chip are shorter.
template <typename T, int V>
__global__ __launch_bounds__(kPickThreads) void sample_row_kernel(SampleArgs a) {
  constexpr int kWaves = kPickThreads / 64;
  __shared__ PickLds l;
  __shared__ u64 hs[kSampBinsAll];
  __shared__ uint32_t hc[kSampBinsAll];
  __shared__ RowCut cut;
  __shared__ float wave_top[kWaves];
  __shared__ int32_t wave_id[kWaves];
  __shared__ u64 end_lds, wave_sum_lds[kWaves];
  __shared__ uint32_t n_keys, n_sure;
  const int r = blockIdx.x, tid = threadIdx.x, w = __builtin_amdgcn_readfirstlane(tid >> 6);
  const T *row = (const T *)a.logits + (int64_t)r * a.stride;
  const int vocab = (int)a.vocab, share = ((vocab + kWaves - 1) / kWaves + 7) / 8 * 8;  // ids of a wave
  const int lo = min(w * share, vocab), hi = min(lo + share, vocab);
  const RowRule q = row_rule(a, r);
  for (int b = tid; b < kSampBins; b += kPickThreads) hs[b] = 0, hc[b] = 0;
  if (tid == 0) n_keys = 0, n_sure = 0;
  // the largest logit and its lowest id
  float top = -INFINITY;
  int32_t id = 0x7fffffff;
  for_range<T, V>(row, lo, hi, [&](float x, uint32_t i) {
    if (x > top) top = x, id = (int32_t)i;
  });
#pragma unroll
  for (int d = 32; d; d >>= 1) {
    const float x = __shfl_xor(top, d);
    const int32_t y = __shfl_xor(id, d);
    if (x > top || (x == top && y < id)) top = x, id = y;
  }
  if ((tid & 63) == 0) wave_top[w] = top, wave_id[w] = id;
  __syncthreads();
  top = wave_top[0], id = wave_id[0];
#pragma unroll
  for (int i = 1; i < kWaves; ++i)
    if (wave_top[i] > top) top = wave_top[i], id = wave_id[i];  // (the waves' ids rise)
  if (q.first || !(top > -INFINITY)) {
    const bool some = top > -INFINITY;
    if (tid == 0) {
      a.tokens[r] = some ? id : -1;
      if (a.prob) a.prob[r] = some ? 1.0f : 0.0f;
      if (a.n_kept) a.n_kept[r] = some;
    }
    return;
  }
  int sure = kSampBins, maybe = -1, k_bin = -1;
  if (q.by_k || q.by_p) {
    with_bins(q, top, hs, hc, [&](auto f) { for_range<T, V>(row, lo, hi, f); });
    __syncthreads();
    row_cut(q, [&](int b) { return hs[b]; }, [&](int b) { return hc[b]; }, l.scan, l.cnt, &cut);
    k_bin = cut.k_bin;
    if (q.by_p) sure = cut.p_lo, maybe = cut.p_hi;
    else sure = k_bin;
  }
  // the list, and the weights kept for certain
  u64 *list = a.list + (int64_t)r * a.vocab;
  u64 sum = 0;
  uint32_t cnt = 0;
  const float least = least_z(q, max(sure, max(maybe, k_bin) + 1));
  auto take = [&](float x, uint32_t i) {
    const float z = below(x, top, q.inv_t);
    if (!(z > least)) return;
    const int b = bin_of(z);
    const bool listed = ((b >= sure) & (b <= maybe)) | (b == k_bin);
    if (b < sure || listed) {
      const float sh = share_of(z);
      const u64 wt = weight_of(sh);
      if (listed) {
        if (!wt) return;
        const uint32_t at = atomicAdd(&n_keys, 1u);
        if (at < kPickList) l.keys[at] = key_of(x, i);
        else list[at] = key_of(x, i);
      } else if (sh >= q.min_p) {
        sum += wt, cnt += wt != 0;
      }
    }
  };
  for_range<T, V>(row, lo, hi, take);
  sum = wave_sum(sum);
  const u64 c = wave_sum((u64)cnt);
  if ((tid & 63) == 0) wave_sum_lds[w] = sum, atomicAdd(&n_sure, (uint32_t)c);
  __syncthreads();
  u64 last = ~0ull, kept = 0;
  const uint32_t n = n_keys;
  if (n) {
    PickKeys k{list, nullptr, n, top, q.inv_t, 0, 0};
    if (n <= kPickList) {
      for (uint32_t i = tid; i < n; i += kPickThreads) l.weights[i] = k.weigh(l.keys[i]);
      k.list = l.keys, k.weights = l.weights;
    } else {
      for (uint32_t i = tid; i < kPickList; i += kPickThreads) list[i] = l.keys[i];
    }
    __syncthreads();
    if (n <= kPickFew) {
      last = pick_few(q, cut, k, l);
    } else if (n <= kPickWave) {
      if (tid < 64) {
        const u64 end = pick_last<64>(q, cut, k, l);
        if (tid == 0) end_lds = end;
      }
      __syncthreads();
      last = end_lds;
    } else {
      last = pick_last<kPickThreads>(q, cut, k, l);
    }
    __syncthreads();
    for (uint32_t i = tid; i < n; i += kPickThreads) {
      const u64 key = k.list[i];
      if (key > last) continue;
      const float sh = share_of(below(key_logit(key), top, q.inv_t));
      if (sh >= q.min_p) atomicAdd(&wave_sum_lds[(uint32_t)key / (uint32_t)share], weight_of(sh)), ++kept;
    }
  }
  u64 count;
  (void)pick_scan(kept, l.scan, &count);
  // the wave's share that holds the draw, then the thread's, then the id
  u64 total = 0;
#pragma unroll
  for (int i = 0; i < kWaves; ++i) total += wave_sum_lds[i];
  const double u = (double)fmaxf(a.u[r], 0.0f);
  u64 at = (u64)fmin(u * (double)total, 0x1p63);
  at = at < total ? at : total - 1;
  u64 base = 0;
  int from = 0;
  for (; from < kWaves - 1 && at >= base + wave_sum_lds[from]; ++from) base += wave_sum_lds[from];
  const int per = (share + kPickThreads - 1) / kPickThreads;
  const int t0 = from * share + tid * per, t1 = min(t0 + per, min((from + 1) * share, vocab));
  auto weight_at = [&](int i) -> u64 {
    const float x = Elem<T>::get(row + i), sh = share_of(below(x, top, q.inv_t));
    return sh >= q.min_p && key_of(x, (uint32_t)i) <= last ? weight_of(sh) : 0;
  };
  u64 own = 0, unused;
  for (int i = t0; i < t1; ++i) own += weight_at(i);
  u64 x = base + pick_scan(own, l.scan, &unused);
  if (at < x || at >= x + own) return;
  for (int i = t0; i < t1; ++i) {
    const u64 wt = weight_at(i);
    if (at < x + wt) {
      a.tokens[r] = (int32_t)i;
      if (a.prob) a.prob[r] = (float)((double)wt / (double)total);
      if (a.n_kept) a.n_kept[r] = (int32_t)(count + n_sure);
      return;
    }
    x += wt;
  }
}

}  // namespace sats

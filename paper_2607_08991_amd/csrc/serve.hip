// Host side of the serving operators declared in include/sats.h: argument checks,
// scratch memory and launches.
#include <hip/hip_runtime.h>

#include <algorithm>
#include <cmath>
#include <type_traits>

#include "host.hpp"

#include "attend_host.hpp"
#include "logits.hpp"
#include "pages.hpp"
#include "rope.hpp"
#include "sample.hpp"

namespace {

using sats_host::clear_error;
using sats_host::fail;
using sats_host::Turn;

bool on16(const void *p) { return (reinterpret_cast<uintptr_t>(p) & 15) == 0; }

size_t align_up(size_t v) { return (v + 255) & ~size_t(255); }

struct Carve {
  char *base;
  size_t off = 0;
  template <typename T> T *take(size_t count) {
    T *p = reinterpret_cast<T *>(base ? base + off : nullptr);
    off += align_up(std::max<size_t>(count, 1) * sizeof(T));
    return p;
  }
};

using sats_host::kMaxGrid;
using sats_host::launched;

constexpr int64_t kMaxCount = (int64_t)1 << 30;

// Rotation: waves that fill the chip.
constexpr int64_t kRopeWaves = 4096;
// Compute units, twice over.
constexpr int kSlots = 512;

// The format of a cache's rows, the bytes of one of its elements, its 8-bit part (or null), and the
// type of what is quantised into it and attends over it.
int form_of(const sats_kv_cache *c) {
  return c->elem_bytes == SATS_KV_E4M3 ? sats::kE4m3 : c->elem_bytes == SATS_KV_INT8 ? sats::kInt8 : sats::kPlain;
}
int stored_bytes(const sats_kv_cache *c) { return form_of(c) ? 1 : c->elem_bytes; }
const sats_kv_cache8 *cache8_of(const sats_kv_cache *c) {
  return form_of(c) ? reinterpret_cast<const sats_kv_cache8 *>(c) : nullptr;
}
int outer_bytes(const sats_kv_cache *c) { return form_of(c) ? cache8_of(c)->q_elem_bytes : c->elem_bytes; }

// Rows (of a token's head) of every layer, and bytes of an array of keys (or values) of every layer.
double pool_rows(const sats_kv_cache *c) {
  return (double)c->n_layers * (double)c->n_pages * (double)c->n_kv_heads * (double)c->page_size;
}
double pool_bytes(const sats_kv_cache *c) { return pool_rows(c) * (double)c->head_dim * stored_bytes(c); }

int check_cache(const sats_kv_cache *c, bool data) {
  if (!c) return fail(SATS_ERR_NULL, "cache must be non-null");
  if (data && (!c->k || !c->v)) return fail(SATS_ERR_NULL, "the cache's k and v must be non-null");
  const sats_kv_cache8 *c8 = cache8_of(c);
  if (!c8 && c->elem_bytes != 2 && c->elem_bytes != 4)
    return fail(SATS_ERR_ARG, "elem_bytes must be 2, 4, SATS_KV_E4M3 or SATS_KV_INT8");
  if (c8 && data && (!c8->k_scale || !c8->v_scale)) return fail(SATS_ERR_NULL, "the cache's k_scale and v_scale must be non-null");
  if (c8 && data && (reinterpret_cast<uintptr_t>(c8->k_scale) % 4 || reinterpret_cast<uintptr_t>(c8->v_scale) % 4))
    return fail(SATS_ERR_ARG, "the cache's k_scale and v_scale must be 4-byte aligned");
  if (c8 && c8->q_elem_bytes != 2 && c8->q_elem_bytes != 4) return fail(SATS_ERR_ARG, "q_elem_bytes must be 2 or 4");
  if (c->n_layers < 1 || c->n_pages < 1 || c->n_kv_heads < 1 || c->n_layers > 4096 || c->n_pages > kMaxCount ||
      c->n_kv_heads > 1024)
    return fail(SATS_ERR_SHAPE, "a cache has 1 to 4096 layers, 1 to 2^30 pages and 1 to 1024 heads");
  if (c->page_size < 1 || c->page_size > 4096 || (c->page_size & (c->page_size - 1)))
    return fail(SATS_ERR_SHAPE, "page_size must be a power of two up to 4096");
  if (c->head_dim < 8 || c->head_dim > 256 || c->head_dim % 8)
    return fail(SATS_ERR_SHAPE, "head_dim must be a multiple of 8 from 8 to 256");
  if (c8 && (c->page_size < 16 || c->head_dim % 16))
    return fail(SATS_ERR_SHAPE, "a cache of 8 bits has pages of at least 16 tokens, and heads of a multiple of 16 dims");
  if (pool_bytes(c) > 1e18) return fail(SATS_ERR_SHAPE, "the cache is too large");
  if (data && (!on16(c->k) || !on16(c->v))) return fail(SATS_ERR_ARG, "the cache's k and v must be 16-byte aligned");
  return SATS_OK;
}

int log2_of(int64_t v) {
  int s = 0;
  while (((int64_t)1 << s) < v) ++s;
  return s;
}

sats::PoolView pool_view(const sats_kv_cache *c) {
  return {c->n_pages, (int)c->n_kv_heads, (int)c->page_size, log2_of(c->page_size)};
}

int check_batch(const sats_kv_batch *b) {
  if (!b) return fail(SATS_ERR_NULL, "batch must be non-null");
  if (b->n_seqs < 0 || b->n_tokens < 0 || b->max_pages < 0 || b->max_q_len < 0 || b->max_kv_len < 0 ||
      b->n_seqs > kMaxCount || b->n_tokens > kMaxCount || b->max_pages > kMaxCount || b->max_q_len > kMaxCount ||
      b->max_kv_len >= (int64_t)1 << 31)
    return fail(SATS_ERR_SHAPE, "a batch's sizes must be >= 0, at most 2^30 (lengths below 2^31)");
  if (b->n_tokens > 0 && b->n_seqs < 1) return fail(SATS_ERR_SHAPE, "tokens without a sequence");
  if (b->n_tokens > 0 && (!b->table || !b->q_start || !b->kv_len))
    return fail(SATS_ERR_NULL, "the batch's table, q_start and kv_len must be non-null");
  return SATS_OK;
}

sats::BatchView batch_view(const sats_kv_batch *b) {
  return {b->table, b->q_start, b->kv_len, (int)b->n_seqs, b->max_pages, b->n_tokens, b->max_q_len, b->max_kv_len};
}

char *layer_of(void *pool, const sats_kv_cache *c, int64_t layer) {
  return static_cast<char *>(pool) + layer * c->n_pages * c->n_kv_heads * c->page_size * c->head_dim * stored_bytes(c);
}
uint8_t *layer_scales(uint8_t *scales, const sats_kv_cache *c, int64_t layer) {
  return scales + layer * c->n_pages * c->n_kv_heads * c->page_size;
}

// Bytes from a row's start to the last row's end, for n rows of `row` elements at a stride.
int64_t span(int64_t n, int64_t stride, int64_t row, int esz) { return n > 0 ? ((n - 1) * stride + row) * esz : 0; }

bool overlap(const void *a, int64_t na, const void *b, int64_t nb) {
  const char *x = static_cast<const char *>(a), *y = static_cast<const char *>(b);
  return na > 0 && nb > 0 && x < y + nb && y < x + na;
}

// n rows of `row` elements at a stride (none: a null pointer, or no elements).
struct Rows {
  const void *p;
  int64_t stride, row;
};
bool same_rows(const Rows &a, const Rows &b) { return a.p == b.p && a.stride == b.stride; }
// Whether any of n rows of a touches one of b.  Rows of one stride may lie between each other (parts
// of one projection's output); of different strides they are apart where their spans are.
bool rows_overlap(const Rows &a, const Rows &b, int64_t n, int esz) {
  if (!a.p || !b.p || !a.row || !b.row || !overlap(a.p, span(n, a.stride, a.row, esz), b.p, span(n, b.stride, b.row, esz))) return false;
  if (n == 1 || a.stride != b.stride) return true;
  const int64_t s = a.stride * esz, off = (int64_t)(reinterpret_cast<uintptr_t>(b.p) - reinterpret_cast<uintptr_t>(a.p));
  const int64_t d = (off % s + s) % s;  // from a row of a to the next one of b
  return d < a.row * esz || d + b.row * esz > s;
}

// Whether n bytes at p touch the cache's arrays.
bool in_cache(const void *p, int64_t n, const sats_kv_cache *c) {
  const int64_t all = (int64_t)pool_bytes(c), rows = (int64_t)pool_rows(c);
  const sats_kv_cache8 *c8 = cache8_of(c);
  return overlap(p, n, c->k, all) || overlap(p, n, c->v, all) ||
         (c8 && (overlap(p, n, c8->k_scale, rows) || overlap(p, n, c8->v_scale, rows)));
}

// ------------------------------------------------------------- norm and rotation

// (cache: where keys and values go, or null)
int run_rope(sats::RopeArgs a, int esz, const sats_kv_cache *cache, hipStream_t stream) {
  const bool append = cache != nullptr;
  const int64_t n = a.n_tokens;
  if (n < 0 || n > kMaxCount || a.n_q < 0 || a.n_kv < 0 || a.n_q > 4096 || a.n_kv > 1024)
    return fail(SATS_ERR_SHAPE, "n_tokens, n_q_heads or n_kv_heads out of range");
  if (a.dim < 2 || a.dim > 256 || a.dim % 2) return fail(SATS_ERR_SHAPE, "head_dim must be even, at most 256");
  if (a.rot < 0 || a.rot > a.dim || a.rot % 2) return fail(SATS_ERR_SHAPE, "rot_dim must be even, 0 to head_dim");
  if (a.rot > 0 && (a.n_pos < 1 || a.n_pos >= (int64_t)1 << 31)) return fail(SATS_ERR_SHAPE, "rope needs 1 to 2^31 positions");
  if (a.pairs < 0 || a.pairs > 1) return fail(SATS_ERR_ARG, "interleaved must be 0 or 1");
  if (!(a.eps >= 0.0f) || std::isinf(a.eps)) return fail(SATS_ERR_ARG, "eps must be finite and >= 0");
  a.rows = a.n_q + a.n_kv * (append ? 2 : 1);
  if (n == 0 || a.rows == 0) return SATS_OK;
  if ((a.n_q && (!a.q || !a.q_out)) || (a.n_kv && (!a.k || (append ? !a.v : !a.k_out))))
    return fail(SATS_ERR_NULL, "q, k, v and the outputs must be non-null");
  if (a.rot > 0 && (!a.rope || (!append && !a.positions))) return fail(SATS_ERR_NULL, "rope and positions must be non-null");
  const int64_t qrow = (int64_t)a.n_q * a.dim, krow = (int64_t)a.n_kv * a.dim;
  if (a.q_stride < qrow || a.q_out_stride < qrow || a.k_stride < krow || (append ? a.v_stride : a.k_out_stride) < krow)
    return fail(SATS_ERR_SHAPE, "a token stride is below the token's row");
  // an output's rows: those of its own input, or apart from every input's and the other output's
  const Rows q{a.q, a.q_stride, qrow}, k{a.k, a.k_stride, krow}, v{append ? a.v : nullptr, a.v_stride, krow};
  const Rows qo{a.q_out, a.q_out_stride, qrow}, ko{append ? nullptr : a.k_out, a.k_out_stride, krow};
  if ((!same_rows(qo, q) && rows_overlap(qo, q, n, esz)) || rows_overlap(qo, k, n, esz) || rows_overlap(qo, v, n, esz))
    return fail(SATS_ERR_ARG, "q_out overlaps the inputs without being q itself");
  if ((!same_rows(ko, k) && rows_overlap(ko, k, n, esz)) || rows_overlap(ko, q, n, esz))
    return fail(SATS_ERR_ARG, "k_out overlaps the inputs without being k itself");
  if (rows_overlap(qo, ko, n, esz)) return fail(SATS_ERR_ARG, "q_out and k_out overlap");
  if (append)
    for (const Rows &r : {q, k, v, qo})
      if (r.p && r.row && in_cache(r.p, span(n, r.stride, r.row, esz), cache))
        return fail(SATS_ERR_ARG, "q, k, v or q_out overlaps the cache");
  const int vec = 16 / esz;
  const bool wide = a.dim % (2 * vec) == 0 && a.rot % (2 * vec) == 0 && on16(a.q) && on16(a.k) && on16(a.v) &&
                    on16(a.q_norm) && on16(a.k_norm) && on16(a.rope) && on16(a.q_out) && on16(a.k_out) &&
                    a.q_stride % vec == 0 && a.k_stride % vec == 0 && a.v_stride % vec == 0 &&
                    a.q_out_stride % vec == 0 && a.k_out_stride % vec == 0;
  const int units = a.dim / (2 * (wide ? vec : 1));
  a.lanes = 1;
  while (a.lanes < units && a.lanes < 64) a.lanes *= 2;
  // rows of a token that a row of lanes takes one after another (they share its angles): as
  // many as leave kRopeWaves waves, 8 at most.  4096 tokens of 48 rows: 1 30.3 us, 2 26.1, 6
  // (a wave a token) 22.9; a few tokens want every row in lanes of its own.
  a.per = 1;
  while (a.per < 8 && a.per < a.rows && n * ((a.rows + a.per) / (a.per + 1)) * a.lanes >= kRopeWaves * 64) ++a.per;
  const int64_t groups = (a.rows + a.per - 1) / a.per, threads = n * groups * a.lanes;
  if (threads > sats::kThreads * kMaxGrid) return fail(SATS_ERR_SHAPE, "too many rows for one call");
  const dim3 grid((unsigned)((threads + sats::kThreads - 1) / sats::kThreads));
  auto go = [&](auto fn) { fn<<<grid, sats::kThreads, 0, stream>>>(a); };
  auto of = [&](auto f) {
    constexpr int F = decltype(f)::value;
    if (esz == 2) wide ? go(sats::rope_kernel<uint16_t, 8, 1, F>) : go(sats::rope_kernel<uint16_t, 1, 2, F>);
    else wide ? go(sats::rope_kernel<float, 4, 1, F>) : go(sats::rope_kernel<float, 1, 2, F>);
  };
  const int form = cache ? form_of(cache) : sats::kPlain;
  if (form == sats::kE4m3) of(std::integral_constant<int, sats::kE4m3>{});
  else if (form == sats::kInt8) of(std::integral_constant<int, sats::kInt8>{});
  else of(std::integral_constant<int, sats::kPlain>{});
  return launched("rope_kernel");
}

// ------------------------------------------------------------- pages

struct PagesScratch {
  int32_t *off, *len_of, *ids, *to, *src, *dst, *valid, *ctl;
};
size_t pages_layout(char *base, int64_t n, int64_t n_pages, PagesScratch *out) {
  Carve c{base};
  PagesScratch s;
  const int64_t moves = std::max(n, n_pages);
  s.ctl = c.take<int32_t>(16);
  s.off = c.take<int32_t>(n);
  s.len_of = c.take<int32_t>(n);
  s.ids = c.take<int32_t>(n_pages);
  s.to = c.take<int32_t>(n_pages);
  s.src = c.take<int32_t>(moves);
  s.dst = c.take<int32_t>(moves);
  s.valid = c.take<int32_t>(n);
  if (out) *out = s;
  return c.off;
}

int check_pages(const sats_kv_cache *c, const sats_kv_pages *p, int64_t n, bool data) {
  int rc = check_cache(c, data);
  if (rc) return rc;
  if (!p) return fail(SATS_ERR_NULL, "pages must be non-null");
  if (p->n_seqs < 0 || p->max_pages < 0 || p->n_seqs > kMaxCount || p->max_pages > kMaxCount || n < 0 || n > 65535 ||
      p->max_pages * c->page_size >= (int64_t)1 << 31)
    return fail(SATS_ERR_SHAPE, "n_seqs or max_pages out of range, or more than 65535 items");
  if (p->n_seqs * std::max<int64_t>(p->max_pages, 1) >= (int64_t)1 << 38) return fail(SATS_ERR_SHAPE, "the page table is too large");
  if (!p->table || !p->len || !p->refs) return fail(SATS_ERR_NULL, "table, len and refs must be non-null");
  return SATS_OK;
}

sats::PagesArgs pages_args(const sats_kv_cache *c, const sats_kv_pages *p, const int32_t *seqs, const int32_t *other,
                           int64_t n, const PagesScratch *s) {
  sats::PagesArgs a{};
  a.table = p->table, a.len = p->len, a.refs = p->refs;
  a.n_seqs = p->n_seqs, a.max_pages = p->max_pages, a.n_pages = c->n_pages;
  a.page = (int)c->page_size, a.shift = log2_of(c->page_size);
  a.seqs = seqs, a.other = other, a.n = (int)n;
  if (s) a.off = s->off, a.len_of = s->len_of, a.ids = s->ids, a.to = s->to, a.src = s->src, a.dst = s->dst, a.valid = s->valid, a.ctl = s->ctl;
  return a;
}

// Workgroups that write `entries` of a table beside the moves of contents (kCopyGrid at most).
// Whether the launch takes them is asked before the plan, which changes the pages' state.
constexpr int64_t kCopyGrid = 8192;
int64_t table_grid(int64_t entries) { return (entries + sats::kThreads - 1) / sats::kThreads; }
int check_table(int64_t entries) {
  return table_grid(entries) + kCopyGrid <= kMaxGrid ? SATS_OK : fail(SATS_ERR_SHAPE, "the page table is too large for one call");
}

// Moves of contents, and with them `entries` of the table (TABLE, t).
template <int TABLE>
int copy_pages(const sats_kv_cache *c, const int32_t *src, const int32_t *dst, const int32_t *valid, const int32_t *ctl,
               int64_t n, const sats::PagesArgs &t, int64_t entries, hipStream_t stream) {
  const int64_t table = table_grid(entries);
  const int64_t waves = n * c->n_layers * 2 * c->n_kv_heads, per = sats::kThreads / 64;
  const int64_t grid = std::clamp<int64_t>((waves + per - 1) / per, 1, kCopyGrid);
  const sats_kv_cache8 *c8 = cache8_of(c);
  sats::CopyArgs a{static_cast<char *>(c->k), static_cast<char *>(c->v), c8 ? c8->k_scale : nullptr, c8 ? c8->v_scale : nullptr,
                   c->n_pages, c->n_layers, (int)c->n_kv_heads, (int)c->page_size, (int)(c->head_dim * stored_bytes(c)),
                   src, dst, valid, ctl, (int)n, (int)table};
  sats::pages_copy_kernel<TABLE><<<(unsigned)(table + grid), sats::kThreads, 0, stream>>>(a, t);
  return launched("pages_copy_kernel");
}

// ------------------------------------------------------------- sampling

struct SampleScratch {
  float *cmax;
  int32_t *cid;
  uint32_t *ccnt, *n_list, *hcnt;
  unsigned *arrived;
  sats::u64 *csum, *hsum, *list;
  sats::RowCut *cuts;
};
size_t sample_layout(char *base, int64_t n, int64_t vocab, SampleScratch *out) {
  Carve c{base};
  SampleScratch s;
  const int64_t chunks = (vocab + sats::kSampChunk - 1) / sats::kSampChunk;
  s.cmax = c.take<float>(n * chunks);
  s.cid = c.take<int32_t>(n * chunks);
  s.ccnt = c.take<uint32_t>(n * chunks);
  s.csum = c.take<sats::u64>(n * chunks);
  s.n_list = c.take<uint32_t>(n);
  s.arrived = c.take<unsigned>(n);
  s.cuts = c.take<sats::RowCut>(n);
  s.hcnt = c.take<uint32_t>(n * sats::kSampBins);
  s.hsum = c.take<sats::u64>(n * sats::kSampBins);
  s.list = c.take<sats::u64>(n * vocab);
  if (out) *out = s;
  return c.off;
}

// One launch, a workgroup a row, or four over chunks of the rows.  Measured (us, rows of
// bf16): 1 x 8000 11.2, 21.0; 1 x 32000 19.0, 21.7; 1 x 64000 29.1, 22.6; 64 x 8000 16.5, 30.4;
// 64 x 32000 32.4, 38.7; 64 x 64000 50.9, 43.1; 256 x 128256 96.3, 102.2: about 0.5 for 1000 ids
// of each round over the compute units, and 16 + 2.3 for a million ids of all rows.
bool sample_by_rows(int64_t n, int64_t vocab) {
  return 0.5e-3 * vocab * std::max(1.0, n / 256.0) < 16.0 + 2.3e-6 * n * vocab;
}

// Rows of a pass: their lists are as long as the vocabulary.
constexpr int64_t kSampleRows = 512;
constexpr int64_t kMaxVocab = (int64_t)sats::kSampChunk * sats::kPickThreads;

template <typename T> void launch_sample(const sats::SampleArgs &a, bool wide, hipStream_t stream) {
  const dim3 grid((unsigned)((a.chunks + a.span - 1) / a.span), (unsigned)a.n);
  constexpr int V = 16 / sizeof(T);
  if (sample_by_rows(a.n, a.vocab)) {
    auto kernel = wide ? sats::sample_row_kernel<T, V> : sats::sample_row_kernel<T, 1>;
    kernel<<<(unsigned)a.n, sats::kPickThreads, 0, stream>>>(a);
    return;
  }
  if (wide) {
    sats::sample_max_kernel<T, V><<<grid, sats::kSampThreads, 0, stream>>>(a);
    sats::sample_hist_kernel<T, V><<<grid, sats::kSampThreads, 0, stream>>>(a);
    sats::sample_cut_kernel<T, V><<<grid, sats::kSampThreads, 0, stream>>>(a);
  } else {
    sats::sample_max_kernel<T, 1><<<grid, sats::kSampThreads, 0, stream>>>(a);
    sats::sample_hist_kernel<T, 1><<<grid, sats::kSampThreads, 0, stream>>>(a);
    sats::sample_cut_kernel<T, 1><<<grid, sats::kSampThreads, 0, stream>>>(a);
  }
  sats::sample_pick_kernel<T><<<(unsigned)a.n, sats::kPickThreads, 0, stream>>>(a);
}

// ------------------------------------------------------------- attention

// The arguments of an attention call, checked; *nothing where there is no row to compute.
int attend_args(const void *q, int64_t q_stride, const sats_kv_cache *cache, int64_t layer, const sats_kv_batch *batch,
                int64_t n_q_heads, float scale, int64_t window, int64_t n_sinks, void *out, float *lse, sats::AttendArgs *args,
                bool *nothing) {
  int rc = check_cache(cache, true);
  if (rc || (rc = check_batch(batch))) return rc;
  if (layer < 0 || layer >= cache->n_layers) return fail(SATS_ERR_SHAPE, "layer outside the cache");
  if (n_q_heads < 1 || n_q_heads > 4096 || n_q_heads % cache->n_kv_heads)
    return fail(SATS_ERR_SHAPE, "n_q_heads must be a multiple of the cache's heads, at most 4096");
  if (window < 0 || n_sinks < 0 || (n_sinks && !window)) return fail(SATS_ERR_ARG, "window and n_sinks must be >= 0, sinks need a window");
  if (!std::isfinite(scale)) return fail(SATS_ERR_ARG, "scale must be finite");
  *nothing = batch->n_tokens == 0;
  if (*nothing) return SATS_OK;
  if (!q || !out) return fail(SATS_ERR_NULL, "q and out must be non-null");
  const int esz = outer_bytes(cache);
  const int64_t row = n_q_heads * cache->head_dim, n = batch->n_tokens;
  if (q_stride < row) return fail(SATS_ERR_SHAPE, "q_stride is below the token's row");
  if (!on16(q) || !on16(out) || q_stride * esz % 16) return fail(SATS_ERR_ARG, "q, out and the rows of q must be 16-byte aligned");
  if (overlap(out, n * row * esz, q, span(n, q_stride, row, esz)) || in_cache(out, n * row * esz, cache))
    return fail(SATS_ERR_ARG, "out overlaps q or the cache");
  const int64_t lse_bytes = lse ? n * n_q_heads * (int64_t)sizeof(float) : 0;
  if (reinterpret_cast<uintptr_t>(lse) % sizeof(float) || overlap(lse, lse_bytes, q, span(n, q_stride, row, esz)) ||
      overlap(lse, lse_bytes, out, n * row * esz) || in_cache(lse, lse_bytes, cache))
    return fail(SATS_ERR_ARG, "lse must be 4-byte aligned, apart from q, out and the cache");
  if (std::min(batch->max_q_len, n) * (n_q_heads / cache->n_kv_heads) > 0x7fffff00)
    return fail(SATS_ERR_SHAPE, "too many rows for one call");
  sats::AttendArgs a{};
  a.q = q, a.q_stride = q_stride, a.out = out, a.lse = lse;
  a.k = layer_of(cache->k, cache, layer), a.v = layer_of(cache->v, cache, layer);
  if (const sats_kv_cache8 *c8 = cache8_of(cache))
    a.k_scale = layer_scales(c8->k_scale, cache, layer), a.v_scale = layer_scales(c8->v_scale, cache, layer);
  a.batch = batch_view(batch), a.pool = pool_view(cache);
  a.n_q = (int)n_q_heads, a.group = (int)(n_q_heads / cache->n_kv_heads), a.dim = (int)cache->head_dim;
  // (places are below 2^31)
  a.scale = scale, a.window = std::min(window, (int64_t)1 << 31), a.sinks = std::min(n_sinks, (int64_t)1 << 31);
  *nothing = batch->max_q_len == 0;
  *args = a;
  return SATS_OK;
}

int check_prefix(const sats_kv_prefix *p) {
  if (!p) return fail(SATS_ERR_NULL, "prefix must be non-null");
  if (p->n_groups < 0 || p->max_tokens < 0 || p->max_len < 0 || p->max_own < 0 || p->n_groups > 65535 || p->max_tokens > kMaxCount ||
      p->max_len >= (int64_t)1 << 31 || p->max_own >= (int64_t)1 << 31)
    return fail(SATS_ERR_SHAPE, "a prefix's sizes must be >= 0, at most 2^30 (groups 65535, lengths below 2^31)");
  if (p->n_groups > 0 && (!p->seq_start || !p->len)) return fail(SATS_ERR_NULL, "the prefix's seq_start and len must be non-null");
  return SATS_OK;
}
void prefix_args(const sats_kv_prefix *p, sats::AttendArgs *a) {
  a->n_groups = (int)p->n_groups, a->seq_start = p->seq_start, a->shared = p->len;
  a->max_tokens = std::min(p->max_tokens, a->batch.n_tokens), a->max_len = p->max_len, a->max_own = p->max_own;
}

// ------------------------------------------------------------- logits

int check_rules(const sats_logit_rules *r, int64_t n, int64_t vocab) {
  if (!r) return fail(SATS_ERR_NULL, "rules must be non-null");
  if (r->n_seqs < 0 || r->max_history < 0 || r->n_bias < 0 || r->n_masks < 0 || r->n_seqs > kMaxCount || r->n_masks > kMaxCount ||
      r->max_history >= (int64_t)1 << 31 || r->n_bias >= (int64_t)1 << 31)
    return fail(SATS_ERR_SHAPE, "the rules' sizes must be >= 0, at most 2^30 (lengths below 2^31)");
  if (r->max_history > 0 && n > 0) {
    if (!r->history) return fail(SATS_ERR_NULL, "history must be non-null");
    if (!r->history_len) return fail(SATS_ERR_NULL, "history needs history_len");
    if (r->history_stride < r->max_history) return fail(SATS_ERR_SHAPE, "history_stride is below max_history");
    if (r->history_stride >= (int64_t)1 << 31) return fail(SATS_ERR_SHAPE, "history_stride must be below 2^31");
    if (!r->seqs && r->n_seqs < n) return fail(SATS_ERR_SHAPE, "history has fewer rows than logits, and seqs is null");
  }
  if (r->n_bias > 0 && (!r->bias || !r->bias_ids || !r->bias_start)) return fail(SATS_ERR_NULL, "biases need bias_start, bias_ids and bias");
  if (r->n_masks > 0) {
    if (!r->masks) return fail(SATS_ERR_NULL, "masks must be non-null");
    if (r->mask_stride < (vocab + 31) / 32) return fail(SATS_ERR_SHAPE, "mask_stride is below a bit an id");
    if (r->mask_stride >= (int64_t)1 << 31) return fail(SATS_ERR_SHAPE, "mask_stride must be below 2^31");
    if (!r->mask_of && r->n_masks < n) return fail(SATS_ERR_SHAPE, "fewer masks than rows, and mask_of is null");
  }
  return SATS_OK;
}

}  // namespace

extern "C" {

int sats_qk_norm_rope(const void *q, int64_t q_stride, const void *k, int64_t k_stride, const void *q_norm,
                      const void *k_norm, float eps, const float *rope, int64_t n_pos, const int32_t *positions,
                      void *q_out, int64_t q_out_stride, void *k_out, int64_t k_out_stride, int64_t n_tokens,
                      int64_t n_q_heads, int64_t n_kv_heads, int64_t head_dim, int64_t rot_dim, int interleaved,
                      int elem_bytes, hipStream_t stream) {
  clear_error();
  if (elem_bytes != 2 && elem_bytes != 4) return fail(SATS_ERR_ARG, "elem_bytes must be 2 or 4");
  if (n_q_heads < 0 || n_q_heads > 4096 || n_kv_heads < 0 || n_kv_heads > 1024 || head_dim < 2 || head_dim > 256 ||
      rot_dim < 0 || rot_dim > head_dim)
    return fail(SATS_ERR_SHAPE, "heads, head_dim or rot_dim out of range");
  sats::RopeArgs a{};
  a.q = q, a.k = k, a.q_stride = q_stride, a.k_stride = k_stride;
  a.q_norm = q_norm, a.k_norm = k_norm, a.eps = eps;
  a.rope = rope, a.n_pos = n_pos, a.positions = positions;
  a.q_out = q_out, a.k_out = k_out, a.q_out_stride = q_out_stride, a.k_out_stride = k_out_stride;
  a.n_q = (int)n_q_heads, a.n_kv = (int)n_kv_heads, a.dim = (int)head_dim, a.rot = (int)rot_dim, a.pairs = interleaved;
  a.n_tokens = n_tokens;
  return run_rope(a, elem_bytes, nullptr, stream);
}

int sats_qkv_append(const void *q, int64_t q_stride, const void *k, int64_t k_stride, const void *v, int64_t v_stride,
                    const void *q_norm, const void *k_norm, float eps, const float *rope, int64_t n_pos,
                    const int32_t *positions, void *q_out, int64_t q_out_stride, const sats_kv_cache *cache,
                    int64_t layer, const sats_kv_batch *batch, int64_t n_q_heads, int64_t rot_dim, int interleaved,
                    hipStream_t stream) {
  clear_error();
  int rc = check_cache(cache, true);
  if (rc || (rc = check_batch(batch))) return rc;
  if (layer < 0 || layer >= cache->n_layers) return fail(SATS_ERR_SHAPE, "layer outside the cache");
  if (n_q_heads < 0 || n_q_heads > 4096 || rot_dim < 0 || rot_dim > cache->head_dim)
    return fail(SATS_ERR_SHAPE, "heads or rot_dim out of range");
  sats::RopeArgs a{};
  a.q = q, a.k = k, a.v = v, a.q_stride = q_stride, a.k_stride = k_stride, a.v_stride = v_stride;
  a.q_norm = q_norm, a.k_norm = k_norm, a.eps = eps;
  a.rope = rope, a.n_pos = n_pos, a.positions = positions;
  a.q_out = q_out, a.q_out_stride = q_out_stride;
  a.n_q = (int)n_q_heads, a.n_kv = (int)cache->n_kv_heads, a.dim = (int)cache->head_dim, a.rot = (int)rot_dim;
  a.pairs = interleaved;
  a.n_tokens = batch->n_tokens;
  a.k_pool = layer_of(cache->k, cache, layer), a.v_pool = layer_of(cache->v, cache, layer);
  if (const sats_kv_cache8 *c8 = cache8_of(cache))
    a.k_scale = layer_scales(c8->k_scale, cache, layer), a.v_scale = layer_scales(c8->v_scale, cache, layer);
  a.batch = batch_view(batch), a.pool = pool_view(cache);
  return run_rope(a, outer_bytes(cache), cache, stream);
}

int sats_paged_attention(const void *q, int64_t q_stride, const sats_kv_cache *cache, int64_t layer,
                         const sats_kv_batch *batch, int64_t n_q_heads, float scale, int64_t window, int64_t n_sinks,
                         void *out, float *lse, hipStream_t stream) {
  clear_error();
  sats::AttendArgs a{};
  bool nothing = false;
  const int rc = attend_args(q, q_stride, cache, layer, batch, n_q_heads, scale, window, n_sinks, out, lse, &a, &nothing);
  return rc || nothing ? rc : sats_host::run_attention(a, form_of(cache), outer_bytes(cache), stream);
}

int sats_prefix_attention(const void *q, int64_t q_stride, const sats_kv_cache *cache, int64_t layer,
                          const sats_kv_batch *batch, const sats_kv_prefix *prefix, int64_t n_q_heads, float scale,
                          int64_t window, int64_t n_sinks, void *out, float *lse, hipStream_t stream) {
  clear_error();
  sats::AttendArgs a{};
  bool nothing = false;
  int rc = check_prefix(prefix);
  if (rc || (rc = attend_args(q, q_stride, cache, layer, batch, n_q_heads, scale, window, n_sinks, out, lse, &a, &nothing)) || nothing)
    return rc;
  if (std::min(prefix->max_tokens, batch->n_tokens) * a.group > 0x7fffff00) return fail(SATS_ERR_SHAPE, "too many rows for one call");
  prefix_args(prefix, &a);
  return sats_host::run_prefix_attention(a, form_of(cache), outer_bytes(cache), stream);
}

int sats_cache_read(const sats_kv_cache *cache, int64_t layer, const sats_kv_batch *batch, void *k_out, int64_t k_stride,
                    void *v_out, int64_t v_stride, int elem_bytes, hipStream_t stream) {
  clear_error();
  int rc = check_cache(cache, true);
  if (rc || (rc = check_batch(batch))) return rc;
  if (layer < 0 || layer >= cache->n_layers) return fail(SATS_ERR_SHAPE, "layer outside the cache");
  if (elem_bytes != 2 && elem_bytes != 4) return fail(SATS_ERR_ARG, "elem_bytes must be 2 or 4");
  const int64_t n = batch->n_tokens, row = cache->n_kv_heads * cache->head_dim;
  if (n == 0 || (!k_out && !v_out)) return SATS_OK;
  if ((k_out && k_stride < row) || (v_out && v_stride < row)) return fail(SATS_ERR_SHAPE, "a token stride is below the token's row");
  const Rows k{k_out, k_stride, row}, v{v_out, v_stride, row};
  if (rows_overlap(k, v, n, elem_bytes)) return fail(SATS_ERR_ARG, "k_out and v_out overlap");
  for (const Rows &r : {k, v}) {
    if (r.p && reinterpret_cast<uintptr_t>(r.p) % elem_bytes) return fail(SATS_ERR_ARG, "k_out and v_out must be aligned to their elements");
    if (r.p && in_cache(r.p, span(n, r.stride, row, elem_bytes), cache)) return fail(SATS_ERR_ARG, "k_out or v_out overlaps the cache");
  }
  sats::ReadArgs a{};
  a.k = layer_of(cache->k, cache, layer), a.v = layer_of(cache->v, cache, layer);
  if (const sats_kv_cache8 *c8 = cache8_of(cache))
    a.k_scale = layer_scales(c8->k_scale, cache, layer), a.v_scale = layer_scales(c8->v_scale, cache, layer);
  a.k_out = k_out, a.v_out = v_out, a.k_stride = k_stride, a.v_stride = v_stride;
  a.batch = batch_view(batch), a.pool = pool_view(cache);
  a.dim = (int)cache->head_dim, a.chunks = a.dim / 8;
  const int64_t grid = (n * cache->n_kv_heads * a.chunks + sats::kThreads - 1) / sats::kThreads;
  if (grid > kMaxGrid) return fail(SATS_ERR_SHAPE, "too many rows for one call");
  const bool wide = on16(k_out) && on16(v_out) && k_stride * elem_bytes % 16 == 0 && v_stride * elem_bytes % 16 == 0;
  auto go = [&](auto fn) { fn<<<(unsigned)grid, sats::kThreads, 0, stream>>>(a); };
  auto of = [&](auto c, auto f) {
    using C = decltype(c);
    constexpr int F = decltype(f)::value;
    if (elem_bytes == 2) wide ? go(sats::cache_read_kernel<C, F, uint16_t, true>) : go(sats::cache_read_kernel<C, F, uint16_t, false>);
    else wide ? go(sats::cache_read_kernel<C, F, float, true>) : go(sats::cache_read_kernel<C, F, float, false>);
  };
  const int form = form_of(cache);
  if (form == sats::kE4m3) of(uint8_t{}, std::integral_constant<int, sats::kE4m3>{});
  else if (form == sats::kInt8) of(uint8_t{}, std::integral_constant<int, sats::kInt8>{});
  else if (cache->elem_bytes == 2) of(uint16_t{}, std::integral_constant<int, sats::kPlain>{});
  else of(float{}, std::integral_constant<int, sats::kPlain>{});
  return launched("cache_read_kernel");
}

int sats_cache_free(const sats_kv_cache *cache, const sats_kv_pages *pages, const int32_t *seqs, const int32_t *begin,
                    const int32_t *end, int64_t n, hipStream_t stream) {
  clear_error();
  int rc = check_pages(cache, pages, n, false);
  if (rc || n == 0) return rc;
  sats::PagesArgs a = pages_args(cache, pages, seqs, nullptr, n, nullptr);
  a.begin = begin, a.end = end;
  sats::pages_free_kernel<<<(unsigned)n, sats::kThreads, 0, stream>>>(a);
  return launched("pages_free_kernel");
}

int sats_cache_extend(const sats_kv_cache *cache, const sats_kv_pages *pages, const int32_t *seqs, const int32_t *add,
                      int64_t n, int32_t *status, hipStream_t stream) {
  clear_error();
  int rc = check_pages(cache, pages, n, true);
  if (rc || n == 0) return rc;
  if (!add) return fail(SATS_ERR_NULL, "add must be non-null");
  char *mem = nullptr;
  Turn turn;
  PagesScratch s;
  if ((rc = sats_host::serve_workspace(stream, pages_layout(nullptr, n, cache->n_pages, nullptr), &mem, &turn))) return rc;
  pages_layout(mem, n, cache->n_pages, &s);
  sats::PagesArgs a = pages_args(cache, pages, seqs, add, n, &s);
  a.status = status;
  sats::pages_plan_kernel<false><<<1, sats::kPlanThreads, 0, stream>>>(a);
  if ((rc = launched("pages_plan_kernel"))) return rc;
  return copy_pages<sats::PAGES_ONLY>(cache, s.src, s.dst, s.valid, s.ctl, n, a, 0, stream);
}

int sats_cache_fork(const sats_kv_cache *cache, const sats_kv_pages *pages, const int32_t *src, const int32_t *dst,
                    int64_t n, int32_t *status, hipStream_t stream) {
  clear_error();
  int rc = check_pages(cache, pages, n, true);
  if (rc || n == 0) return rc;
  if (!src || !dst) return fail(SATS_ERR_NULL, "src and dst must be non-null");
  if ((rc = check_table(n * pages->max_pages))) return rc;
  char *mem = nullptr;
  Turn turn;
  PagesScratch s;
  if ((rc = sats_host::serve_workspace(stream, pages_layout(nullptr, n, cache->n_pages, nullptr), &mem, &turn))) return rc;
  pages_layout(mem, n, cache->n_pages, &s);
  sats::PagesArgs a = pages_args(cache, pages, src, dst, n, &s);
  a.status = status;
  sats::pages_plan_kernel<true><<<1, sats::kPlanThreads, 0, stream>>>(a);
  if ((rc = launched("pages_plan_kernel"))) return rc;
  return copy_pages<sats::PAGES_FORK>(cache, s.src, s.dst, s.valid, s.ctl, n, a, n * pages->max_pages, stream);
}

int sats_cache_compact(const sats_kv_cache *cache, const sats_kv_pages *pages, int32_t *n_used, hipStream_t stream) {
  clear_error();
  int rc = check_pages(cache, pages, 0, true);
  if (rc || (rc = check_table(pages->n_seqs * pages->max_pages))) return rc;
  char *mem = nullptr;
  Turn turn;
  PagesScratch s;
  if ((rc = sats_host::serve_workspace(stream, pages_layout(nullptr, 0, cache->n_pages, nullptr), &mem, &turn))) return rc;
  pages_layout(mem, 0, cache->n_pages, &s);
  sats::PagesArgs a = pages_args(cache, pages, nullptr, nullptr, 0, &s);
  a.n_used = n_used;
  sats::pages_compact_plan_kernel<<<1, sats::kPlanThreads, 0, stream>>>(a);
  if ((rc = launched("pages_compact_plan_kernel"))) return rc;
  return copy_pages<sats::PAGES_REMAP>(cache, s.src, s.dst, nullptr, s.ctl, std::max<int64_t>(cache->n_pages / 2, 1), a,
                                       pages->n_seqs * pages->max_pages, stream);
}

int sats_cache_copy(const sats_kv_cache *cache, const int32_t *src_pages, const int32_t *dst_pages, int64_t n,
                    hipStream_t stream) {
  clear_error();
  const int rc = check_cache(cache, true);
  if (rc) return rc;
  if (n < 0 || n > kMaxCount) return fail(SATS_ERR_SHAPE, "n must be >= 0, at most 2^30");
  if (n == 0) return SATS_OK;
  if (!src_pages || !dst_pages) return fail(SATS_ERR_NULL, "src_pages and dst_pages must be non-null");
  return copy_pages<sats::PAGES_ONLY>(cache, src_pages, dst_pages, nullptr, nullptr, n, sats::PagesArgs{}, 0, stream);
}

int sats_sample(const void *logits, int elem_bytes, int64_t stride, int64_t n, int64_t vocab, const float *temperature,
                const int32_t *top_k, const float *top_p, const float *min_p, const float *u, int32_t *tokens,
                float *prob, int32_t *n_kept, hipStream_t stream) {
  clear_error();
  if (elem_bytes != 2 && elem_bytes != 4) return fail(SATS_ERR_ARG, "elem_bytes must be 2 or 4");
  if (n < 0 || n > 65535 || vocab < 1 || vocab > kMaxVocab) return fail(SATS_ERR_SHAPE, "need 0 <= n < 65536 and 1 <= vocab <= 2^22");
  if (n == 0) return SATS_OK;
  if (!logits || !u || !tokens) return fail(SATS_ERR_NULL, "logits, u and tokens must be non-null");
  if (stride < vocab) return fail(SATS_ERR_SHAPE, "stride is below vocab");
  char *mem = nullptr;
  Turn turn;
  SampleScratch s;
  const int64_t pass = std::min(n, kSampleRows);
  int rc = sats_host::serve_workspace(stream, sample_layout(nullptr, pass, vocab, nullptr), &mem, &turn);
  if (rc) return rc;
  sample_layout(mem, pass, vocab, &s);
  sats::SampleArgs a{};
  a.stride = stride, a.vocab = vocab;
  a.chunks = (int)((vocab + sats::kSampChunk - 1) / sats::kSampChunk);
  a.cmax = s.cmax, a.cid = s.cid, a.hsum = s.hsum, a.hcnt = s.hcnt, a.csum = s.csum, a.ccnt = s.ccnt;
  a.list = s.list, a.n_list = s.n_list, a.arrived = s.arrived, a.cuts = s.cuts;
  const bool wide = on16(logits) && stride * elem_bytes % 16 == 0;
  for (int64_t r = 0; r < n && !rc; r += pass) {
    auto at = [r](auto *p) { return p ? p + r : p; };
    a.logits = static_cast<const char *>(logits) + r * stride * elem_bytes;
    a.n = (int)std::min(pass, n - r);
    a.temperature = at(temperature), a.top_k = at(top_k), a.top_p = at(top_p), a.min_p = at(min_p), a.u = at(u);
    a.tokens = at(tokens), a.prob = at(prob), a.n_kept = at(n_kept);
    // chunks of a workgroup: about two workgroups per compute unit
    a.span = 1;
    while (a.span < sats::kSampSpan && a.n * a.chunks > kSlots * a.span) a.span *= 2;
    if (elem_bytes == 2) launch_sample<uint16_t>(a, wide, stream);
    else launch_sample<float>(a, wide, stream);
    rc = launched("sample kernels");
  }
  return rc;
}

int sats_adjust_logits(const void *logits, int elem_bytes, int64_t stride, const sats_logit_rules *rules, void *out,
                       int out_elem_bytes, int64_t out_stride, int64_t n, int64_t vocab, hipStream_t stream) {
  clear_error();
  if ((elem_bytes != 2 && elem_bytes != 4) || (out_elem_bytes != 2 && out_elem_bytes != 4))
    return fail(SATS_ERR_ARG, "elem_bytes must be 2 or 4");
  if (n < 0 || n > 65535 || vocab < 1 || vocab > kMaxVocab) return fail(SATS_ERR_SHAPE, "need 0 <= n < 65536 and 1 <= vocab <= 2^22");
  const int rc = check_rules(rules, n, vocab);
  if (rc || n == 0) return rc;
  if (!logits || !out) return fail(SATS_ERR_NULL, "logits and out must be non-null");
  if (stride < vocab || out_stride < vocab || stride > (int64_t)1 << 40 || out_stride > (int64_t)1 << 40)
    return fail(SATS_ERR_SHAPE, "a stride is below vocab, or too large");
  if (reinterpret_cast<uintptr_t>(logits) % elem_bytes || reinterpret_cast<uintptr_t>(out) % out_elem_bytes)
    return fail(SATS_ERR_ARG, "logits and out must be aligned to their elements");
  const int64_t in_bytes = span(n, stride, vocab, elem_bytes), out_bytes = span(n, out_stride, vocab, out_elem_bytes);
  const bool same = out == logits && (n == 1 || out_stride == stride) && out_elem_bytes == elem_bytes;
  if (!same && overlap(out, out_bytes, logits, in_bytes)) return fail(SATS_ERR_ARG, "out overlaps logits without being logits");
  sats_logit_rules r = *rules;
  if (!r.max_history) r.seqs = r.history = r.history_len = r.prompt_len = nullptr;
  if (!r.n_bias) r.bias_start = r.bias_ids = nullptr, r.bias = nullptr;
  if (!r.n_masks) r.masks = nullptr, r.mask_of = nullptr;
  const int64_t rows = r.seqs ? r.n_seqs : std::max(n, r.n_seqs);
  const struct {
    const void *p;
    int64_t bytes;
  } read[] = {{r.seqs, n * 4}, {r.history, r.history ? span(r.n_seqs, r.history_stride, r.max_history, 4) : 0}, {r.history_len, rows * 4},
              {r.prompt_len, rows * 4}, {r.repetition, n * 4}, {r.frequency, n * 4}, {r.presence, n * 4}, {r.bias_start, (n + 1) * 4},
              {r.bias_ids, r.n_bias * 4}, {r.bias, r.n_bias * 4}, {r.masks, r.n_masks * r.mask_stride * 4}, {r.mask_of, n * 4}};
  for (const auto &x : read)
    if (x.p && overlap(out, out_bytes, x.p, x.bytes)) return fail(SATS_ERR_ARG, "out overlaps the rules' arrays");
  sats::LogitArgs a{};
  a.logits = logits, a.out = out, a.stride = stride, a.out_stride = out_stride, a.vocab = vocab;
  a.seqs = r.seqs, a.history = r.history, a.history_len = r.history_len, a.prompt_len = r.prompt_len;
  a.n_seqs = r.n_seqs, a.history_stride = r.history_stride, a.max_history = r.max_history;
  a.repetition = r.repetition, a.frequency = r.frequency, a.presence = r.presence;
  a.bias_start = r.bias_start, a.bias_ids = r.bias_ids, a.bias = r.bias, a.n_bias = r.n_bias;
  a.masks = r.masks, a.mask_of = r.mask_of, a.n_masks = r.n_masks, a.mask_stride = r.mask_stride;
  a.in_place = same;
  const bool wide = on16(logits) && on16(out) && (n == 1 || (stride * elem_bytes % 16 == 0 && out_stride * out_elem_bytes % 16 == 0));
  const dim3 grid((unsigned)((vocab + sats::kLogitChunk - 1) / sats::kLogitChunk), (unsigned)n);
  const size_t lds = ((r.history ? 1 : 0) + (r.bias ? 1 : 0)) * sats::kLogitChunk * sizeof(float);
  auto go = [&](auto fn) { fn<<<grid, sats::kLogitThreads, lds, stream>>>(a); };
  auto of = [&](auto t, auto o) {
    using T = decltype(t);
    using O = decltype(o);
    wide ? go(sats::logits_kernel<T, O, 8>) : go(sats::logits_kernel<T, O, 1>);
  };
  if (elem_bytes == 2) out_elem_bytes == 2 ? of(uint16_t{}, uint16_t{}) : of(uint16_t{}, float{});
  else out_elem_bytes == 2 ? of(float{}, uint16_t{}) : of(float{}, float{});
  return launched("logits_kernel");
}

int sats_reserve_prefix(const sats_kv_cache *cache, const sats_kv_batch *batch, const sats_kv_prefix *prefix, int64_t n_q_heads,
                        hipStream_t stream) {
  clear_error();
  int rc = check_cache(cache, false);
  if (rc) return rc;
  if (!batch) return fail(SATS_ERR_NULL, "batch must be non-null");
  sats_kv_batch b = *batch;
  b.table = b.q_start = b.kv_len = reinterpret_cast<const int32_t *>(16);  // (sizes alone count here)
  if ((rc = check_batch(&b))) return rc;
  if (!prefix) return fail(SATS_ERR_NULL, "prefix must be non-null");
  sats_kv_prefix p = *prefix;
  p.seq_start = p.len = b.table;
  if ((rc = check_prefix(&p))) return rc;
  if (n_q_heads < 1 || n_q_heads > 4096 || n_q_heads % cache->n_kv_heads)
    return fail(SATS_ERR_SHAPE, "n_q_heads must be a multiple of the cache's heads, at most 4096");
  sats::AttendArgs a{};
  a.batch = batch_view(&b), a.pool = pool_view(cache);
  a.n_q = (int)n_q_heads, a.group = (int)(n_q_heads / cache->n_kv_heads), a.dim = (int)cache->head_dim;
  if (std::min(std::max(p.max_tokens, b.max_q_len), b.n_tokens) * a.group > 0x7fffff00) return fail(SATS_ERR_SHAPE, "too many rows for one call");
  prefix_args(&p, &a);
  size_t bytes = 0;
  if ((rc = sats_host::prefix_scratch(a, form_of(cache), outer_bytes(cache), &bytes))) return rc;
  bytes = std::max(bytes, sats_host::attention_scratch(cache->head_dim));
  char *mem = nullptr;
  Turn turn;
  return sats_host::serve_workspace(stream, bytes, &mem, &turn);
}

int sats_reserve_serving(int64_t max_items, int64_t n_pages, int64_t max_rows, int64_t vocab, int64_t head_dim,
                         hipStream_t stream) {
  clear_error();
  if (max_items < 0 || max_items > 65535 || n_pages < 0 || n_pages > kMaxCount || max_rows < 0 || max_rows > 65535 ||
      vocab < 0 || vocab > kMaxVocab || head_dim < 0 || head_dim > 256)
    return fail(SATS_ERR_SHAPE, "bad sizes for sats_reserve_serving");
  size_t bytes = head_dim ? sats_host::attention_scratch(head_dim) : 0;
  if (n_pages) bytes = std::max(bytes, pages_layout(nullptr, max_items, n_pages, nullptr));
  if (max_rows && vocab) bytes = std::max(bytes, sample_layout(nullptr, std::min(max_rows, kSampleRows), vocab, nullptr));
  char *mem = nullptr;
  Turn turn;
  return sats_host::serve_workspace(stream, bytes, &mem, &turn);
}

}  // extern "C"

// Host side of the serving operators declared in include/sats.h: argument checks,
// scratch memory and launches.
#include <hip/hip_runtime.h>

#include <algorithm>
#include <cmath>

#include "host.hpp"

#include "attend.hpp"
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

constexpr int64_t kMaxCount = (int64_t)1 << 30;
// Workgroups of 256 threads in a row of a launch, at most: HIP takes less than 2^32 threads there.
constexpr int64_t kMaxGrid = ((int64_t)1 << 24) - 1;
static_assert(sats::kThreads == 256, "");

// Rotation: waves that fill the chip.
constexpr int64_t kRopeWaves = 4096;
// Parts up to which one wave joins a row, four above.  us where the limit is 8, 16, 32, 64: a sequence
// of 4000 keys (16 parts) 12.2, 13.3, 13.3, 13.3; of 6000 12.6, 12.6, 14.5, 14.5; of 16000 (63) 22.5, 22.5,
// 22.5, 34.3; 128 new tokens on 4000, whose tiles have 128 rows, 38.9, 35.4, 35.3, 35.3.
constexpr int kJoinWave = 16;
// Attention: workgroups that the chip holds at once (two a compute unit; of the kernels for
// heads above 128 one, of the 16-row kernels for heads up to 96 three), which a launch that
// splits its tiles aims at: a few more would wait for a second round.  8 sequences of 2000 to 6000
// keys: 512 workgroups 30.8 us, 768 38.1.
// Tiles of 16 rows whose parts stay at kLongBlocks blocks or more are split over up to
// kSlotsLong workgroups, since sequences of different lengths then share the chip more
// evenly (64 sequences of 500 to 8000 keys 156 -> 150 us).
// Key blocks of a part, at least, of 16 rows and of 128.  us for 4, 8, 16 blocks of 16 rows: a sequence
// of 500 keys 10.1, 11.8, 14.8; of 2000 11.5, 12.5, 16.4; of 4000 10.7, 13.3, 16.7; of 8000 16.0, 14.2, 20.1.
// For 2, 4, 8 blocks of 128: 64 new tokens on 500 18.8, 21.2, 26.6; on 2000 25.5, 23.6, 28.2; 256 on 1000
// 34.5, 34.2, 31.5; 512 alone 31.8, 31.0, 32.6.
constexpr int kSlots = 512, kSlotsLong = 2048, kLongBlocks = 24, kRowsLeast = 8, kTileLeast = 4;

int launched(const char *what) {
  const hipError_t e = hipGetLastError();
  return e == hipSuccess ? SATS_OK : fail(SATS_ERR_HIP, "%s: %s", what, hipGetErrorString(e));
}

// Bytes of an array of keys (or values) of every layer.
double pool_bytes(const sats_kv_cache *c) {
  return (double)c->n_layers * (double)c->n_pages * (double)c->n_kv_heads * (double)c->page_size * (double)c->head_dim *
         c->elem_bytes;
}

int check_cache(const sats_kv_cache *c, bool data) {
  if (!c) return fail(SATS_ERR_NULL, "cache must be non-null");
  if (data && (!c->k || !c->v)) return fail(SATS_ERR_NULL, "the cache's k and v must be non-null");
  if (c->elem_bytes != 2 && c->elem_bytes != 4) return fail(SATS_ERR_ARG, "elem_bytes must be 2 or 4");
  if (c->n_layers < 1 || c->n_pages < 1 || c->n_kv_heads < 1 || c->n_layers > 4096 || c->n_pages > kMaxCount ||
      c->n_kv_heads > 1024)
    return fail(SATS_ERR_SHAPE, "a cache has 1 to 4096 layers, 1 to 2^30 pages and 1 to 1024 heads");
  if (c->page_size < 1 || c->page_size > 4096 || (c->page_size & (c->page_size - 1)))
    return fail(SATS_ERR_SHAPE, "page_size must be a power of two up to 4096");
  if (c->head_dim < 8 || c->head_dim > 256 || c->head_dim % 8)
    return fail(SATS_ERR_SHAPE, "head_dim must be a multiple of 8 from 8 to 256");
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
  return static_cast<char *>(pool) + layer * c->n_pages * c->n_kv_heads * c->page_size * c->head_dim * c->elem_bytes;
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
  const int64_t all = (int64_t)pool_bytes(c);
  return overlap(p, n, c->k, all) || overlap(p, n, c->v, all);
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
  if (esz == 2) wide ? go(sats::rope_kernel<uint16_t, 8, 1>) : go(sats::rope_kernel<uint16_t, 1, 2>);
  else wide ? go(sats::rope_kernel<float, 4, 1>) : go(sats::rope_kernel<float, 1, 2>);
  return launched("rope_kernel");
}

// ------------------------------------------------------------- attention

// The split of a launch: row tiles of R rows, their number at most, and over how many
// workgroups a tile's blocks of `keys` keys go.
struct AttendPlan {
  int64_t tiles;
  int splits, per_split;
};
AttendPlan attend_plan(const sats::AttendArgs &a, int R, int keys, int least, int64_t max_q) {
  const sats::BatchView &b = a.batch;
  const int64_t per_seq = (max_q * a.group + R - 1) / R;
  AttendPlan p;
  p.tiles = b.n_tokens * a.group / R + b.n_seqs;
  if (b.n_seqs && per_seq <= p.tiles / b.n_seqs) p.tiles = b.n_seqs * per_seq;
  int64_t range = std::min<int64_t>(b.max_kv, b.max_pages << a.pool.shift);  // keys that a tile can see
  if (a.window) range = std::min(range, a.window + R / a.group + 1 + a.sinks + 2 * keys);
  const int64_t blocks = std::max<int64_t>(1, (range + keys - 1) / keys + 1);
  const int64_t wgs = std::max<int64_t>(1, p.tiles * a.pool.n_kv);
  int64_t slots = a.dim > 128 ? kSlots / 2 : kSlots;
  if (R == 16 && a.dim <= 96) slots = kSlots * 3 / 2;
  int64_t want = std::max<int64_t>(1, slots / wgs);
  if (R == 16) want = std::max(want, std::min<int64_t>(kSlotsLong / wgs, blocks / kLongBlocks));
  p.per_split = (int)std::max<int64_t>(least, (blocks + want - 1) / want);
  p.splits = (int)((blocks + p.per_split - 1) / p.per_split);
  return p;
}

size_t attend_bytes(const AttendPlan &p, int R, int n_kv, int dim) {
  return p.splits > 1 ? (size_t)p.tiles * n_kv * p.splits * R * (dim + 2) * sizeof(float) : 0;
}

template <typename T, int R, typename Kernel>
int launch_attention(sats::AttendArgs a, const AttendPlan &p, Kernel kernel, char *mem, hipStream_t stream) {
  const int64_t grid_x = p.tiles * a.pool.n_kv;
  a.splits = p.splits, a.per_split = p.per_split;
  a.part = reinterpret_cast<float *>(mem);
  a.part_ml = a.part + grid_x * p.splits * R * a.dim;
  kernel<<<dim3((unsigned)grid_x, (unsigned)p.splits), 256, 0, stream>>>(a);
  int rc = launched("attention kernel");
  if (rc || p.splits == 1) return rc;
  const int64_t rows = std::min<int64_t>(R, a.batch.max_q * a.group);
  if (p.splits > kJoinWave) sats::attend_join_kernel<T, R, 4><<<dim3((unsigned)grid_x, (unsigned)rows), 256, 0, stream>>>(a);
  else sats::attend_join_kernel<T, R, 1><<<dim3((unsigned)grid_x, (unsigned)((rows + 3) / 4)), 256, 0, stream>>>(a);
  return launched("attend_join_kernel");
}

// The second argument is true for heads of exactly the first one's dims only: such a kernel
// loads rows of that width.
typedef void (*AttendKernel)(sats::AttendArgs);
template <typename T> AttendKernel rows_kernel(int dim) {
  using namespace sats;
  return dim <= 64    ? (dim == 64 ? attend_rows_kernel<T, 64, true> : attend_rows_kernel<T, 64, false>)
         : dim <= 96  ? (dim == 96 ? attend_rows_kernel<T, 96, true> : attend_rows_kernel<T, 96, false>)
         : dim <= 128 ? (dim == 128 ? attend_rows_kernel<T, 128, true> : attend_rows_kernel<T, 128, false>)
                      : (dim == 256 ? attend_rows_kernel<T, 256, true> : attend_rows_kernel<T, 256, false>);
}
AttendKernel tile_kernel(int dim) {
  using namespace sats;
  return dim <= 64    ? (dim == 64 ? attend_tile_kernel<64, true> : attend_tile_kernel<64, false>)
         : dim <= 128 ? (dim == 128 ? attend_tile_kernel<128, true> : attend_tile_kernel<128, false>)
                      : (dim == 256 ? attend_tile_kernel<256, true> : attend_tile_kernel<256, false>);
}

// Sequences of at most 16 rows a cache head, and all of float32, go in tiles of 16 rows,
// the others in tiles of 128.  A batch of one sequence needs no launch for the former.
template <typename T> int run_attention(sats::AttendArgs a, hipStream_t stream) {
  constexpr bool bf16 = sizeof(T) == 2;
  AttendPlan small{}, large{};
  const bool any_large = bf16 && a.batch.max_q * a.group > 16;
  if (!any_large || a.batch.n_seqs > 1) {
    small = attend_plan(a, 16, sats::RowsOf<T>::kKeys, kRowsLeast, any_large ? 16 / a.group : a.batch.max_q);
  }
  if (any_large) large = attend_plan(a, sats::kTileRows, sats::kTileKeys, kTileLeast, a.batch.max_q);
  for (const AttendPlan *p : {&small, &large})
    if (p->tiles * a.pool.n_kv > kMaxGrid || p->splits > 65535) return fail(SATS_ERR_SHAPE, "too many rows for one call");
  const size_t bytes = std::max(attend_bytes(small, 16, a.pool.n_kv, a.dim),
                                attend_bytes(large, sats::kTileRows, a.pool.n_kv, a.dim));
  char *mem = nullptr;
  Turn turn;
  int rc = bytes ? sats_host::serve_workspace(stream, bytes, &mem, &turn) : SATS_OK;
  if (rc) return rc;
  if (small.tiles) {
    a.small = 1, a.large = !bf16;
    auto kernel = rows_kernel<T>(a.dim);
    if ((rc = launch_attention<T, 16>(a, small, kernel, mem, stream))) return rc;
  }
  if constexpr (bf16)
    if (large.tiles) {
      a.small = small.tiles == 0, a.large = 1;
      auto kernel = tile_kernel(a.dim);
      rc = launch_attention<T, sats::kTileRows>(a, large, kernel, mem, stream);
    }
  return rc;
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
  sats::CopyArgs a{static_cast<char *>(c->k), static_cast<char *>(c->v), c->n_pages, c->n_layers, (int)c->n_kv_heads,
                   (int)c->page_size, (int)(c->head_dim * c->elem_bytes), src, dst, valid, ctl, (int)n, (int)table};
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
  a.batch = batch_view(batch), a.pool = pool_view(cache);
  return run_rope(a, cache->elem_bytes, cache, stream);
}

int sats_paged_attention(const void *q, int64_t q_stride, const sats_kv_cache *cache, int64_t layer,
                         const sats_kv_batch *batch, int64_t n_q_heads, float scale, int64_t window, int64_t n_sinks,
                         void *out, float *lse, hipStream_t stream) {
  clear_error();
  int rc = check_cache(cache, true);
  if (rc || (rc = check_batch(batch))) return rc;
  if (layer < 0 || layer >= cache->n_layers) return fail(SATS_ERR_SHAPE, "layer outside the cache");
  if (n_q_heads < 1 || n_q_heads > 4096 || n_q_heads % cache->n_kv_heads)
    return fail(SATS_ERR_SHAPE, "n_q_heads must be a multiple of the cache's heads, at most 4096");
  if (window < 0 || n_sinks < 0 || (n_sinks && !window)) return fail(SATS_ERR_ARG, "window and n_sinks must be >= 0, sinks need a window");
  if (!std::isfinite(scale)) return fail(SATS_ERR_ARG, "scale must be finite");
  if (batch->n_tokens == 0) return SATS_OK;
  if (!q || !out) return fail(SATS_ERR_NULL, "q and out must be non-null");
  const int esz = cache->elem_bytes;
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
  a.batch = batch_view(batch), a.pool = pool_view(cache);
  a.n_q = (int)n_q_heads, a.group = (int)(n_q_heads / cache->n_kv_heads), a.dim = (int)cache->head_dim;
  // (places are below 2^31)
  a.scale = scale, a.window = std::min(window, (int64_t)1 << 31), a.sinks = std::min(n_sinks, (int64_t)1 << 31);
  if (batch->max_q_len == 0) return SATS_OK;
  return esz == 2 ? run_attention<uint16_t>(a, stream) : run_attention<float>(a, stream);
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

int sats_reserve_serving(int64_t max_items, int64_t n_pages, int64_t max_rows, int64_t vocab, int64_t head_dim,
                         hipStream_t stream) {
  clear_error();
  if (max_items < 0 || max_items > 65535 || n_pages < 0 || n_pages > kMaxCount || max_rows < 0 || max_rows > 65535 ||
      vocab < 0 || vocab > kMaxVocab || head_dim < 0 || head_dim > 256)
    return fail(SATS_ERR_SHAPE, "bad sizes for sats_reserve_serving");
  size_t bytes = 0;
  // attention: a launch that splits its tiles has at most kSlotsLong workgroups of 16 rows, kSlots of 128
  if (head_dim)
    bytes = (size_t)std::max(kSlotsLong * 16, kSlots * sats::kTileRows) * (head_dim + 2) * sizeof(float);
  if (n_pages) bytes = std::max(bytes, pages_layout(nullptr, max_items, n_pages, nullptr));
  if (max_rows && vocab) bytes = std::max(bytes, sample_layout(nullptr, std::min(max_rows, kSampleRows), vocab, nullptr));
  char *mem = nullptr;
  Turn turn;
  return sats_host::serve_workspace(stream, bytes, &mem, &turn);
}

}  // extern "C"

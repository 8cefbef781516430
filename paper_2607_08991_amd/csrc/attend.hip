// Host side of the attention over the paged cache: plans and launches, and the kernels of bf16 and
// float32 caches.
#include <hip/hip_runtime.h>

#include <algorithm>

#include "attend_host.hpp"

namespace sats_host {
namespace {

// Parts up to which one wave joins a row, four above.  us where the limit is 8, 16, 32, 64: a sequence
// of 4000 keys (16 parts) 12.2, 13.3, 13.3, 13.3; of 6000 12.6, 12.6, 14.5, 14.5; of 16000 (63) 22.5, 22.5,
// 22.5, 34.3; 128 new tokens on 4000, whose tiles have 128 rows, 38.9, 35.4, 35.3, 35.3.
constexpr int kJoinWave = 16;
// In phases: up to this many rows.  us for four waves and one: 2048 rows of 33 parts 118.8, 124.1; 12000 of up to 20 116, 100.
constexpr int kJoinRows = 4096;
// Attention: workgroups that the chip holds at once (two a compute unit; of the kernels for
// heads above 128 one, of the 16-row kernels for heads up to 96 three: up to 64 over 8 bits and in
// phases, and never beside tiles of 128 rows in one launch), which a launch that
// splits its tiles aims at: a few more would wait for a second round.  8 sequences of 2000 to 6000
// keys: 512 workgroups 30.8 us, 768 38.1; heads of 96 over E4M3 29.0, 36.5, and one of 32000 27.7, 35.4 (but 20 of
// 500 to 3000, of unlike lengths, 31.8, 29.0); 16 sequences on 4000 shared keys, heads of 64, 23.3, 26.9.
// Tiles of 16 rows whose parts stay at kLongBlocks blocks or more are split over up to
// kSlotsLong workgroups, since sequences of different lengths then share the chip more
// evenly (64 sequences of 500 to 8000 keys 156 -> 150 us).
// Key blocks of a part, at least, of 16 rows and of 128.  us for 4, 8, 16 blocks of 16 rows: a sequence
// of 500 keys 10.1, 11.8, 14.8; of 2000 11.5, 12.5, 16.4; of 4000 10.7, 13.3, 16.7; of 8000 16.0, 14.2, 20.1.
// For 2, 4, 8 blocks of 128: 64 new tokens on 500 18.8, 21.2, 26.6; on 2000 25.5, 23.6, 28.2; 256 on 1000
// 34.5, 34.2, 31.5; 512 alone 31.8, 31.0, 32.6.
// Of 8 bits: 4, 8, 16 blocks, a sequence of 4000 keys 12.3, 14.7, 17.2.  Tiles of 20 blocks (six sequences, a window of 512)
// 20.7 as they are and 25.6 in two, where the join takes 5.
constexpr int kRowsLeast8 = 4, kRowsAlone8 = 24;
constexpr int kSlots = 512, kSlotsLong = 2048, kLongBlocks = 24, kRowsLeast = 8, kTileLeast = 4;

// The split of a launch: row tiles of R rows, their number at most, and over how many
// workgroups a tile's blocks of `keys` keys go.
struct AttendPlan {
  int64_t tiles;
  int splits, per_split;
  int64_t most;  // workgroups, at most, of any call up to these sizes (fewer blocks can be more splits: 33 in 7, 32 in 8)
};
// Tiles of `units` sequences or groups with up to max_q tokens each, which see `range` keys at most.
// (least: blocks of a split; alone: blocks up to which a tile is not split where that would cost a join.)
// (three: head dims up to which a compute unit holds three of the 16-row kernel's workgroups.)
AttendPlan attend_plan(const sats::AttendArgs &a, int R, int keys, int least, int alone, int three, int64_t max_q, int64_t units, int64_t range) {
  const sats::BatchView &b = a.batch;
  const int64_t per_unit = (max_q * a.group + R - 1) / R;
  AttendPlan p;
  p.tiles = b.n_tokens * a.group / R + units;
  if (units && per_unit <= p.tiles / units) p.tiles = units * per_unit;
  range = std::min<int64_t>(range, std::min<int64_t>(b.max_kv, b.max_pages << a.pool.shift));  // keys that a tile can see
  // (rows of several sequences have windows far from each other)
  if (a.window && a.phase != sats::kShared) range = std::min(range, a.window + R / a.group + 1 + a.sinks + 2 * keys);
  const int64_t blocks = std::max<int64_t>(1, (range + keys - 1) / keys + 1);
  const int64_t wgs = std::max<int64_t>(1, p.tiles * a.pool.n_kv);
  int64_t slots = a.dim > 128 ? kSlots / 2 : kSlots;
  if (R == 16 && a.dim <= three) slots = kSlots * 3 / 2;
  // A group alone leaves half of the chip to its sequences' own keys where these are as many.  us for 512 and 256
  // workgroups: 64 sequences on 32000 keys with 100 to 2000 of their own 118.8, 108.3; with one each 82.8, 83.1 and on
  // 64000 128, 142; three groups of 500 to 9000 100, 124.
  if (R != 16 && a.phase == sats::kShared && units == 1 && b.n_seqs * a.max_own >= p.tiles * range) slots /= 2;
  int64_t want = std::max<int64_t>(1, slots / wgs);
  if (R == 16) want = std::max(want, std::min<int64_t>(kSlotsLong / wgs, blocks / kLongBlocks));
  const int64_t limit = R == 16 ? kSlotsLong : kSlots;
  p.most = wgs >= limit ? wgs : std::min(limit, wgs * ((blocks + least - 1) / least));
  if (a.phase == sats::kWhole && blocks <= alone) want = 1;
  p.per_split = (int)std::max<int64_t>(least, (blocks + want - 1) / want);
  p.splits = (int)((blocks + p.per_split - 1) / p.per_split);
  return p;
}

// The launches of a phase: of tiles of 16 rows and of 128 (tiles 0: none).  Units of at most 16 rows a cache
// head, and all of float32, go in tiles of 16 rows, the others in tiles of 128.  A single unit needs no
// launch for the former.
struct PhasePlan {
  AttendPlan small{}, large{};
};
PhasePlan phase_plan(const sats::AttendArgs &a, int form, int esz, int64_t max_q, int64_t units, int64_t range) {
  PhasePlan p;
  const bool any_large = esz == 2 && max_q * a.group > 16;
  const bool beside = a.phase != sats::kWhole && esz == 2 && std::max(a.batch.max_q, a.max_tokens) * a.group > 16;
  const int three = beside ? 0 : form || a.phase != sats::kWhole ? 64 : 96;
  if (!any_large || units > 1)
    p.small = attend_plan(a, 16, form || esz == 2 ? 32 : 16, form ? kRowsLeast8 : kRowsLeast, form ? kRowsAlone8 : 0, three, any_large ? 16 / a.group : max_q, units, range);
  if (any_large) p.large = attend_plan(a, sats::kTileRows, sats::kTileKeys, kTileLeast, 0, three, max_q, units, range);
  return p;
}
int check_plan(const sats::AttendArgs &a, const PhasePlan &p) {
  for (const AttendPlan *x : {&p.small, &p.large})
    if (x->tiles * a.pool.n_kv > kMaxGrid || x->splits > 65535) return fail(SATS_ERR_SHAPE, "too many rows for one call");
  return SATS_OK;
}

size_t part_rows(const AttendPlan &p, int R, int n_kv) { return (size_t)p.tiles * n_kv * p.splits * R; }
size_t attend_bytes(const AttendPlan &p, int R, int n_kv, int dim) {
  return p.splits > 1 ? part_rows(p, R, n_kv) * (dim + 2) * sizeof(float) : 0;
}
// The parts of a launch at *mem, which moves past them.
void place_parts(sats::AttendArgs &a, const AttendPlan &p, int R, char **mem) {
  const size_t rows = part_rows(p, R, a.pool.n_kv);
  a.splits = p.splits, a.per_split = p.per_split;
  a.part = reinterpret_cast<float *>(*mem);
  a.part_ml = a.part + rows * a.dim;
  *mem += (rows * (a.dim + 2) * sizeof(float) + 255) & ~size_t(255);
}

int launch_tiles(const sats::AttendArgs &a, const AttendPlan &p, AttendKernel kernel, hipStream_t stream) {
  kernel<<<dim3((unsigned)(p.tiles * a.pool.n_kv), (unsigned)p.splits), 256, 0, stream>>>(a);
  return launched("attention kernel");
}
// A join of up to `parts` parts of each row, by one wave a row or (kernel4) by four.
int launch_join(const sats::AttendArgs &a, const AttendPlan &p, int R, int parts, AttendKernel kernel1, AttendKernel kernel4,
                hipStream_t stream) {
  const unsigned grid_x = (unsigned)(p.tiles * a.pool.n_kv);
  const int64_t rows = std::min<int64_t>(R, a.batch.max_q * a.group);
  if (parts > kJoinWave) kernel4<<<dim3(grid_x, (unsigned)rows), 256, 0, stream>>>(a);
  else kernel1<<<dim3(grid_x, (unsigned)((rows + 3) / 4)), 256, 0, stream>>>(a);
  return launched("attention join");
}

// The second argument is true for heads of exactly the first one's dims only: such a kernel
// loads rows of that width.
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
// The join of tiles of R rows (those of 16 count blocks of the kernel's keys).
AttendKernel join_kernel(int R, int esz, int form, bool four) {
  using namespace sats;
  if (R != 16) return four ? attend_join_kernel<uint16_t, kTileRows, 4, kTileKeys> : attend_join_kernel<uint16_t, kTileRows, 1, kTileKeys>;
  if (esz == 2) return four ? attend_join_kernel<uint16_t, 16, 4, 32> : attend_join_kernel<uint16_t, 16, 1, 32>;
  if (form) return four ? attend_join_kernel<float, 16, 4, 32> : attend_join_kernel<float, 16, 1, 32>;
  return four ? attend_join_kernel<float, 16, 4, 16> : attend_join_kernel<float, 16, 1, 16>;
}
PhasesKernel join_phases_kernel(int esz, bool four) {
  using namespace sats;
  if (esz == 2) return four ? attend_join_phases_kernel<uint16_t, 4> : attend_join_phases_kernel<uint16_t, 1>;
  return four ? attend_join_phases_kernel<float, 4> : attend_join_phases_kernel<float, 1>;
}

struct PrefixPlan {
  PhasePlan pre, own;
};
PrefixPlan prefix_plan(sats::AttendArgs a, int form, int esz) {
  PrefixPlan p;
  a.phase = sats::kShared;
  p.pre = phase_plan(a, form, esz, a.max_tokens, a.n_groups, a.max_len);
  a.phase = sats::kOwn;
  p.own = phase_plan(a, form, esz, a.batch.max_q, a.batch.n_seqs, a.max_own);
  return p;
}
// The bytes of so many parts' rows, and of where each row's parts are.
size_t set_bytes(const sats::AttendArgs &a, size_t rows) {
  return rows * (a.dim + 2) * sizeof(float) + a.batch.n_tokens * a.n_q * sizeof(sats::RowParts);
}
constexpr size_t kTooMany = ~(size_t)0;
// The four sets, their parts from mem on; the bytes that these take, or kTooMany.
size_t place_sets(const sats::AttendArgs &a, const PrefixPlan &plan, int esz, char *mem, sats::PhaseArgs *out) {
  const AttendPlan *plans[4] = {&plan.pre.small, &plan.pre.large, &plan.own.small, &plan.own.large};
  size_t rows = 0;
  for (int i = 0; i < 4; ++i) {
    const AttendPlan &x = *plans[i];
    const bool there = x.tiles > 0;
    const size_t own = part_rows(x, i & 1 ? sats::kTileRows : 16, a.pool.n_kv);
    if (rows + own > 0x7fffffff) return kTooMany;
    out->set[i] = {x.tiles, x.splits, x.per_split, there && (!(i & 1) || !plans[i - 1]->tiles), there && ((i & 1) || esz != 2),
                   (int)rows, (int)own};
    rows += own;
  }
  out->part = reinterpret_cast<float *>(mem);
  out->part_ml = out->part + rows * a.dim;
  out->parts = reinterpret_cast<sats::RowParts *>(out->part_ml + rows * 2);
  return set_bytes(a, rows);
}

// Under a window the groups' rows of the table come behind the sets, at mem: their width, and the bytes that they take.
int64_t group_width(const sats::AttendArgs &a) {
  const int64_t top = std::min({a.max_len, a.batch.max_kv, a.batch.max_pages << a.pool.shift});
  return (top + a.pool.page - 1) >> a.pool.shift;
}
// (A wave reads 64 entries at a time, of the last row past its end too.)
size_t group_bytes(const sats::AttendArgs &a) { return ((size_t)a.n_groups * group_width(a) + 64) * sizeof(int32_t); }

// Workgroups of the launch of the four sets.
int64_t phase_wgs(const sats::AttendArgs &a, const sats::PhaseArgs &p) {
  double n = 0;
  for (const sats::PhaseSet &s : p.set) n += (double)s.tiles * a.pool.n_kv * s.splits;
  return (int64_t)std::min(n, 1e18);
}

// Workgroups of their join, by four waves a row or by one (more than kJoinRows rows).
int64_t join_wgs(const sats::AttendArgs &a, bool four) {
  const int64_t rows = a.batch.n_tokens * a.n_q;
  return four ? rows : (rows + 3) / 4;
}

// The bytes of the sets of a plan.
int prefix_sets(const sats::AttendArgs &a, const PrefixPlan &p, int esz, size_t *bytes) {
  int rc = check_plan(a, p.pre);
  if (rc || (rc = check_plan(a, p.own))) return rc;
  sats::PhaseArgs args;
  *bytes = place_sets(a, p, esz, nullptr, &args);
  if (*bytes == kTooMany || phase_wgs(a, args) > kMaxGrid || join_wgs(a, false) > kMaxGrid) return fail(SATS_ERR_SHAPE, "too many rows for one call");
  return SATS_OK;
}

}  // namespace

int run_attention(sats::AttendArgs a, int form, int esz, hipStream_t stream) {
  a.phase = sats::kWhole;
  const PhasePlan p = phase_plan(a, form, esz, a.batch.max_q, a.batch.n_seqs, (int64_t)1 << 31);
  int rc = check_plan(a, p);
  if (rc) return rc;
  const size_t bytes = std::max(attend_bytes(p.small, 16, a.pool.n_kv, a.dim),
                                attend_bytes(p.large, sats::kTileRows, a.pool.n_kv, a.dim));
  char *mem = nullptr;
  Turn turn;
  if (bytes && (rc = serve_workspace(stream, bytes, &mem, &turn))) return rc;
  if (p.small.tiles) {
    char *at = mem;
    place_parts(a, p.small, 16, &at);
    a.small = 1, a.large = esz != 2;
    const AttendKernel kernel = form == sats::kE4m3   ? e4m3_rows_kernel(esz, a.dim)
                                : form == sats::kInt8 ? int8_rows_kernel(esz, a.dim)
                                : esz == 2            ? rows_kernel<uint16_t>(a.dim) : rows_kernel<float>(a.dim);
    if ((rc = launch_tiles(a, p.small, kernel, stream))) return rc;
    if (p.small.splits > 1 && (rc = launch_join(a, p.small, 16, p.small.splits, join_kernel(16, esz, form, false),
                                                join_kernel(16, esz, form, true), stream)))
      return rc;
  }
  if (p.large.tiles) {
    char *at = mem;
    place_parts(a, p.large, sats::kTileRows, &at);
    a.small = p.small.tiles == 0, a.large = 1;
    const AttendKernel kernel = form == sats::kE4m3 ? e4m3_tile_kernel(a.dim) : form == sats::kInt8 ? int8_tile_kernel(a.dim) : tile_kernel(a.dim);
    if ((rc = launch_tiles(a, p.large, kernel, stream))) return rc;
    if (p.large.splits > 1)
      rc = launch_join(a, p.large, sats::kTileRows, p.large.splits, join_kernel(sats::kTileRows, esz, form, false),
                       join_kernel(sats::kTileRows, esz, form, true), stream);
  }
  return rc;
}

// (Under a window the groups' pages,) the groups' tiles and the sequences' tiles, and the joins of the latter's rows
// with both.
int run_prefix_attention(sats::AttendArgs a, int form, int esz, hipStream_t stream) {
  if (a.n_groups == 0 || a.max_len == 0 || a.max_tokens == 0) return run_attention(a, form, esz, stream);
  const PrefixPlan plan = prefix_plan(a, form, esz);
  size_t sets = 0;
  int rc = prefix_sets(a, plan, esz, &sets);
  if (rc) return rc;
  char *mem = nullptr;
  Turn turn;
  const int64_t width = a.window ? group_width(a) : 0, width_wgs = (width + 31) / 32;
  if (width_wgs > kMaxGrid) return fail(SATS_ERR_SHAPE, "too many pages for one call");
  if ((rc = serve_workspace(stream, sets + (width ? group_bytes(a) : 0), &mem, &turn))) return rc;
  if (width) {
    a.group_rows = reinterpret_cast<int32_t *>(mem + sets), a.group_width = width;
    sats::attend_group_pages_kernel<<<dim3((unsigned)width_wgs, (unsigned)a.n_groups), 256, 0, stream>>>(a);
    if ((rc = launched("attend_group_pages_kernel"))) return rc;
  }
  sats::PhaseArgs p;
  place_sets(a, plan, esz, mem, &p);
  const bool large = p.set[sats::kSharedLarge].tiles || p.set[sats::kOwnLarge].tiles;
  const PhasesKernel kernel = form == sats::kE4m3   ? e4m3_phases_kernel(esz, a.dim, large)
                              : form == sats::kInt8 ? int8_phases_kernel(esz, a.dim, large)
                                                    : phases_kernel(esz, a.dim, large);
  kernel<<<(unsigned)phase_wgs(a, p), 256, 0, stream>>>(a, p);
  if ((rc = launched("attention kernel"))) return rc;
  const int parts = std::max(plan.pre.small.splits, plan.pre.large.splits) + std::max(plan.own.small.splits, plan.own.large.splits);
  const bool four = parts > kJoinWave && a.batch.n_tokens * a.n_q <= kJoinRows;
  join_phases_kernel(esz, four)<<<(unsigned)join_wgs(a, four), 256, 0, stream>>>(a, p);
  return launched("attention join");
}

size_t attention_scratch(int64_t head_dim) {
  // a launch that splits its tiles has at most kSlotsLong workgroups of 16 rows, kSlots of 128
  return (size_t)std::max(kSlotsLong * 16, kSlots * sats::kTileRows) * (head_dim + 2) * sizeof(float);
}
int prefix_scratch(const sats::AttendArgs &a, int form, int esz, size_t *bytes) {
  const PrefixPlan plan = prefix_plan(a, form, esz);
  int rc = prefix_sets(a, plan, esz, bytes);
  if (rc) return rc;
  // a smaller batch can need more: it is split further, and of so few tokens that its tiles have 16 rows
  sats::AttendArgs few = a;
  few.batch.max_q = std::min<int64_t>(a.batch.max_q, 16 / a.group), few.max_tokens = std::min<int64_t>(a.max_tokens, 16 / a.group);
  const PrefixPlan small = prefix_plan(few, form, esz);
  size_t rows = 0;
  for (const PhasePlan PrefixPlan::*set : {&PrefixPlan::pre, &PrefixPlan::own})
    rows += std::max((plan.*set).small.most, (small.*set).small.most) * 16 + (plan.*set).large.most * sats::kTileRows;
  *bytes = std::max(*bytes, set_bytes(a, rows)) + group_bytes(a);
  return SATS_OK;
}

}  // namespace sats_host

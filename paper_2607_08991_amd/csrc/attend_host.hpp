// What the attention's translation units hand each other and the entry points.
#pragma once

#include "host.hpp"

#include "attend.hpp"

namespace sats_host {

typedef void (*AttendKernel)(sats::AttendArgs);
typedef void (*PhasesKernel)(sats::AttendArgs, sats::PhaseArgs);

// Kernels for heads of `dim`: of 8-bit caches; of calls in phases (large: with tiles of 128 rows among them).
AttendKernel e4m3_rows_kernel(int elem_bytes, int dim);
AttendKernel e4m3_tile_kernel(int dim);
AttendKernel int8_rows_kernel(int elem_bytes, int dim);
AttendKernel int8_tile_kernel(int dim);
PhasesKernel phases_kernel(int elem_bytes, int dim, bool large);
PhasesKernel e4m3_phases_kernel(int elem_bytes, int dim, bool large);
PhasesKernel int8_phases_kernel(int elem_bytes, int dim, bool large);

// Attention of a batch, q and out of elem_bytes over a cache of this format: enqueued, or an error.
int run_attention(sats::AttendArgs a, int form, int elem_bytes, hipStream_t stream);
// The same with a's groups of sequences that share prefixes.
int run_prefix_attention(sats::AttendArgs a, int form, int elem_bytes, hipStream_t stream);

// Scratch memory of any run_attention with heads of head_dim, and of any run_prefix_attention up to these sizes
// (a has no window: of any).
size_t attention_scratch(int64_t head_dim);
int prefix_scratch(const sats::AttendArgs &a, int form, int elem_bytes, size_t *bytes);

}  // namespace sats_host

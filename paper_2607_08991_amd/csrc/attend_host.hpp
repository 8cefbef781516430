// What the attention's translation units hand each other and the entry points.
#pragma once

#include "host.hpp"

#include "attend.hpp"

namespace sats_host {

typedef void (*AttendKernel)(sats::AttendArgs);

// Kernels for heads of `dim`: in phases, of bf16 or float32 caches; of 8-bit caches, every phase.
AttendKernel phase_rows_kernel(int elem_bytes, int dim);
AttendKernel phase_tile_kernel(int dim);
AttendKernel rows8_kernel(int form, int elem_bytes, int dim);
AttendKernel tile8_kernel(int form, int dim);

// Attention of a batch, q and out of elem_bytes over a cache of this format: enqueued, or an error.
int run_attention(sats::AttendArgs a, int form, int elem_bytes, hipStream_t stream);
// The same with a's groups of sequences that share prefixes.
int run_prefix_attention(sats::AttendArgs a, int form, int elem_bytes, hipStream_t stream);

// Scratch memory of any run_attention with heads of head_dim, and of these run_prefix_attention.
size_t attention_scratch(int64_t head_dim);
int prefix_scratch(const sats::AttendArgs &a, int form, int elem_bytes, size_t *bytes);

}  // namespace sats_host

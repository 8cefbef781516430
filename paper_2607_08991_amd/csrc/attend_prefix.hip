// Attention of bf16 and float32 caches in phases, for sequences that share prefixes: the kernels'
// instances.
#include <hip/hip_runtime.h>

#include "attend_host.hpp"

namespace sats_host {
namespace {

// (As in attend.hip the last argument is true for heads of exactly the one's dims before it.)
template <typename T> PhasesKernel rows_kernel(int dim) {
  using namespace sats;
  return dim <= 64    ? (dim == 64 ? attend_rows_phases_kernel<T, 64, true> : attend_rows_phases_kernel<T, 64, false>)
         : dim <= 128 ? (dim == 128 ? attend_rows_phases_kernel<T, 128, true> : attend_rows_phases_kernel<T, 128, false>)
                      : (dim == 256 ? attend_rows_phases_kernel<T, 256, true> : attend_rows_phases_kernel<T, 256, false>);
}

}  // namespace

PhasesKernel phases_kernel(int elem_bytes, int dim, bool large) {
  using namespace sats;
  if (!large) return elem_bytes == 2 ? rows_kernel<uint16_t>(dim) : rows_kernel<float>(dim);
  return dim <= 64    ? (dim == 64 ? attend_phases_kernel<64, true> : attend_phases_kernel<64, false>)
         : dim <= 128 ? (dim == 128 ? attend_phases_kernel<128, true> : attend_phases_kernel<128, false>)
                      : (dim == 256 ? attend_phases_kernel<256, true> : attend_phases_kernel<256, false>);
}

}  // namespace sats_host

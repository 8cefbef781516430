// Attention of bf16 and float32 caches in phases, for sequences that share prefixes: the kernels'
// instances.
#include <hip/hip_runtime.h>

#include "attend_host.hpp"

namespace sats_host {
namespace {

// (As in attend.hip the second argument is true for heads of exactly the first one's dims.)
template <typename T> AttendKernel rows_kernel(int dim) {
  using namespace sats;
  return dim <= 64    ? (dim == 64 ? attend_rows_kernel<T, 64, true, true> : attend_rows_kernel<T, 64, false, true>)
         : dim <= 128 ? (dim == 128 ? attend_rows_kernel<T, 128, true, true> : attend_rows_kernel<T, 128, false, true>)
                      : (dim == 256 ? attend_rows_kernel<T, 256, true, true> : attend_rows_kernel<T, 256, false, true>);
}

}  // namespace

AttendKernel phase_rows_kernel(int elem_bytes, int dim) {
  return elem_bytes == 2 ? rows_kernel<uint16_t>(dim) : rows_kernel<float>(dim);
}
AttendKernel phase_tile_kernel(int dim) {
  using namespace sats;
  return dim <= 64    ? (dim == 64 ? attend_tile_kernel<64, true, true> : attend_tile_kernel<64, false, true>)
         : dim <= 128 ? (dim == 128 ? attend_tile_kernel<128, true, true> : attend_tile_kernel<128, false, true>)
                      : (dim == 256 ? attend_tile_kernel<256, true, true> : attend_tile_kernel<256, false, true>);
}

}  // namespace sats_host

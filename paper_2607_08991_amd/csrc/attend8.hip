// Attention over 8-bit caches: the kernels' instances.
#include <hip/hip_runtime.h>

#include "attend8.hpp"
#include "attend_host.hpp"

namespace sats_host {
namespace {

// (As in attend.hip the last argument is true for heads of exactly the one's dims before it.)
template <typename T, int F> AttendKernel rows_kernel(int dim) {
  using namespace sats;
  return dim <= 64    ? (dim == 64 ? attend_rows8_kernel<T, F, 64, true> : attend_rows8_kernel<T, F, 64, false>)
         : dim <= 128 ? (dim == 128 ? attend_rows8_kernel<T, F, 128, true> : attend_rows8_kernel<T, F, 128, false>)
                      : (dim == 256 ? attend_rows8_kernel<T, F, 256, true> : attend_rows8_kernel<T, F, 256, false>);
}
template <int F> AttendKernel tile_kernel(int dim) {
  using namespace sats;
  return dim <= 64    ? (dim == 64 ? attend_tile8_kernel<F, 64, true> : attend_tile8_kernel<F, 64, false>)
         : dim <= 128 ? (dim == 128 ? attend_tile8_kernel<F, 128, true> : attend_tile8_kernel<F, 128, false>)
                      : (dim == 256 ? attend_tile8_kernel<F, 256, true> : attend_tile8_kernel<F, 256, false>);
}

}  // namespace

AttendKernel rows8_kernel(int form, int elem_bytes, int dim) {
  using namespace sats;
  if (elem_bytes == 2) return form == kE4m3 ? rows_kernel<uint16_t, kE4m3>(dim) : rows_kernel<uint16_t, kInt8>(dim);
  return form == kE4m3 ? rows_kernel<float, kE4m3>(dim) : rows_kernel<float, kInt8>(dim);
}
AttendKernel tile8_kernel(int form, int dim) { return form == sats::kE4m3 ? tile_kernel<sats::kE4m3>(dim) : tile_kernel<sats::kInt8>(dim); }

}  // namespace sats_host

// Attention over caches of INT8 codes: the kernels' instances.
#include <hip/hip_runtime.h>

#include "attend8.hpp"
#include "attend_host.hpp"

namespace sats_host {
namespace {

constexpr int F = sats::kInt8;

// (As in attend.hip the last argument is true for heads of exactly the one's dims before it.)
template <typename T> AttendKernel rows_kernel(int dim) {
  using namespace sats;
  return dim <= 64    ? (dim == 64 ? attend_rows8_kernel<T, F, 64, true> : attend_rows8_kernel<T, F, 64, false>)
         : dim <= 128 ? (dim == 128 ? attend_rows8_kernel<T, F, 128, true> : attend_rows8_kernel<T, F, 128, false>)
                      : (dim == 256 ? attend_rows8_kernel<T, F, 256, true> : attend_rows8_kernel<T, F, 256, false>);
}
template <typename T> PhasesKernel rows_phases_kernel(int dim) {
  using namespace sats;
  return dim <= 64    ? (dim == 64 ? attend_rows8_phases_kernel<T, F, 64, true> : attend_rows8_phases_kernel<T, F, 64, false>)
         : dim <= 128 ? (dim == 128 ? attend_rows8_phases_kernel<T, F, 128, true> : attend_rows8_phases_kernel<T, F, 128, false>)
                      : (dim == 256 ? attend_rows8_phases_kernel<T, F, 256, true> : attend_rows8_phases_kernel<T, F, 256, false>);
}

}  // namespace

AttendKernel int8_rows_kernel(int elem_bytes, int dim) { return elem_bytes == 2 ? rows_kernel<uint16_t>(dim) : rows_kernel<float>(dim); }
AttendKernel int8_tile_kernel(int dim) {
  using namespace sats;
  return dim <= 64    ? (dim == 64 ? attend_tile8_kernel<F, 64, true> : attend_tile8_kernel<F, 64, false>)
         : dim <= 128 ? (dim == 128 ? attend_tile8_kernel<F, 128, true> : attend_tile8_kernel<F, 128, false>)
                      : (dim == 256 ? attend_tile8_kernel<F, 256, true> : attend_tile8_kernel<F, 256, false>);
}
PhasesKernel int8_phases_kernel(int elem_bytes, int dim, bool large) {
  using namespace sats;
  if (!large) return elem_bytes == 2 ? rows_phases_kernel<uint16_t>(dim) : rows_phases_kernel<float>(dim);
  return dim <= 64    ? (dim == 64 ? attend8_phases_kernel<F, 64, true> : attend8_phases_kernel<F, 64, false>)
         : dim <= 128 ? (dim == 128 ? attend8_phases_kernel<F, 128, true> : attend8_phases_kernel<F, 128, false>)
                      : (dim == 256 ? attend8_phases_kernel<F, 256, true> : attend8_phases_kernel<F, 256, false>);
}

}  // namespace sats_host

// The stand-in runtime for calls from several threads: its log, memory and launch
// configurations are safe to use from any thread, every launch names its thread (`by K`,
// set with fake_thread) and gives the others time to come in between before it returns.
#define hipLaunchKernel one_hipLaunchKernel
#define hipExtLaunchKernel one_hipExtLaunchKernel
#define hipMalloc one_hipMalloc
#define hipFree one_hipFree
#define hipStreamSynchronize one_hipStreamSynchronize
#define hipDeviceSynchronize one_hipDeviceSynchronize
#define hipMemsetAsync one_hipMemsetAsync
#define __hipPushCallConfiguration one_push
#define __hipPopCallConfiguration one_pop
#include "fake_hip.cpp"
#undef hipLaunchKernel
#undef hipExtLaunchKernel
#undef hipMalloc
#undef hipFree
#undef hipStreamSynchronize
#undef hipDeviceSynchronize
#undef hipMemsetAsync
#undef __hipPushCallConfiguration
#undef __hipPopCallConfiguration

#include <chrono>
#include <cstdlib>
#include <mutex>
#include <new>
#include <thread>

namespace {
std::mutex g_mu;
thread_local int g_thread = 0;
thread_local Dim g_my_grid, g_my_block;
thread_local size_t g_my_shared;
thread_local void *g_my_stream;

int launch_by(const void *f, Dim grid) {
  {
    std::lock_guard<std::mutex> lk(g_mu);
    g_log += "by " + std::to_string(g_thread) + "\n";
    launch(f, grid);
  }
  std::this_thread::sleep_for(std::chrono::milliseconds(2));
  return 0;
}
}  // namespace

// Host memory that runs out: while fake_no_memory is set, nothing can be allocated with `new`.
namespace {
bool g_no_memory = false;
}
void *operator new(size_t n) {
  void *p = g_no_memory ? nullptr : malloc(n ? n : 1);
  if (!p) throw std::bad_alloc();
  return p;
}
void operator delete(void *p) noexcept { free(p); }
void operator delete(void *p, size_t) noexcept { free(p); }

extern "C" {
void fake_no_memory(int on) { g_no_memory = on; }
void fake_thread(int k) { g_thread = k; }
int hipLaunchKernel(const void *f, Dim grid, Dim, void **, size_t, void *) { return launch_by(f, grid); }
int hipExtLaunchKernel(const void *f, Dim grid, Dim, void **, size_t, void *, void *, void *, int) {
  return launch_by(f, grid);
}
int __hipPushCallConfiguration(Dim grid, Dim block, size_t shared, void *stream) {
  g_my_grid = grid, g_my_block = block, g_my_shared = shared, g_my_stream = stream;
  return 0;
}
int __hipPopCallConfiguration(Dim *grid, Dim *block, size_t *shared, void **stream) {
  *grid = g_my_grid, *block = g_my_block, *shared = g_my_shared, *stream = g_my_stream;
  return 0;
}
int hipMalloc(void **p, size_t n) {
  std::lock_guard<std::mutex> lk(g_mu);
  return one_hipMalloc(p, n);
}
int hipFree(void *p) {
  std::lock_guard<std::mutex> lk(g_mu);
  return one_hipFree(p);
}
int hipStreamSynchronize(void *s) {
  std::lock_guard<std::mutex> lk(g_mu);
  return one_hipStreamSynchronize(s);
}
int hipDeviceSynchronize() {
  std::lock_guard<std::mutex> lk(g_mu);
  return one_hipDeviceSynchronize();
}
int hipMemsetAsync(void *p, int v, size_t n, void *s) {
  std::lock_guard<std::mutex> lk(g_mu);
  return one_hipMemsetAsync(p, v, n, s);
}
}

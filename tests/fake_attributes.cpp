// fake_launches.cpp's runtime, with the most dynamic shared memory that a kernel may be launched with kept as the runtime keeps it: one number for a kernel, whoever sets
// it, 48 KB to begin with.  A launch that asks for more fails.  Threads that have set it wait for one another (fake_meet) before they go on.
#include <cuda.h>
#include <cuda_runtime.h>
#define cudaFuncSetAttribute fake_ignored_attribute
#define cudaLaunchKernelExC fake_noted_launch
extern "C" cudaError_t fake_ignored_attribute(const void*, cudaFuncAttribute, int);
extern "C" cudaError_t fake_noted_launch(const cudaLaunchConfig_t*, const void*, void**);
#include "fake_launches.cpp"
#undef cudaFuncSetAttribute
#undef cudaLaunchKernelExC
#include <chrono>
#include <condition_variable>
#include <mutex>

static std::mutex g_lock;
static std::condition_variable g_met;
static std::map<const void*, size_t> g_most;
static int g_awaited = 0, g_there = 0;

extern "C" {
__attribute__((visibility("default"))) void fake_meet(int threads) {
  std::lock_guard<std::mutex> hold(g_lock);
  g_awaited = threads;
  g_there = 0;
}
cudaError_t cudaFuncSetAttribute(const void* f, cudaFuncAttribute a, int v) {
  if (a != cudaFuncAttributeMaxDynamicSharedMemorySize) return cudaSuccess;
  std::unique_lock<std::mutex> hold(g_lock);
  g_most[f] = (size_t)v;
  if (++g_there >= g_awaited) g_met.notify_all();
  g_met.wait_for(hold, std::chrono::seconds(5), [] { return g_there >= g_awaited; });
  return cudaSuccess;
}
cudaError_t cudaLaunchKernelExC(const cudaLaunchConfig_t* c, const void* f, void** p) {
  std::lock_guard<std::mutex> hold(g_lock);
  const size_t most = g_most.count(f) ? g_most[f] : 49152;
  return c->dynamicSmemBytes > most ? cudaErrorInvalidValue : fake_noted_launch(c, f, p);
}
}

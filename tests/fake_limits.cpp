// A runtime that keeps the limits of kernels' dynamic shared memory as a device does, without a GPU:
// one for each kernel, whichever thread set it last.  Before a launch a test may make another call,
// which stands for another thread's.
#include <cuda_runtime_api.h>

#include <algorithm>
#include <map>

namespace {

constexpr size_t FREE = 48 * 1024;
int g_changed, g_refused, g_launches, g_inside;
size_t g_most;
void (*g_meanwhile)();
std::map<const void*, size_t> g_limit;

}  // namespace

extern "C" {

void fake_meanwhile(void (*call)()) { g_meanwhile = call; }
int fake_changed() { return g_changed; }    // limits that were set once more, to another value
int fake_refused() { return g_refused; }    // launches above their kernel's limit
int fake_launches() { return g_launches; }
size_t fake_most() { return g_most; }       // the largest launch's dynamic shared memory

cudaError_t cudaFuncSetAttribute(const void* f, cudaFuncAttribute which, int value) {
  if (which != cudaFuncAttributeMaxDynamicSharedMemorySize || value > 227 * 1024) return cudaErrorInvalidValue;
  const auto it = g_limit.find(f);
  g_changed += it != g_limit.end() && it->second != (size_t)value;
  g_limit[f] = (size_t)value;
  return cudaSuccess;
}
cudaError_t cudaLaunchKernelExC(const cudaLaunchConfig_t* c, const void* f, void**) {
  if (g_meanwhile && !g_inside) {
    g_inside = 1;
    g_meanwhile();
    g_inside = 0;
  }
  const auto it = g_limit.find(f);
  g_most = std::max(g_most, c->dynamicSmemBytes);
  if (c->dynamicSmemBytes > (it == g_limit.end() ? FREE : std::max(FREE, it->second))) {
    ++g_refused;
    return cudaErrorInvalidValue;
  }
  ++g_launches;
  return cudaSuccess;
}
void** __cudaRegisterFatBinary(void*) { return nullptr; }
void __cudaRegisterFatBinaryEnd(void**) {}
void __cudaUnregisterFatBinary(void**) {}
void __cudaRegisterFunction(void**, const char*, char*, const char*, int, void*, void*, void*, void*, int*) {}
cudaError_t __cudaPopCallConfiguration(void*, void*, size_t*, void*) { return cudaErrorInvalidValue; }
cudaError_t __cudaGetKernel(cudaKernel_t*, const void*) { return cudaErrorInvalidValue; }
cudaError_t __cudaLaunchKernel(cudaKernel_t, dim3, dim3, void**, size_t, cudaStream_t) { return cudaErrorInvalidValue; }

}  // extern "C"

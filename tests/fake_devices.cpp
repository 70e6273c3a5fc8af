// A runtime of several devices without a GPU: which is current, and what layer norm's launches
// ask of it on each.  A kernel may use more than 48 KB of shared memory, its own included, only
// on a device where the attribute that allows it was set.
#include <cuda_runtime_api.h>

#include <map>
#include <utility>

namespace {

constexpr size_t OWN_SMEM = 128;  // of the kernels whose shared memory is checked to the byte
int g_device, g_refused, g_launches;
unsigned g_grid, g_threads;
size_t g_smem;
std::map<std::pair<int, const void*>, size_t> g_allowed;

bool fits(const void* f, size_t dynamic) {
  const auto it = g_allowed.find({g_device, f});
  return dynamic + OWN_SMEM <= 48 * 1024 || (it != g_allowed.end() && dynamic <= it->second);
}
int held(int threads, size_t dynamic) {
  const int by_smem = (int)(228 * 1024 / (dynamic + OWN_SMEM + 1024)), by_threads = 2048 / threads;
  return by_smem < by_threads ? by_smem : by_threads;
}

}  // namespace

extern "C" {

void fake_device(int d) { g_device = d; }
int fake_refused() { return g_refused; }
int fake_launches() { return g_launches; }
// of the last launch: its grid, and how many blocks of it an SM holds
unsigned fake_grid() { return g_grid; }
int fake_held() { return held((int)g_threads, g_smem); }

cudaError_t cudaFuncSetAttribute(const void* f, cudaFuncAttribute which, int value) {
  if (which != cudaFuncAttributeMaxDynamicSharedMemorySize || value > 227 * 1024) return cudaErrorInvalidValue;
  g_allowed[{g_device, f}] = (size_t)value;
  return cudaSuccess;
}
cudaError_t cudaOccupancyMaxActiveBlocksPerMultiprocessorWithFlags(int* blocks, const void* f, int threads,
                                                                   size_t dynamic, unsigned) {
  *blocks = fits(f, dynamic) ? held(threads, dynamic) : 0;
  return cudaSuccess;
}
cudaError_t cudaLaunchKernelExC(const cudaLaunchConfig_t* c, const void* f, void**) {
  if (!fits(f, c->dynamicSmemBytes)) {
    ++g_refused;
    return cudaErrorInvalidValue;
  }
  ++g_launches;
  g_grid = c->gridDim.x;
  g_threads = c->blockDim.x;
  g_smem = c->dynamicSmemBytes;
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

// Keeps count of which device is current (the link's --wrap sends these two calls here), for a
// runtime that otherwise has one (fake_runtime.cpp).
#include <cuda_runtime_api.h>

static int g_current, g_launch_device = -1;

extern "C" {

int fake_current() { return g_current; }
void fake_make_current(int d) { g_current = d; }
// the device that was current at the last call of the runtime that works on a stream
int fake_worked_on() { return g_launch_device; }

cudaError_t __wrap_cudaSetDevice(int d) { return g_current = d, cudaSuccess; }
cudaError_t __wrap_cudaGetDevice(int* d) { return *d = g_current, cudaSuccess; }
cudaError_t __real_cudaStreamSynchronize(cudaStream_t s);
cudaError_t __wrap_cudaStreamSynchronize(cudaStream_t s) {
  g_launch_device = g_current;
  return __real_cudaStreamSynchronize(s);
}
cudaError_t __real_cudaMemsetAsync(void* p, int v, size_t n, cudaStream_t s);
cudaError_t __wrap_cudaMemsetAsync(void* p, int v, size_t n, cudaStream_t s) {
  g_launch_device = g_current;
  return __real_cudaMemsetAsync(p, v, n, s);
}
cudaError_t __real_cudaMalloc(void** p, size_t n);
cudaError_t __wrap_cudaMalloc(void** p, size_t n) {
  g_launch_device = g_current;
  return __real_cudaMalloc(p, n);
}

}  // extern "C"

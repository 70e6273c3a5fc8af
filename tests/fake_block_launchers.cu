// Stand-ins for the launchers of a block's operators (see fake_worker_launchers.cu).
#include "gba_internal.cuh"
#include "gba_worker.cuh"

extern "C" void fake_need(const void* p, size_t bytes);

static int g_block_launches;
extern "C" int fake_block_launches() { return g_block_launches; }

namespace gba {

cudaError_t launch_residual_norm(const ResNormArgs&, int32_t, int32_t, int, cudaStream_t) {
  ++g_block_launches;
  return cudaSuccess;
}
size_t residual_norm_grad_workspace(const ResNormArgs& a, int32_t, int32_t, int) { return (size_t)a.d * 16; }
cudaError_t launch_residual_norm_grad(const ResNormArgs& a, int32_t, int32_t, int, cudaStream_t) {
  ++g_block_launches;
  fake_need(a.parts, (size_t)a.d * 16);
  return cudaSuccess;
}
size_t scan_workspace(const ScanArgs& a, int32_t, int32_t, bool, int) { return 256 + (size_t)a.n * 4; }
cudaError_t launch_scan(const ScanArgs& a, int32_t, int32_t, bool, char* ws, int, cudaStream_t) {
  ++g_block_launches;
  fake_need(ws, 256 + (size_t)a.n * 4);
  return cudaSuccess;
}
cudaError_t launch_adamw(const gba_adamw_part*, int32_t, AdamWArgs a, int, cudaStream_t) {
  ++g_block_launches;
  fake_need(a.ticket, 4);
  return cudaSuccess;
}
cudaError_t launch_adamw_values(const gba_adamw_part*, int32_t, float* const*, float* const*, int, cudaStream_t) {
  ++g_block_launches;
  return cudaSuccess;
}

}  // namespace gba

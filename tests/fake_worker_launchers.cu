// Stand-ins for the launchers of the worker's operators (see fake_runtime.cpp): they run
// nothing, but check that the workspace they are given is live and large enough.
#include "gba_internal.cuh"
#include "gba_worker.cuh"

extern "C" void fake_need(const void* p, size_t bytes);

static int g_launches;
extern "C" int fake_launches() { return g_launches; }

namespace gba {

gba_status table_view(gba_handle* h, int32_t, TableView*) { return h ? GBA_E_STATE : GBA_E_ARG; }

cudaError_t launch_embed(const EmbedArgs& a, int32_t, int32_t, int, cudaStream_t) {
  ++g_launches;
  fake_need(a.err.step, 4);
  return cudaSuccess;
}
size_t embed_grad_workspace(const EmbedGradArgs& a, size_t* step_word) {
  *step_word = 64;
  return 128 + (size_t)a.n * (size_t)a.d;
}
cudaError_t launch_embed_grad(const EmbedGradArgs& a, char* ws, int64_t, int, cudaStream_t) {
  ++g_launches;
  fake_need(ws, 128 + (size_t)a.n * (size_t)a.d);
  fake_need(a.err.step, 4);
  return cudaSuccess;
}
size_t norm_workspace(int64_t n_parts, int) { return 256 + (size_t)n_parts * 8; }
cudaError_t launch_norm(const gba_grad_part*, int32_t n_parts, bool, float, float*, char* ws,
                        uint32_t* ticket, int, cudaStream_t) {
  ++g_launches;
  fake_need(ws, 256 + (size_t)n_parts * 8);
  fake_need(ticket, 4);
  return cudaSuccess;
}
cudaError_t launch_layer_norm(const LayerNormArgs&, int32_t, const RingWait&, int, cudaStream_t) {
  ++g_launches;
  return cudaSuccess;
}
size_t layer_norm_grad_workspace(const LayerNormArgs& a, int32_t, int) { return (size_t)a.d * 8; }
cudaError_t launch_layer_norm_grad(const LayerNormArgs& a, int32_t, const RingWait&, int, cudaStream_t) {
  ++g_launches;
  fake_need(a.parts, (size_t)a.d * 8);
  return cudaSuccess;
}

}  // namespace gba

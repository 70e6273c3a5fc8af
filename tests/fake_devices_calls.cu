// Calls of layer norm's launchers for a test without a GPU (see fake_devices.cpp).
#include "gba_internal.cuh"
#include "gba_worker.cuh"

extern "C" int fake_layer_norm(int64_t n, int32_t d, int64_t stride, int32_t type, int grad) {
  gba::LayerNormArgs a{};
  alignas(16) static char at[16];  // nothing is read: no kernel runs
  a.x = a.dy = a.gamma = a.y = at;
  a.mean = a.rstd = a.dgamma = a.dbeta = a.parts = reinterpret_cast<float*>(at);
  a.n = n;
  a.d = d;
  a.x_stride = a.y_stride = a.dy_stride = stride;
  a.param_type = GBA_F32;
  if (grad) return (int)gba::launch_layer_norm_grad(a, type, gba::RingWait{}, 152, nullptr);
  a.dy = nullptr;
  return (int)gba::launch_layer_norm(a, type, gba::RingWait{}, 152, nullptr);
}

// Calls of the launchers of a block's norms and scans for a test without a GPU (see fake_limits.cpp).
#include "gba_internal.cuh"
#include "gba_worker.cuh"

alignas(16) static char at[16];  // nothing is read: no kernel runs

extern "C" int fake_norm(int64_t n, int32_t d, int64_t stride, int32_t type, int32_t wide, int grad, int biases) {
  gba::ResNormArgs a{};
  a.x = a.r = a.g = a.dy = a.dz = a.zin = {at, stride};
  a.z = a.y = a.dx = a.dr = a.dg = {at, stride};
  a.stats = reinterpret_cast<float4*>(at);
  a.post_weight = a.pre_weight = at;
  a.parts = reinterpret_cast<float*>(at);
  for (int i = 0; i < 4; ++i) a.sums[i] = biases || i % 2 == 0 ? a.parts : nullptr;
  a.n = n;
  a.d = d;
  a.post = a.pre = GBA_NORM_RMS;
  a.gate = GBA_GATE_SILU;
  return (int)(grad ? gba::launch_residual_norm_grad(a, type, wide, 152, nullptr)
                    : gba::launch_residual_norm(a, type, wide, 152, nullptr));
}

extern "C" int fake_scan(int64_t n_seq, int64_t n, int32_t d, int64_t stride, int32_t type, int32_t out, int ragged,
                         int grad) {
  gba::ScanArgs a{};
  a.x = a.f = a.y = a.dy = {at, stride};
  a.out = a.df = {at, stride};
  a.n_seq = n_seq;
  a.n = n;
  a.d = d;
  a.offsets = ragged ? reinterpret_cast<const int64_t*>(at) : nullptr;
  return (int)gba::launch_scan(a, type, out, grad != 0, at, 152, nullptr);
}

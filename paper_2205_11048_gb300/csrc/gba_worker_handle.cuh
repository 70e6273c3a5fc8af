// The worker handle, its workspace and the checks of arguments that its operators share.
#pragma once

#include <cuda_runtime.h>

#include <cstdio>

#include "gba.h"
#include "gba_internal.cuh"
#include "gba_worker.cuh"

struct gba_worker {
  int device = 0;
  int num_sms = 152;
  cudaStream_t stream = nullptr;
  cudaEvent_t event = nullptr;  // orders a lookup in a server's table
  char* ws = nullptr;
  size_t ws_bytes = 0;
  // Workspaces that a larger one took the place of.  Graphs captured before hold their addresses.
  // One is at least 1.25 times the one before, and the first 256 bytes, so 128 are never reached.
  char* old_ws[128];
  int n_old = 0;
  uint32_t* words = nullptr;   // device: the latched errors, a ticket
  uint32_t* h_flag = nullptr;  // mapped pinned: something is latched
  gba::ErrSink sink{};
  char last_error[256] = "";
};

namespace gba {

constexpr int64_t WAIT_NS = 2000000000ll;  // bound of the kernels' waits
constexpr int32_t MAX_COLS = 1 << 20;

inline gba_status fail(gba_worker* w, gba_status s, const char* msg) {
  snprintf(w->last_error, sizeof w->last_error, "%s", msg);
  return s;
}

inline gba_status cuda_fail(gba_worker* w, cudaError_t e, const char* what) {
  snprintf(w->last_error, sizeof w->last_error, "%s: %s", what, cudaGetErrorString(e));
  cudaGetLastError();
  return e == cudaErrorMemoryAllocation ? GBA_E_OOM : GBA_E_CUDA;
}

// Makes the handle's device current for a call, and the caller's again at its end.
struct OnDevice {
  int before = -1;
  bool moved = false;
  explicit OnDevice(int device) {
    moved = cudaGetDevice(&before) == cudaSuccess && before != device;
    if (moved) cudaSetDevice(device);
  }
  ~OnDevice() {
    if (moved) cudaSetDevice(before);
  }
  OnDevice(const OnDevice&) = delete;
  OnDevice& operator=(const OnDevice&) = delete;
};

// The workspace, at least `bytes` of it.  What it replaces lives on until the handle is destroyed.
inline gba_status reserve(gba_worker* w, size_t bytes) {
  if (bytes <= w->ws_bytes) return GBA_OK;
  const size_t want = (bytes + bytes / 4 + 255) / 256 * 256;
  char* ws = nullptr;
  const cudaError_t e = cudaMalloc((void**)&ws, want);
  if (e != cudaSuccess) return cuda_fail(w, e, "allocate the worker's workspace");
  if (w->ws) w->old_ws[w->n_old++] = w->ws;
  w->ws = ws;
  w->ws_bytes = want;
  return GBA_OK;
}

inline const char* bad_matrix(const gba_matrix* m) {
  if (!m) return "a matrix is NULL";
  if (m->type != GBA_F32 && m->type != GBA_BF16 && m->type != GBA_F16) return "unknown type";
  if (m->rows < 0 || m->cols < 1 || m->cols > MAX_COLS) return "a matrix needs rows >= 0 and 1 <= cols <= 2^20";
  if (m->stride < m->cols) return "stride < cols";
  if (m->rows > 0 && m->stride > (int64_t)(1ll << 60) / m->rows) return "a matrix is too large";
  if (m->rows > 0 && !m->data) return "a matrix has no data";
  if ((uintptr_t)m->data % type_bytes(m->type) != 0) return "data not aligned to its type";
  return nullptr;
}

// Bytes from the first element to past the last.
inline uint64_t span(const gba_matrix* m) {
  return m->rows == 0 ? 0 : ((uint64_t)(m->rows - 1) * m->stride + m->cols) * type_bytes(m->type);
}

inline bool overlap(const void* a, uint64_t na, const void* b, uint64_t nb) {
  return na > 0 && nb > 0 && (uintptr_t)a < (uintptr_t)b + nb && (uintptr_t)b < (uintptr_t)a + na;
}

inline const char* bad_floats(const float* p) {
  return (uintptr_t)p % 4 != 0 ? "a float array is not 4-byte aligned" : nullptr;
}

inline const char* bad_param(const void* p, int32_t type) {
  if (type < GBA_F32 || type > GBA_F16) return "unknown param_type";
  return (uintptr_t)p % type_bytes(type) != 0 ? "a parameter is not aligned to its type" : nullptr;
}

inline const char* not_alike(const gba_matrix* a, const gba_matrix* b) {
  return a->rows != b->rows || a->cols != b->cols || a->type != b->type ? "matrices of different shape or type"
                                                                        : nullptr;
}

// May out be written while in is read?  Only where they are the same matrix, or apart.
inline const char* not_apart(const gba_matrix* out, const gba_matrix* in) {
  if (out->data == in->data && out->stride == in->stride) return nullptr;
  return overlap(out->data, span(out), in->data, span(in)) ? "an output overlaps an input" : nullptr;
}

}  // namespace gba

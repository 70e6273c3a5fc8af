// Internal declarations of the worker's operators (lookup, its gradient, norm and
// clipping, layer norm, and those of a block), shared by their translation units.
#pragma once

#include <cuda_bf16.h>
#include <cuda_fp16.h>

#include <string.h>

#include <type_traits>

#include "gba.h"
#include "gba_internal.cuh"

namespace gba {

using bf16 = __nv_bfloat16;
using f16 = __half;

// ---- types and vectors ------------------------------------------------------
inline size_t type_bytes(int32_t type) { return type == GBA_F32 ? 4 : 2; }

template <typename T>
__device__ __forceinline__ float to_float(T x) {
  if constexpr (sizeof(T) == 4)
    return x;
  else if constexpr (std::is_same_v<T, bf16>)
    return __bfloat162float(x);
  else
    return __half2float(x);
}
template <typename T>
__device__ __forceinline__ T from_float(float x) {
  if constexpr (sizeof(T) == 4)
    return x;
  else if constexpr (std::is_same_v<T, bf16>)
    return __float2bfloat16_rn(x);
  else
    return __float2half_rn(x);
}

template <int BYTES>
struct WordOf;
template <>
struct WordOf<2> { using type = uint16_t; };
template <>
struct WordOf<4> { using type = uint32_t; };
template <>
struct WordOf<8> { using type = uint2; };
template <>
struct WordOf<16> { using type = uint4; };

// V consecutive elements in accesses of up to 16 bytes; p is aligned to
// min(16, V * sizeof(T)) bytes.
template <typename T, int V>
struct Pack {
  static constexpr int B = V * (int)sizeof(T) < 16 ? V * (int)sizeof(T) : 16;
  static constexpr int W = V * (int)sizeof(T) / B;
  using Word = typename WordOf<B>::type;
  Word w[W];
  __device__ __forceinline__ void load(const T* p) {
#pragma unroll
    for (int i = 0; i < W; ++i) w[i] = reinterpret_cast<const Word*>(p)[i];
  }
  __device__ __forceinline__ void store(T* p) const {
#pragma unroll
    for (int i = 0; i < W; ++i) reinterpret_cast<Word*>(p)[i] = w[i];
  }
  __device__ __forceinline__ void get(float (&x)[V]) const {
    T t[V];
    memcpy(t, w, sizeof t);
#pragma unroll
    for (int i = 0; i < V; ++i) x[i] = to_float(t[i]);
  }
  __device__ __forceinline__ void set(const float (&x)[V]) {
    if constexpr (sizeof(T) == 2 && V % 2 == 0) {  // two in one conversion
      using Two = std::conditional_t<std::is_same_v<T, bf16>, __nv_bfloat162, __half2>;
      Two t[V / 2];
#pragma unroll
      for (int i = 0; i < V / 2; ++i) {
        if constexpr (std::is_same_v<T, bf16>)
          t[i] = __floats2bfloat162_rn(x[2 * i], x[2 * i + 1]);
        else
          t[i] = __floats2half2_rn(x[2 * i], x[2 * i + 1]);
      }
      memcpy(w, t, sizeof t);
    } else {
      T t[V];
#pragma unroll
      for (int i = 0; i < V; ++i) t[i] = from_float<T>(x[i]);
      memcpy(w, t, sizeof t);
    }
  }
};

// 16 bytes of a matrix from an address that is only aligned to its type, by the two aligned
// words that hold them, brought into place when they are used.  Rows of odd widths are read
// so: by single elements a warp would fetch 64 bytes at a time.
template <typename T>
struct Loose {
  static constexpr int V = 16 / (int)sizeof(T);
  uint4 w[2];
  uint32_t shift;  // bytes
  // n of the elements exist, at least one; words outside the matrix's bytes [lo, hi) are not touched.
  __device__ __forceinline__ void load(const T* p, int64_t n, const char* lo, const char* hi) {
    const uintptr_t at = (uintptr_t)p, base = at & ~(uintptr_t)15;
    if (base >= (uintptr_t)lo && base + 32 <= (uintptr_t)hi) {
      shift = (uint32_t)(at & 15);
      w[0] = reinterpret_cast<const uint4*>(base)[0];
      w[1] = reinterpret_cast<const uint4*>(base)[1];
    } else {
      T t[V] = {};
#pragma unroll
      for (int j = 0; j < V; ++j)
        if (j < n) t[j] = p[j];
      shift = 0;
      memcpy(w, t, sizeof t);
    }
  }
  __device__ __forceinline__ void get(float (&x)[V]) const {
    uint32_t v[8] = {w[0].x, w[0].y, w[0].z, w[0].w, w[1].x, w[1].y, w[1].z, w[1].w};
    if (shift & 8)
#pragma unroll
      for (int k = 0; k < 6; ++k) v[k] = v[k + 2];
    if (shift & 4)
#pragma unroll
      for (int k = 0; k < 5; ++k) v[k] = v[k + 1];
    if constexpr (sizeof(T) == 2)
#pragma unroll
      for (int k = 0; k < 4; ++k) v[k] = __funnelshift_r(v[k], v[k + 1], (shift & 2) * 8);
    T t[V];
    memcpy(t, v, sizeof t);
#pragma unroll
    for (int j = 0; j < V; ++j) x[j] = to_float(t[j]);
  }
};

// ---- two floats in one operation ---------------------------------------------------
struct f2 {
  unsigned long long u;
};
__device__ __forceinline__ f2 pair(float lo, float hi) {
  f2 r;
  asm("mov.b64 %0, {%1, %2};" : "=l"(r.u) : "f"(lo), "f"(hi));
  return r;
}
__device__ __forceinline__ void split(f2 a, float& lo, float& hi) {
  asm("mov.b64 {%0, %1}, %2;" : "=f"(lo), "=f"(hi) : "l"(a.u));
}
__device__ __forceinline__ f2 add2(f2 a, f2 b) {
  f2 r;
  asm("add.rn.f32x2 %0, %1, %2;" : "=l"(r.u) : "l"(a.u), "l"(b.u));
  return r;
}
__device__ __forceinline__ f2 mul2(f2 a, f2 b) {
  f2 r;
  asm("mul.rn.f32x2 %0, %1, %2;" : "=l"(r.u) : "l"(a.u), "l"(b.u));
  return r;
}
__device__ __forceinline__ f2 fma2(f2 a, f2 b, f2 c) {
  f2 r;
  asm("fma.rn.f32x2 %0, %1, %2, %3;" : "=l"(r.u) : "l"(a.u), "l"(b.u), "l"(c.u));
  return r;
}
__device__ __forceinline__ float both(f2 a) {
  float lo, hi;
  split(a, lo, hi);
  return lo + hi;
}

// The most elements (a power of two, at most `most`) that an access may take of rows of
// `cols` elements of `bytes` each, `stride` apart from `p` on.
inline int vector_of(int most, const void* p, int64_t stride, int64_t cols, size_t bytes) {
  int v = most;
  for (; v > 1; v >>= 1) {
    const uint64_t a = (uint64_t)v * bytes < 16 ? (uint64_t)v * bytes : 16;
    if (cols % v == 0 && (uintptr_t)p % a == 0 && (uint64_t)stride * bytes % a == 0) break;
  }
  return v;
}

// ---- launches ---------------------------------------------------------------
// The kernels of one call follow one another on the worker's stream.  Like the
// kernels of a step they are launched so that a kernel's blocks may be set up while
// the one before still runs; follow(), first in such a kernel, returns when every
// earlier kernel has completed.  Nothing that a kernel writes may be read through the
// read-only path by them: they use ordinary loads throughout.
__device__ __forceinline__ void follow() {
  asm volatile("griddepcontrol.wait;" ::: "memory");
  asm volatile("griddepcontrol.launch_dependents;" ::: "memory");
}
template <typename... P, typename... A>
inline cudaError_t launch_following(void (*kernel)(P...), dim3 grid, unsigned threads, size_t smem,
                                    cudaStream_t s, A... args) {
  cudaLaunchAttribute at[1];
  at[0].id = cudaLaunchAttributeProgrammaticStreamSerialization;
  at[0].val.programmaticStreamSerializationAllowed = 1;
  cudaLaunchConfig_t cfg{};
  cfg.gridDim = grid;
  cfg.blockDim = dim3(threads);
  cfg.dynamicSmemBytes = smem;
  cfg.stream = s;
  cfg.attrs = at;
  cfg.numAttrs = 1;
  return cudaLaunchKernelEx(&cfg, kernel, static_cast<P>(args)...);
}

// ---- the table of a server handle, as a reader sees it ------------------------
struct TableView {
  const float* w;
  int64_t rows;
  int32_t dim;
  int32_t id_mode;
  uint64_t mod_magic;
  const HashInfo* hinfo;
  cudaStream_t stream;  // ordered after every step enqueued so far
  int device;
};
// Of table t of h, after joining its steps into its stream (gba_host.cu).
gba_status table_view(gba_handle* h, int32_t t, TableView* v);

// ---- lookup -------------------------------------------------------------------
struct EmbedArgs {
  const void* w;
  int64_t w_stride;
  int64_t V;
  uint64_t mod_magic;
  const HashInfo* hinfo;  // HASH tables (float32)
  const int64_t* ids;
  int64_t n;
  int64_t pad_id;
  void* out;
  int64_t out_stride;
  int32_t d;
  int32_t id_mode;
  float scale;
  ErrSink err;
};
cudaError_t launch_embed(const EmbedArgs& a, int32_t type, int32_t out_type, int num_sms,
                         cudaStream_t s);

// ---- gradient of the lookup -----------------------------------------------------
struct EmbedGradArgs {
  const int64_t* ids;
  int64_t n;
  int64_t pad_id;
  const void* grad;
  int64_t stride;
  int32_t type;
  int32_t d;
  int64_t V;
  uint64_t mod_magic;
  int32_t id_mode;
  float scale;
  // message form (dense = null)
  int64_t* ids_out;
  float* rows_out;
  int64_t* n_out;
  // dense form
  float* dense;
  int64_t dense_stride;
  int32_t accumulate;
  ErrSink err;  // .step: the call's own word, within its workspace
};
// Workspace of a call, and where the call's error word is in it.
size_t embed_grad_workspace(const EmbedGradArgs& a, size_t* step_word);
cudaError_t launch_embed_grad(const EmbedGradArgs& a, char* ws, int64_t wait_ns, int num_sms,
                              cudaStream_t s);

// ---- norm and clipping ------------------------------------------------------------
// parts_at: the caller's list.  ws: norm_workspace() bytes; ticket: a zero word that is
// zero again afterwards.  clip: write the outputs too.
size_t norm_workspace(int64_t n_parts, int num_sms);
cudaError_t launch_norm(const gba_grad_part* parts, int32_t n_parts, bool clip, float max_norm,
                        float* norm, char* ws, uint32_t* ticket, int num_sms, cudaStream_t s);

// ---- layer norm ---------------------------------------------------------------------
struct LayerNormArgs {
  const void* x;
  int64_t x_stride;
  const void* gamma;
  const void* beta;
  void* y;  // dx of the gradient
  int64_t y_stride;
  const void* dy;
  int64_t dy_stride;
  float* mean;
  float* rstd;
  float* dgamma;
  float* dbeta;
  int64_t n;
  int32_t d;
  int32_t param_type;
  float eps;
  float* parts;  // workspace of the gradient
};
// Where a wait for a copy that runs out reports it, and its limit.
struct RingWait {
  ErrSink err;
  int64_t limit_ns;
};
cudaError_t launch_layer_norm(const LayerNormArgs& a, int32_t type, const RingWait& w, int num_sms,
                              cudaStream_t s);
size_t layer_norm_grad_workspace(const LayerNormArgs& a, int32_t type, int num_sms);
cudaError_t launch_layer_norm_grad(const LayerNormArgs& a, int32_t type, const RingWait& w, int num_sms,
                                   cudaStream_t s);

// ---- the end of a block and the norm before the next ----------------------------------
struct Rows {
  const void* p;  // null: not there
  int64_t stride;
};
struct OutRows {
  void* p;
  int64_t stride;
};
struct ResNormArgs {
  Rows x, r, g;     // the block's output, the residual, the gate
  OutRows z, y;
  float4* stats;
  Rows dy, dz, zin; // of the gradient, whose input z is
  OutRows dx, dr, dg;
  const void* post_weight;
  const void* post_bias;
  const void* pre_weight;
  const void* pre_bias;
  float* sums[4];   // gradients of those, in that order; null: not wanted
  float* parts;     // workspace of the gradient
  int64_t n;
  int32_t d;
  int32_t post, pre, gate, param_type;
  float eps, rscale, bscale;
};
// type: of x; wide: of the residual and z
cudaError_t launch_residual_norm(const ResNormArgs& a, int32_t type, int32_t wide, int num_sms, cudaStream_t s);
size_t residual_norm_grad_workspace(const ResNormArgs& a, int32_t type, int32_t wide, int num_sms);
cudaError_t launch_residual_norm_grad(const ResNormArgs& a, int32_t type, int32_t wide, int num_sms, cudaStream_t s);

// ---- gated scan -----------------------------------------------------------------------
struct ScanArgs {
  Rows x, f;
  Rows y;           // of the gradient
  Rows dy;
  OutRows out;      // y, or dx of the gradient
  OutRows df;
  const float* state;  // what comes in before a first row (the gradient's: after a last row), or null
  int64_t state_stride;
  float* last;         // what goes out behind a last row (before a first row), or null
  int64_t last_stride;
  const float* h0;     // the gradient's: the first states, or null
  int64_t h0_stride;
  const int64_t* lengths;
  const int64_t* offsets;
  int64_t n_seq, n;    // sequences, rows
  int32_t d;
  int32_t decay, tied;
  ErrSink err;
};
size_t scan_workspace(const ScanArgs& a, int32_t type, int32_t out_type, bool grad, int num_sms);
// out_type: of y (and dy)
cudaError_t launch_scan(const ScanArgs& a, int32_t type, int32_t out_type, bool grad, char* ws, int num_sms,
                        cudaStream_t s);

// ---- AdamW ------------------------------------------------------------------------------
struct AdamWArgs {
  float lr, beta1, beta2, rest1, rest2, eps;  // rest: 1 - beta
  double log1, log2;                          // logarithms of the betas
  const float* lr_now;
  const float* norm;
  float max_norm;
  int64_t* step;
  int32_t rounding;
  uint32_t* ticket;  // a zero word that is zero again afterwards
};
cudaError_t launch_adamw(const gba_adamw_part* parts, int32_t n_parts, AdamWArgs a, int num_sms, cudaStream_t s);
cudaError_t launch_adamw_values(const gba_adamw_part* parts, int32_t n_parts, float* const* m_out,
                                float* const* v_out, int num_sms, cudaStream_t s);

}  // namespace gba

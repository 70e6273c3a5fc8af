// The end of a block and the norm before the next, and their gradient:
//   u = (x - mx) rx wq + bq,  z = rs r + bs act(g) u,  y = (z - mz) rz wp + bp.
// Backwards, with gy = dy wp and zh = (z - mz) rz:
//   D = dz + rz (gy - mean(gy) - zh mean(gy zh)),  dr = rs D,  t = bs D,
//   dg = t u act'(g),  e = t act(g),  gu = e wq,  dx = rx (gu - mean(gu) - xh mean(gu xh)),
//   dwp = sum dy zh, dbp = sum dy, dwq = sum e xh, dbq = sum e over the rows;
// the means without a product only for layer norms, and no mean where there is no norm.
//
// Bound by HBM bandwidth: every input is read once and every output written once.  A row is
// held in the registers of a warp or a block; the rows of wider calls than those hold are
// read again from L2 by one block each.
#include <algorithm>

#include "gba_worker.cuh"

namespace gba {

namespace {

constexpr int CHAIN = 512;  // rows that one thread adds to a parameter's gradient in one chain

// V parameters from column c on, of a type known at run time.
template <int V>
__device__ __forceinline__ void params(const void* p, int32_t type, int c, float fill, float (&w)[V]) {
  if (!p) {
#pragma unroll
    for (int j = 0; j < V; ++j) w[j] = fill;
  } else if (type == GBA_F32) {
    Pack<float, V> k;
    k.load(static_cast<const float*>(p) + c);
    k.get(w);
  } else if (type == GBA_BF16) {
    Pack<bf16, V> k;
    k.load(static_cast<const bf16*>(p) + c);
    k.get(w);
  } else {
    Pack<f16, V> k;
    k.load(static_cast<const f16*>(p) + c);
    k.get(w);
  }
}

// The gate's factor, and its derivative.  1 / (1 + exp(-g)) and one minus it are formed from
// exp(-|g|), which neither overflows nor cancels.
__device__ __forceinline__ float gate_of(int32_t kind, float g, float& slope) {
  if (kind == GBA_GATE_MUL) {
    slope = 1.f;
    return g;
  }
  const float t = __expf(-fabsf(g)), q = __fdividef(1.f, 1.f + t);
  const float sig = g >= 0.f ? q : t * q, rest = g >= 0.f ? t * q : q;
  const float nan = g != g ? g : 0.f;
  if (kind == GBA_GATE_SIGMOID) {
    slope = sig * rest + nan;
    return sig + nan;
  }
  slope = sig * (1.f + g * rest);
  return g * sig;
}

// Sums over a row's threads: a warp, or the block.  red: 2 x 32 x N floats of shared memory,
// used in turns, so that one barrier a sum is enough.
template <int N, bool BLOCK>
__device__ __forceinline__ void row_sums(float (&v)[N], float* red, int& turn) {
#pragma unroll
  for (int o = 16; o > 0; o >>= 1)
#pragma unroll
    for (int i = 0; i < N; ++i) v[i] += __shfl_xor_sync(0xffffffffu, v[i], o);
  if constexpr (BLOCK) {
    const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5, warps = blockDim.x >> 5;
    float* buf = red + turn * (64);
    turn ^= 1;
    if (lane == 0)
#pragma unroll
      for (int i = 0; i < N; ++i) buf[i * 32 + warp] = v[i];
    __syncthreads();
#pragma unroll
    for (int i = 0; i < N; ++i) {
      v[i] = lane < warps ? buf[i * 32 + lane] : 0.f;
#pragma unroll
      for (int o = 16; o > 0; o >>= 1) v[i] += __shfl_xor_sync(0xffffffffu, v[i], o);
    }
  }
}

// Where a thread stands: which of the row's threads it is, and the rows it goes through.
template <bool BLOCK>
struct Place {
  int t, threads;
  int64_t row, step;
  __device__ __forceinline__ Place() {
    if constexpr (BLOCK) {
      t = threadIdx.x, threads = blockDim.x;
      row = blockIdx.x, step = gridDim.x;
    } else {
      const int warps = blockDim.x >> 5;
      t = threadIdx.x & 31, threads = 32;
      row = (int64_t)blockIdx.x * warps + (threadIdx.x >> 5), step = (int64_t)gridDim.x * warps;
    }
  }
};

template <typename T>
__device__ __forceinline__ const T* at(const Rows& m, int64_t row) {
  return static_cast<const T*>(m.p) + row * m.stride;
}
template <typename T>
__device__ __forceinline__ T* at(const OutRows& m, int64_t row) {
  return static_cast<T*>(m.p) + row * m.stride;
}

// ---- rows in shared memory -----------------------------------------------------------------
// A thread's pieces of a row, under way while the row before is worked on.  Each thread copies what
// it reads itself, so nothing is waited for but its own copies.
__device__ __forceinline__ void copy_async(void* to, const void* from) {
  asm volatile("cp.async.cg.shared.global [%0], [%1], 16;" ::"r"(smem_addr(to)), "l"(from) : "memory");
}
__device__ __forceinline__ void copies_begun() { asm volatile("cp.async.commit_group;" ::: "memory"); }
template <int N>  // all but the last N groups of this thread
__device__ __forceinline__ void copies_done() {
  asm volatile("cp.async.wait_group %0;" ::"n"(N) : "memory");
}

template <typename T, int V, int P, bool BLOCK>
struct Rowed {
  T* at;
  // the next matrix of a stage behind `base`, which moves on
  __device__ __forceinline__ Rowed(char*& base, int, const Place<BLOCK>&) {
    at = reinterpret_cast<T*>(base) + threadIdx.x * V;
    base += (size_t)blockDim.x * P * V * sizeof(T);
  }
  __device__ __forceinline__ void fetch(const Rows& m, int64_t row, int64_t, int d, const Place<BLOCK>& pl) const {
    const T* p = static_cast<const T*>(m.p) + row * m.stride;
#pragma unroll
    for (int k = 0; k < P; ++k) {
      const int c = (k * pl.threads + pl.t) * V;
      if (c < d) {
        T* to = at + (size_t)k * blockDim.x * V;
        copy_async(to, p + c);
        if constexpr (V * sizeof(T) > 16) copy_async(to + 16 / sizeof(T), p + c + 16 / sizeof(T));
      }
    }
  }
  __device__ __forceinline__ void aim(const Rows&, int64_t, int, const Place<BLOCK>&) {}
  __device__ __forceinline__ void get(int k, const Place<BLOCK>&, float (&x)[V]) const {
    Pack<T, V> w;
    w.load(at + (size_t)k * blockDim.x * V);
    w.get(x);
  }
};
// Rows that start anywhere: the aligned 16 bytes that hold them, copied by the row's threads together
// (so a barrier is needed before they are read, and one before they are filled again).  By single
// elements bf16 32,768 x 2,049 took 1,715 us backwards.
template <typename T, int P, bool BLOCK>
struct Rowed<T, 1, P, BLOCK> {
  char* at;
  const T* row;  // the row's first element
  int d;
  __host__ __device__ static constexpr size_t bytes(int d) { return ((size_t)d * sizeof(T) + 30) / 16 * 16; }
  __device__ __forceinline__ Rowed(char*& base, int cols, const Place<BLOCK>&) : d(cols) {
    at = base + (BLOCK ? 0 : (threadIdx.x >> 5) * bytes(d));
    base += (BLOCK ? 1 : blockDim.x >> 5) * bytes(d);
  }
  __device__ __forceinline__ void fetch(const Rows& m, int64_t r, int64_t n, int, const Place<BLOCK>& pl) const {
    const uintptr_t lo = (uintptr_t)m.p, hi = lo + ((n - 1) * m.stride + d) * (int64_t)sizeof(T);  // of the matrix
    const uintptr_t from = lo + r * m.stride * (int64_t)sizeof(T), to = from + (uintptr_t)d * sizeof(T);
    for (uintptr_t p = (from & ~(uintptr_t)15) + pl.t * 16; p < to; p += pl.threads * 16) {
      char* q = at + (p - (from & ~(uintptr_t)15));
      if (p >= lo && p + 16 <= hi) {
        copy_async(q, (const void*)p);
      } else {
        for (int b = 0; b < 16; b += (int)sizeof(T))
          if (p + b >= lo && p + b < hi) *reinterpret_cast<T*>(q + b) = *(const T*)(p + b);
      }
    }
  }
  __device__ __forceinline__ void aim(const Rows& m, int64_t r, int, const Place<BLOCK>&) {
    row = reinterpret_cast<const T*>(at + ((uintptr_t)(static_cast<const T*>(m.p) + r * m.stride) & 15));
  }
  __device__ __forceinline__ void get(int k, const Place<BLOCK>& pl, float (&x)[1]) const {
    const int c = k * pl.threads + pl.t;
    x[0] = c < d ? to_float(row[c]) : 0.f;
  }
};

// Single float32 elements stay in registers: a warp's are 128 bytes as they lie (5,003 x 1,001 44 us
// against 66 through shared memory).
template <int P, bool BLOCK>
struct Rowed<float, 1, P, BLOCK> {
  float v[P];
  __host__ __device__ static constexpr size_t bytes(int) { return 0; }
  __device__ __forceinline__ Rowed(char*&, int, const Place<BLOCK>&) {}
  __device__ __forceinline__ void fetch(const Rows&, int64_t, int64_t, int, const Place<BLOCK>&) const {}
  __device__ __forceinline__ void aim(const Rows& m, int64_t row, int d, const Place<BLOCK>& pl) {
    if (!m.p) return;
    const float* p = static_cast<const float*>(m.p) + row * m.stride;
#pragma unroll
    for (int k = 0; k < P; ++k) {
      const int c = k * pl.threads + pl.t;
      v[k] = c < d ? p[c] : 0.f;
    }
  }
  __device__ __forceinline__ void get(int k, const Place<BLOCK>&, float (&x)[1]) const { x[0] = v[k]; }
};

// A thread's parameters.  Where it has single elements it keeps them as floats in shared memory, in
// `most` arrays of P for each thread: their types are not asked for row by row.
template <int V, int P, bool BLOCK>
struct Params {
  const ResNormArgs& a;
  const float* held;
  __device__ __forceinline__ Params(const ResNormArgs& args, char* at, const Place<BLOCK>& pl) : a(args) {
    if constexpr (V == 1) {
      float* to = reinterpret_cast<float*>(at) + threadIdx.x;
      held = to;
      for (int k = 0; k < 4; ++k)
        for (int p = 0; p < P; ++p) {
          const int c = p * pl.threads + pl.t;
          float w[1] = {0.f};
          if (c < a.d) params<1>(of(k), a.param_type, c, k & 1 ? 0.f : 1.f, w);
          to[(k * P + p) * blockDim.x] = w[0];
        }
    }
  }
  __device__ __forceinline__ const void* of(int k) const {
    return k == 0 ? a.post_weight : k == 1 ? a.post_bias : k == 2 ? a.pre_weight : a.pre_bias;
  }
  // piece p, from column c on, of the post weight and bias and the pre weight and bias
  __device__ __forceinline__ void get(int k, int p, int c, float (&w)[V]) const {
    if constexpr (V == 1)
      w[0] = held[(k * P + p) * blockDim.x];
    else
      params<V>(of(k), a.param_type, c, k & 1 ? 0.f : 1.f, w);
  }
};
template <int V, int P>
constexpr size_t HELD_BYTES = V == 1 ? 4 * P * sizeof(float) : 0;  // of a thread

// Where a thread has single elements it goes through all its P, those past the row as zeros: a branch
// at each would let it work on one at a time.

// The threads of a row that read what others of them copied.
template <typename T, int V, bool BLOCK>
__device__ __forceinline__ void sync_row() {
  if constexpr (V == 1 && sizeof(T) == 2) {
    if constexpr (BLOCK)
      __syncthreads();
    else
      __syncwarp();
  }
}

// Shared memory of a block's rows: nt matrices of T and nr of R.
template <typename T, typename R, int V, int P>
__host__ __device__ constexpr size_t stage_bytes(int nt, int nr, int d, int threads, bool block) {
  if (V == 1) return (block ? 1 : threads / 32) * (nt * Rowed<T, 1, P, true>::bytes(d) + nr * Rowed<R, 1, P, true>::bytes(d));
  return (size_t)threads * V * P * (nt * sizeof(T) + nr * sizeof(R));
}

// ---- forward -------------------------------------------------------------------------
// The mean and the reciprocal deviation of a row; value(p, x) gives piece p.
template <int V, int P, bool BLOCK, typename F>
__device__ __forceinline__ float2 row_stats(F value, int32_t kind, const ResNormArgs& a, const Place<BLOCK>& at,
                                            float* red, int& turn) {
  if (kind == GBA_NORM_NONE) return make_float2(0.f, 1.f);
  const float inv = 1.f / (float)a.d;
  float mean = 0.f;
  if (kind == GBA_NORM_LAYER) {
    float s[1] = {0.f};
#pragma unroll
    for (int p = 0; p < P; ++p)
      if (V == 1 || (p * at.threads + at.t) * V < a.d) {
        float x[V];
        value(p, x);
#pragma unroll
        for (int j = 0; j < V; ++j) s[0] += x[j];
      }
    row_sums<1, BLOCK>(s, red, turn);
    mean = s[0] * inv;
  }
  float q[1] = {0.f};
#pragma unroll
  for (int p = 0; p < P; ++p)
    if (V == 1 || (p * at.threads + at.t) * V < a.d) {
      float x[V];
      value(p, x);
#pragma unroll
      for (int j = 0; j < V; ++j) {
        const float e = V > 1 || p * at.threads + at.t < a.d ? x[j] - mean : 0.f;
        q[0] = fmaf(e, e, q[0]);
      }
    }
  row_sums<1, BLOCK>(q, red, turn);
  return make_float2(mean, 1.f / sqrtf(q[0] * inv + a.eps));
}

// B: the most threads of a block that holds one row; 0: a row is a warp's
template <typename T, typename R, int V, int P, int B>
__global__ void __launch_bounds__(B ? B : 256, B == 1024 ? 1 : 4) k_residual_norm(ResNormArgs a) {
  constexpr bool BLOCK = B > 0;
  extern __shared__ __align__(16) char smem[];
  __shared__ float red[2 * 64];
  int turn = 0;
  follow();
  const Place<BLOCK> pl;
  using Tm = Rowed<T, V, P, BLOCK>;
  using Rm = Rowed<R, V, P, BLOCK>;
  const size_t bytes = stage_bytes<T, R, V, P>(2, 1, a.d, blockDim.x, BLOCK);
  auto fetch = [&](int64_t row, int stage) {
    char* base = smem + stage * bytes;
    const Rm r(base, a.d, pl);
    const Tm x(base, a.d, pl), g(base, a.d, pl);
    if (row < a.n) {
      x.fetch(a.x, row, a.n, a.d, pl);
      if (a.r.p) r.fetch(a.r, row, a.n, a.d, pl);
      if (a.g.p) g.fetch(a.g, row, a.n, a.d, pl);
    }
    copies_begun();
  };
  const Params<V, P, BLOCK> par(a, smem + 2 * bytes, pl);
  fetch(pl.row, 0);
  int stage = 0;
  for (int64_t row = pl.row; row < a.n; row += pl.step, stage ^= 1) {
    sync_row<T, V, BLOCK>();
    fetch(row + pl.step, stage ^ 1);
    copies_done<1>();
    sync_row<T, V, BLOCK>();
    char* base = smem + stage * bytes;
    Rm rs(base, a.d, pl);
    Tm xs(base, a.d, pl), gs(base, a.d, pl);
    xs.aim(a.x, row, a.d, pl), rs.aim(a.r, row, a.d, pl), gs.aim(a.g, row, a.d, pl);
    const float2 sx = row_stats<V, P, BLOCK>([&](int p, float (&x)[V]) { xs.get(p, pl, x); }, a.post, a, pl, red, turn);
    float z[P][V];
#pragma unroll
    for (int p = 0; p < P; ++p) {
      const int c = (p * pl.threads + pl.t) * V;
#pragma unroll
      for (int j = 0; j < V; ++j) z[p][j] = 0.f;
      if (V == 1 || c < a.d) {
        float x[V], w[V];
        xs.get(p, pl, x);
        par.get(0, p, c, w);
#pragma unroll
        for (int j = 0; j < V; ++j) z[p][j] = (x[j] - sx.x) * sx.y * w[j];
        if (a.post_bias) {
          par.get(1, p, c, w);
#pragma unroll
          for (int j = 0; j < V; ++j) z[p][j] += w[j];
        }
        if (a.gate != GBA_GATE_NONE) {
          gs.get(p, pl, x);
#pragma unroll
          for (int j = 0; j < V; ++j) {
            float slope;
            z[p][j] *= gate_of(a.gate, x[j], slope);
          }
        }
#pragma unroll
        for (int j = 0; j < V; ++j) z[p][j] *= a.bscale;
        if (a.r.p) {
          rs.get(p, pl, x);
#pragma unroll
          for (int j = 0; j < V; ++j) z[p][j] = fmaf(a.rscale, x[j], z[p][j]);
        }
        if (a.z.p) {
          Pack<R, V> o;
          o.set(z[p]);
          if (V > 1 || c < a.d) o.store(at<R>(a.z, row) + c);
        }
      }
    }
    const float2 sz = row_stats<V, P, BLOCK>(
        [&](int p, float (&x)[V]) {
#pragma unroll
          for (int j = 0; j < V; ++j) x[j] = z[p][j];
        },
        a.pre, a, pl, red, turn);
    if (a.stats && pl.t == 0) a.stats[row] = make_float4(sx.x, sx.y, sz.x, sz.y);
    if (a.y.p)
#pragma unroll
      for (int p = 0; p < P; ++p) {
        const int c = (p * pl.threads + pl.t) * V;
        if (V == 1 || c < a.d) {
          float w[V];
          par.get(2, p, c, w);
#pragma unroll
          for (int j = 0; j < V; ++j) z[p][j] = (z[p][j] - sz.x) * sz.y * w[j];
          if (a.pre_bias) {
            par.get(3, p, c, w);
#pragma unroll
            for (int j = 0; j < V; ++j) z[p][j] += w[j];
          }
          Pack<T, V> o;
          o.set(z[p]);
          if (V > 1 || c < a.d) o.store(at<T>(a.y, row) + c);
        }
      }
  }
  copies_done<0>();
}

constexpr int WIDE = 1024;

// Rows of any width: a block goes over its row once for each sum and once for the outputs.
template <typename T, typename R>
__global__ void __launch_bounds__(WIDE) k_residual_norm_wide(ResNormArgs a) {
  __shared__ float red[2 * 64];
  int turn = 0;
  follow();
  const float inv = 1.f / (float)a.d;
  for (int64_t row = blockIdx.x; row < a.n; row += gridDim.x) {
    float2 sx = make_float2(0.f, 1.f), sz = sx;
    auto x_of = [&](int c) { return to_float(at<T>(a.x, row)[c]); };
    auto z_of = [&](int c) {
      float w[1], b[1], slope;
      params<1>(a.post_weight, a.param_type, c, 1.f, w);
      params<1>(a.post_bias, a.param_type, c, 0.f, b);
      float u = fmaf((x_of(c) - sx.x) * sx.y, w[0], b[0]);
      if (a.gate != GBA_GATE_NONE) u *= gate_of(a.gate, to_float(at<T>(a.g, row)[c]), slope);
      u *= a.bscale;
      return a.r.p ? fmaf(a.rscale, to_float(at<R>(a.r, row)[c]), u) : u;
    };
    auto stats = [&](int32_t kind, auto value) {
      if (kind == GBA_NORM_NONE) return make_float2(0.f, 1.f);
      float mean = 0.f;
      if (kind == GBA_NORM_LAYER) {
        float s[1] = {0.f};
        for (int c = threadIdx.x; c < a.d; c += WIDE) s[0] += value(c);
        row_sums<1, true>(s, red, turn);
        mean = s[0] * inv;
      }
      float q[1] = {0.f};
      for (int c = threadIdx.x; c < a.d; c += WIDE) {
        const float e = value(c) - mean;
        q[0] = fmaf(e, e, q[0]);
      }
      row_sums<1, true>(q, red, turn);
      return make_float2(mean, 1.f / sqrtf(q[0] * inv + a.eps));
    };
    sx = stats(a.post, x_of);
    sz = stats(a.pre, z_of);
    if (a.stats && threadIdx.x == 0) a.stats[row] = make_float4(sx.x, sx.y, sz.x, sz.y);
    // z may be the residual: an element is read for the last time before it is written
    for (int c = threadIdx.x; c < a.d; c += WIDE) {
      const float z = z_of(c);
      if (a.y.p) {
        float w[1], b[1];
        params<1>(a.pre_weight, a.param_type, c, 1.f, w);
        params<1>(a.pre_bias, a.param_type, c, 0.f, b);
        at<T>(a.y, row)[c] = from_float<T>(fmaf((z - sz.x) * sz.y, w[0], b[0]));
      }
      if (a.z.p) at<R>(a.z, row)[c] = from_float<R>(z);
    }
  }
}

// ---- gradient --------------------------------------------------------------------------
// Writes a block's partial sums of the parameters' gradients (4 x d) to its slot.
template <int V, int P, bool BLOCK>
__device__ __forceinline__ void flush(const ResNormArgs& a, const Place<BLOCK>& pl, float (&acc)[4][P][V],
                                      float* slot, float* joined) {
  if constexpr (BLOCK) {
#pragma unroll
    for (int k = 0; k < 4; ++k)
      if (a.sums[k])
#pragma unroll
        for (int p = 0; p < P; ++p) {
          const int c = (p * pl.threads + pl.t) * V;
#pragma unroll
          for (int j = 0; j < V; ++j) {
            if (c + j < a.d) slot[(int64_t)k * a.d + c + j] = acc[k][p][j];
            acc[k][p][j] = 0.f;
          }
        }
  } else {
    const int warp = threadIdx.x >> 5, warps = blockDim.x >> 5;
    constexpr int COLS = 32 * P * V;
    for (int i = 0; i < warps; ++i) {  // the warps one after another, so the order is fixed
      if (warp == i)
#pragma unroll
        for (int k = 0; k < 4; ++k)
#pragma unroll
          for (int p = 0; p < P; ++p)
#pragma unroll
            for (int j = 0; j < V; ++j) {
              float* q = joined + k * COLS + (p * 32 + pl.t) * V + j;
              *q = i ? *q + acc[k][p][j] : acc[k][p][j];
              acc[k][p][j] = 0.f;
            }
      __syncthreads();
    }
    for (int i = threadIdx.x; i < 4 * a.d; i += blockDim.x) {
      const int k = i / a.d, c = i - k * a.d;
      if (a.sums[k]) slot[i] = joined[k * COLS + c];
    }
    __syncthreads();
  }
}

// BIAS: the gradients of biases are wanted.  Without their sums three blocks of 256 fit an SM.
template <typename T, typename R, int V, int P, int B, bool BIAS>
__global__ void __launch_bounds__(B ? B : 256, B == 1024 || B == 512 ? 1 : BIAS || V == 1 ? 2 : 3)
    k_residual_norm_grad(ResNormArgs a, int slots) {
  constexpr bool BLOCK = B > 0;
  extern __shared__ __align__(16) char smem[];
  __shared__ float red[2 * 64];
  __shared__ float joined[BLOCK ? 1 : 4 * 32 * P * V];
  int turn = 0;
  follow();
  const Place<BLOCK> pl;
  const float inv = 1.f / (float)a.d;
  float acc[4][P][V];
#pragma unroll
  for (int k = 0; k < 4; ++k)
#pragma unroll
    for (int p = 0; p < P; ++p)
#pragma unroll
      for (int j = 0; j < V; ++j) acc[k][p][j] = 0.f;
  float* slot = a.parts + (int64_t)blockIdx.x * slots * 4 * a.d;
  int chain = 0, filled = 0;
  using Tm = Rowed<T, V, P, BLOCK>;
  using Rm = Rowed<R, V, P, BLOCK>;
  const size_t bytes = stage_bytes<T, R, V, P>(3, 2, a.d, blockDim.x, BLOCK);
  auto fetch = [&](int64_t row, int stage) {
    char* base = smem + stage * bytes;
    const Rm z(base, a.d, pl), dz(base, a.d, pl);
    const Tm dy(base, a.d, pl), x(base, a.d, pl), g(base, a.d, pl);
    if (row < a.n) {
      if (a.dy.p) {
        dy.fetch(a.dy, row, a.n, a.d, pl);
        z.fetch(a.zin, row, a.n, a.d, pl);
      }
      if (a.dz.p) dz.fetch(a.dz, row, a.n, a.d, pl);
      x.fetch(a.x, row, a.n, a.d, pl);
      if (a.g.p) g.fetch(a.g, row, a.n, a.d, pl);
    }
    copies_begun();
  };
  const Params<V, P, BLOCK> par(a, smem + 2 * bytes, pl);
  fetch(pl.row, 0);
  int stage = 0;
  // the block's threads go round together: flush() is for all of them
  const int64_t first = BLOCK ? (int64_t)blockIdx.x : (int64_t)blockIdx.x * (blockDim.x >> 5);
  int64_t row = pl.row;
  for (int64_t base = first; base < a.n; base += pl.step, row += pl.step, stage ^= 1) {
    sync_row<T, V, BLOCK>();
    fetch(row + pl.step, stage ^ 1);
    if (row < a.n) {
      const float4 st = a.stats[row];
      copies_done<1>();
      sync_row<T, V, BLOCK>();
      char* from = smem + stage * bytes;
      Rm zs(from, a.d, pl), dzs(from, a.d, pl);
      Tm dys(from, a.d, pl), xs(from, a.d, pl), gs(from, a.d, pl);
      zs.aim(a.zin, row, a.d, pl), dzs.aim(a.dz, row, a.d, pl);
      dys.aim(a.dy, row, a.d, pl), xs.aim(a.x, row, a.d, pl), gs.aim(a.g, row, a.d, pl);
      float D[P][V];  // the gradient of z; first gy
      float s[2] = {0.f, 0.f};
      if (a.dy.p) {
#pragma unroll
        for (int p = 0; p < P; ++p) {
          const int c = (p * pl.threads + pl.t) * V;
          if (V == 1 || c < a.d) {
            float z[V], w[V];
            dys.get(p, pl, D[p]);
            zs.get(p, pl, z);
            par.get(2, p, c, w);
#pragma unroll
            for (int j = 0; j < V; ++j) {
              const float zh = (z[j] - st.z) * st.w;
              acc[2][p][j] = fmaf(D[p][j], zh, acc[2][p][j]);
              if (BIAS) acc[3][p][j] += D[p][j];
              D[p][j] *= w[j];
              s[0] = fmaf(D[p][j], zh, s[0]);
              s[1] += D[p][j];
            }
          }
        }
        row_sums<2, BLOCK>(s, red, turn);
        s[0] *= inv;
        s[1] = a.pre == GBA_NORM_LAYER ? s[1] * inv : 0.f;
      }
      float q[2] = {0.f, 0.f};
#pragma unroll
      for (int p = 0; p < P; ++p) {
        const int c = (p * pl.threads + pl.t) * V;
        if (V == 1 || c < a.d) {
          float x[V], v[V], w[V];
          if (a.dy.p) {
            zs.get(p, pl, v);
#pragma unroll
            for (int j = 0; j < V; ++j) D[p][j] = V > 1 || c < a.d ? st.w * (D[p][j] - s[1] - (v[j] - st.z) * st.w * s[0]) : 0.f;
          } else {
#pragma unroll
            for (int j = 0; j < V; ++j) D[p][j] = 0.f;
          }
          if (a.dz.p) {
            dzs.get(p, pl, v);
#pragma unroll
            for (int j = 0; j < V; ++j) D[p][j] += v[j];
          }
          if (a.dr.p) {
#pragma unroll
            for (int j = 0; j < V; ++j) v[j] = a.rscale * D[p][j];
            Pack<R, V> o;
            o.set(v);
            if (V > 1 || c < a.d) o.store(at<R>(a.dr, row) + c);
          }
          xs.get(p, pl, x);
          par.get(0, p, c, w);
#pragma unroll
          for (int j = 0; j < V; ++j) x[j] = (x[j] - st.x) * st.y, D[p][j] *= a.bscale;
          if (a.gate != GBA_GATE_NONE) {
            float b[V];
            gs.get(p, pl, v);
            par.get(1, p, c, b);
#pragma unroll
            for (int j = 0; j < V; ++j) {
              float slope;
              const float act = gate_of(a.gate, v[j], slope);
              v[j] = D[p][j] * fmaf(x[j], w[j], b[j]) * slope;
              D[p][j] *= act;
            }
            Pack<T, V> o;
            o.set(v);
            if (V > 1 || c < a.d) o.store(at<T>(a.dg, row) + c);
          }
#pragma unroll
          for (int j = 0; j < V; ++j) {
            acc[0][p][j] = fmaf(D[p][j], x[j], acc[0][p][j]);
            if (BIAS) acc[1][p][j] += D[p][j];
            D[p][j] *= w[j];  // gu
            q[0] = fmaf(D[p][j], x[j], q[0]);
            q[1] += D[p][j];
          }
        }
      }
      if (a.post != GBA_NORM_NONE) {
        row_sums<2, BLOCK>(q, red, turn);
        q[0] *= inv;
        q[1] = a.post == GBA_NORM_LAYER ? q[1] * inv : 0.f;
      } else {
        q[0] = q[1] = 0.f;
      }
#pragma unroll
      for (int p = 0; p < P; ++p) {
        const int c = (p * pl.threads + pl.t) * V;
        if (V == 1 || c < a.d) {
          float x[V];
          xs.get(p, pl, x);
#pragma unroll
          for (int j = 0; j < V; ++j) x[j] = st.y * (D[p][j] - q[1] - (x[j] - st.x) * st.y * q[0]);
          Pack<T, V> o;
          o.set(x);
          if (V > 1 || c < a.d) o.store(at<T>(a.dx, row) + c);
        }
      }
    }
    if (++chain == CHAIN) {
      flush<V, P, BLOCK>(a, pl, acc, slot + (int64_t)filled++ * 4 * a.d, joined);
      chain = 0;
    }
  }
  copies_done<0>();
  for (; filled < slots; ++filled) flush<V, P, BLOCK>(a, pl, acc, slot + (int64_t)filled * 4 * a.d, joined);
}

// Rows of any width: one pass for each pair of sums and one for the outputs; the parameters'
// sums lie in the block's slots, each column added to by one thread.
template <typename T, typename R>
__global__ void __launch_bounds__(WIDE) k_residual_norm_grad_wide(ResNormArgs a, int slots) {
  __shared__ float red[2 * 64];
  int turn = 0;
  follow();
  const float inv = 1.f / (float)a.d;
  float* slot = a.parts + (int64_t)blockIdx.x * slots * 4 * a.d;
  for (int64_t i = threadIdx.x; i < (int64_t)slots * 4 * a.d; i += WIDE) slot[i] = 0.f;
  __syncthreads();  // of other threads' columns too
  int chain = 0;
  for (int64_t row = blockIdx.x; row < a.n; row += gridDim.x) {
    const float4 st = a.stats[row];
    float s[2] = {0.f, 0.f}, q[2] = {0.f, 0.f};
    float w[1], b[1];
    if (a.dy.p) {
      for (int c = threadIdx.x; c < a.d; c += WIDE) {
        params<1>(a.pre_weight, a.param_type, c, 1.f, w);
        const float dy = to_float(at<T>(a.dy, row)[c]);
        const float zh = (to_float(at<R>(a.zin, row)[c]) - st.z) * st.w;
        s[0] = fmaf(dy * w[0], zh, s[0]);
        s[1] += dy * w[0];
        if (a.sums[2]) slot[2 * (int64_t)a.d + c] += dy * zh;
        if (a.sums[3]) slot[3 * (int64_t)a.d + c] += dy;
      }
      row_sums<2, true>(s, red, turn);
      s[0] *= inv;
      s[1] = a.pre == GBA_NORM_LAYER ? s[1] * inv : 0.f;
    }
    auto D_of = [&](int c) {
      float D = 0.f;
      if (a.dy.p) {
        params<1>(a.pre_weight, a.param_type, c, 1.f, w);
        const float zh = (to_float(at<R>(a.zin, row)[c]) - st.z) * st.w;
        D = st.w * (to_float(at<T>(a.dy, row)[c]) * w[0] - s[1] - zh * s[0]);
      }
      return a.dz.p ? D + to_float(at<R>(a.dz, row)[c]) : D;
    };
    auto e_of = [&](int c, float D, float& dg, float xh) {
      float e = a.bscale * D;
      params<1>(a.post_weight, a.param_type, c, 1.f, w);
      if (a.gate != GBA_GATE_NONE) {
        params<1>(a.post_bias, a.param_type, c, 0.f, b);
        float slope;
        const float act = gate_of(a.gate, to_float(at<T>(a.g, row)[c]), slope);
        dg = e * fmaf(xh, w[0], b[0]) * slope;
        e *= act;
      }
      return e;
    };
    float dg = 0.f;
    if (a.post != GBA_NORM_NONE) {
      for (int c = threadIdx.x; c < a.d; c += WIDE) {
        const float xh = (to_float(at<T>(a.x, row)[c]) - st.x) * st.y;
        const float gu = e_of(c, D_of(c), dg, xh) * w[0];
        q[0] = fmaf(gu, xh, q[0]);
        q[1] += gu;
      }
      row_sums<2, true>(q, red, turn);
      q[0] *= inv;
      q[1] = a.post == GBA_NORM_LAYER ? q[1] * inv : 0.f;
    }
    // dr may be dz: an element is read for the last time before it is written
    for (int c = threadIdx.x; c < a.d; c += WIDE) {
      const float D = D_of(c), xh = (to_float(at<T>(a.x, row)[c]) - st.x) * st.y;
      const float e = e_of(c, D, dg, xh);
      if (a.sums[0]) slot[c] += e * xh;
      if (a.sums[1]) slot[(int64_t)a.d + c] += e;
      if (a.dr.p) at<R>(a.dr, row)[c] = from_float<R>(a.rscale * D);
      if (a.g.p) at<T>(a.dg, row)[c] = from_float<T>(dg);
      at<T>(a.dx, row)[c] = from_float<T>(st.y * (e * w[0] - q[1] - xh * q[0]));
    }
    if (++chain == CHAIN) {
      slot += 4 * (int64_t)a.d;
      chain = 0;
    }
  }
}

// Adds the slots of every column in order, with compensation: 16 threads a column, each
// every 16th slot, then those of the column.
constexpr int SUM_LANES = 16;
__global__ void __launch_bounds__(32 * SUM_LANES) k_residual_norm_sums(ResNormArgs a, int slots) {
  __shared__ float part[SUM_LANES][33];
  follow();
  const int k = blockIdx.y, c = blockIdx.x * 32 + threadIdx.x;
  float* out = a.sums[k];
  if (!out) return;
  float sum = 0.f, off = 0.f;
  if (c < a.d)
    for (int i = threadIdx.y; i < slots; i += SUM_LANES) {
      const float v = a.parts[((int64_t)i * 4 + k) * a.d + c], s = sum + v, bb = s - sum;
      off += (sum - (s - bb)) + (v - bb);
      sum = s;
    }
  // a sum that is infinite is its plain sum: the correction of an infinity is a NaN
  part[threadIdx.y][threadIdx.x] = isfinite(sum) ? sum + off : sum;
  __syncthreads();
  if (threadIdx.y == 0 && c < a.d) {
    float s = 0.f;
#pragma unroll
    for (int i = 0; i < SUM_LANES; ++i) s += part[i][threadIdx.x];
    out[c] = s;
  }
}

// ---- launches ------------------------------------------------------------------------------
// Elements of an access, packs of a thread, threads of a row; 0 packs: the wide form.
struct Shape {
  int v, packs, threads;
  bool block;
  int rows;  // rows that a block holds at a time
  unsigned grid;
  int slots;  // of a block
};

int vector_for(const ResNormArgs& a, int32_t type, int32_t wide, bool grad) {
  int v = type == GBA_F32 ? 4 : 8;
  auto fits = [&](const void* p, int64_t stride, int32_t t) {
    return !p || vector_of(v, p, stride, a.d, type_bytes(t)) == v;
  };
  bool ok = fits(a.x.p, a.x.stride, type) && fits(a.g.p, a.g.stride, type);
  if (grad)
    ok = ok && fits(a.dy.p, a.dy.stride, type) && fits(a.dz.p, a.dz.stride, wide) && fits(a.zin.p, a.zin.stride, wide) &&
         fits(a.dx.p, a.dx.stride, type) && fits(a.dr.p, a.dr.stride, wide) && fits(a.dg.p, a.dg.stride, type);
  else
    ok = ok && fits(a.r.p, a.r.stride, wide) && fits(a.z.p, a.z.stride, wide) && fits(a.y.p, a.y.stride, type);
  for (const void* p : {a.post_weight, a.post_bias, a.pre_weight, a.pre_bias}) ok = ok && fits(p, 0, a.param_type);
  return ok ? v : 1;
}

Shape shape_of(const ResNormArgs& a, int32_t type, int32_t wide, bool grad, int num_sms) {
  Shape s{};
  s.v = vector_for(a, type, wide, grad);
  const int d = a.d, vecs = (d + s.v - 1) / s.v;
  if (grad || s.v == 1) {  // eight elements a thread; the gradient's go with four sums of parameters' gradients
    s.packs = 8 / s.v;
    s.block = d > 256;
  } else {
    s.block = vecs > 128;
    s.packs = s.block ? 2 : vecs <= 32 ? 1 : vecs <= 64 ? 2 : 4;
  }
  const int each = s.v * s.packs;
  s.threads = s.block ? ((d + each - 1) / each + 31) / 32 * 32 : 32;
  s.rows = s.block ? 1 : 8;
  // two rows of each block lie in shared memory; wider ones are read again for each sum
  const size_t b = type_bytes(type), w = type_bytes(wide), room = 226 << 10;
  const size_t nt = grad ? 3 : 2, nr = grad ? 2 : 1;
  size_t bytes = 2 * (size_t)s.threads * s.rows * each * (nt * b + nr * w);
  if (s.v == 1) {  // those of 16 bits, and the parameters
    bytes = b == 2 ? 2 * s.rows * nt * ((size_t)d * 2 + 32) : 0;
    if (w == 2) bytes += 2 * s.rows * nr * ((size_t)d * 2 + 32);
    bytes += (size_t)s.threads * s.rows * HELD_BYTES<1, 8>;
  }
  // that registers are for
  const size_t threads = !grad ? 1024 : s.v == 1 || a.sums[1] || a.sums[3] ? 576 : 768;
  size_t most = 2;  // blocks of an SM
  if (s.threads > 1024 || bytes > room) {
    s.packs = 0;
    s.threads = WIDE;
    s.block = true;
    s.rows = 1;
  } else {
    most = std::max<size_t>(1, std::min(room / (bytes + 5120), threads / (s.threads * s.rows)));
  }
  s.grid = (unsigned)std::min<int64_t>((a.n + s.rows - 1) / s.rows, (int64_t)num_sms * (int64_t)most);
  const int64_t chain = (a.n + (int64_t)s.grid * s.rows - 1) / ((int64_t)s.grid * s.rows);
  s.slots = (int)((chain + CHAIN - 1) / CHAIN);
  return s;
}

// Two rows of each of a block's lie in shared memory.
template <typename K, typename... A>
cudaError_t start(K kernel, const Shape& h, size_t stage, size_t held, cudaStream_t s, A... args) {
  const size_t bytes = 2 * stage + held * h.threads * h.rows;
  const cudaError_t e = cudaFuncSetAttribute(kernel, cudaFuncAttributeMaxDynamicSharedMemorySize, (int)bytes);
  if (e != cudaSuccess) return e;
  return launch_following(kernel, dim3(h.grid), h.threads * h.rows, bytes, s, args...);
}

template <typename T, typename R, int V, int P>
cudaError_t forward_in(const ResNormArgs& a, const Shape& h, cudaStream_t s) {
  const size_t stage = stage_bytes<T, R, V, P>(2, 1, a.d, h.threads * h.rows, h.block);
  if (!h.block) return start(k_residual_norm<T, R, V, P, 0>, h, stage, HELD_BYTES<V, P>, s, a);
  if constexpr (P <= 2 || V == 1) {  // four vectors a thread are a warp's
    if (h.threads <= 256) return start(k_residual_norm<T, R, V, P, 256>, h, stage, HELD_BYTES<V, P>, s, a);
    return start(k_residual_norm<T, R, V, P, 1024>, h, stage, HELD_BYTES<V, P>, s, a);
  }
  return cudaErrorInvalidValue;
}

template <typename T, typename R>
cudaError_t forward(const ResNormArgs& a, const Shape& h, cudaStream_t s) {
  constexpr int V = 16 / (int)sizeof(T);
  if (h.packs == 0) return launch_following(k_residual_norm_wide<T, R>, dim3(h.grid), WIDE, 0, s, a);
  if (h.v == 1) return forward_in<T, R, 1, 8>(a, h, s);
  if (h.packs == 1) return forward_in<T, R, V, 1>(a, h, s);
  return h.packs == 2 ? forward_in<T, R, V, 2>(a, h, s) : forward_in<T, R, V, 4>(a, h, s);
}

template <typename T, typename R, int V, int P, bool BIAS>
cudaError_t backward_as(const ResNormArgs& a, const Shape& h, cudaStream_t s) {
  const size_t stage = stage_bytes<T, R, V, P>(3, 2, a.d, h.threads * h.rows, h.block);
  if (!h.block) return start(k_residual_norm_grad<T, R, V, P, 0, BIAS>, h, stage, HELD_BYTES<V, P>, s, a, h.slots);
  if (h.threads <= 256) return start(k_residual_norm_grad<T, R, V, P, 256, BIAS>, h, stage, HELD_BYTES<V, P>, s, a, h.slots);
  if (h.threads <= 512) return start(k_residual_norm_grad<T, R, V, P, 512, BIAS>, h, stage, HELD_BYTES<V, P>, s, a, h.slots);
  return start(k_residual_norm_grad<T, R, V, P, 1024, BIAS>, h, stage, HELD_BYTES<V, P>, s, a, h.slots);
}
template <typename T, typename R, int V, int P>
cudaError_t backward_in(const ResNormArgs& a, const Shape& h, cudaStream_t s) {
  if constexpr (V > 1)
    if (!a.sums[1] && !a.sums[3]) return backward_as<T, R, V, P, false>(a, h, s);
  return backward_as<T, R, V, P, true>(a, h, s);
}

template <typename T, typename R>
cudaError_t backward(const ResNormArgs& a, const Shape& h, cudaStream_t s) {
  constexpr int V = 16 / (int)sizeof(T);
  if (h.packs == 0) return launch_following(k_residual_norm_grad_wide<T, R>, dim3(h.grid), WIDE, 0, s, a, h.slots);
  return h.v == 1 ? backward_in<T, R, 1, 8>(a, h, s) : backward_in<T, R, V, 8 / V>(a, h, s);
}

}  // namespace

cudaError_t launch_residual_norm(const ResNormArgs& a, int32_t type, int32_t wide, int num_sms, cudaStream_t s) {
  const Shape h = shape_of(a, type, wide, false, num_sms);
  if (type == GBA_F32) return forward<float, float>(a, h, s);
  if (type == GBA_BF16) return wide == GBA_F32 ? forward<bf16, float>(a, h, s) : forward<bf16, bf16>(a, h, s);
  return wide == GBA_F32 ? forward<f16, float>(a, h, s) : forward<f16, f16>(a, h, s);
}

size_t residual_norm_grad_workspace(const ResNormArgs& a, int32_t type, int32_t wide, int num_sms) {
  const Shape h = shape_of(a, type, wide, true, num_sms);
  return (size_t)h.grid * h.slots * 4 * (size_t)a.d * sizeof(float);
}

cudaError_t launch_residual_norm_grad(const ResNormArgs& a, int32_t type, int32_t wide, int num_sms, cudaStream_t s) {
  const Shape h = shape_of(a, type, wide, true, num_sms);
  cudaError_t e;
  if (type == GBA_F32)
    e = backward<float, float>(a, h, s);
  else if (type == GBA_BF16)
    e = wide == GBA_F32 ? backward<bf16, float>(a, h, s) : backward<bf16, bf16>(a, h, s);
  else
    e = wide == GBA_F32 ? backward<f16, float>(a, h, s) : backward<f16, f16>(a, h, s);
  if (e != cudaSuccess) return e;
  if (!a.sums[0] && !a.sums[1] && !a.sums[2] && !a.sums[3]) return cudaSuccess;
  cudaLaunchAttribute attr[1];
  attr[0].id = cudaLaunchAttributeProgrammaticStreamSerialization;
  attr[0].val.programmaticStreamSerializationAllowed = 1;
  cudaLaunchConfig_t cfg{};
  cfg.gridDim = dim3((unsigned)((a.d + 31) / 32), 4);
  cfg.blockDim = dim3(32, SUM_LANES);
  cfg.stream = s;
  cfg.attrs = attr;
  cfg.numAttrs = 1;
  return cudaLaunchKernelEx(&cfg, k_residual_norm_sums, a, (int)(h.grid * h.slots));
}

}  // namespace gba

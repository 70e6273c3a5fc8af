// The end of a block and the norm before the next, and their gradient:
//   u = (x - mx) rx wq + bq,  z = rs r + bs act(g) u,  y = (z - mz) rz wp + bp.
// Backwards, with gy = dy wp and zh = (z - mz) rz:
//   D = dz + rz (gy - mean(gy) - zh mean(gy zh)),  dr = rs D,  t = bs D,
//   dg = t u act'(g),  e = t act(g),  gu = e wq,  dx = rx (gu - mean(gu) - xh mean(gu xh)),
//   dwp = sum dy zh, dbp = sum dy, dwq = sum e xh, dbq = sum e over the rows;
// the means without a product only for layer norms, and no mean where there is no norm.
//
// Bound by HBM bandwidth where a row is in memory and its arithmetic is short: every input is read once
// and every output written once.  A row is a warp's (up to some hundred columns, when there is no barrier)
// or a block's; the next row's pieces are copied to shared memory while a row is worked on, and z or D stays
// in registers between the sums.  Rows that do not fit so are read again from L2 by one block each.
//   forward  bf16 32,768 x 4,096, float32 residual, one norm   260 us, 6.2 TB/s: HBM
//            bf16 32,768 x 2,048, two norms and a gate         145 us, 4.6 TB/s: 73% of the issue slots, and two
//            sums over the block one after another
//   gradient bf16 32,768 x 2,048, the same                     236 us, 4.5 TB/s: latency, with 24% of the warps
//            (the parameters' sums take the registers) and 58% of the issue slots: 76 instructions an element,
//            as 16-bit values are widened in every pass, and pairs of floats built
//            float32 5,003 x 1,001, layer norms with biases     82 us, 1.9 TB/s: single elements, and 4 rows an SM
//            at a time, because the sums of four parameters' gradients take the registers
// Single elements (rows or parameters that do not lie on 16 bytes): reading 16-bit rows by vectors that are
// brought into place, with outputs through shared memory, took bf16 32,768 x 2,049 787 us against 1,110
// backwards, but 131,072 x 201 250 against 219 and float32 8,192 x 4,001 612 against 432, and is not here.
#include <algorithm>
#include <cfloat>

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

// V floats, two in one instruction where there are two: backwards the arithmetic of single floats took
// bf16 32,768 x 2,048 from HBM's bound to the instructions' (283 us).
template <int V>
struct Vals {
  using E = std::conditional_t<V == 1, float, f2>;
  static constexpr int N = V == 1 ? 1 : V / 2;
  E v[N];
  Vals() = default;
  __device__ __forceinline__ explicit Vals(const float (&x)[V]) {
    if constexpr (V == 1) {
      v[0] = x[0];
    } else {
#pragma unroll
      for (int j = 0; j < N; ++j) v[j] = pair(x[2 * j], x[2 * j + 1]);
    }
  }
  __device__ __forceinline__ explicit Vals(float x) {
#pragma unroll
    for (int j = 0; j < N; ++j)
      if constexpr (V == 1)
        v[j] = x;
      else
        v[j] = pair(x, x);
  }
  __device__ __forceinline__ void get(float (&x)[V]) const {
    if constexpr (V == 1) {
      x[0] = v[0];
    } else {
#pragma unroll
      for (int j = 0; j < N; ++j) split(v[j], x[2 * j], x[2 * j + 1]);
    }
  }
  __device__ __forceinline__ float sum() const {
    if constexpr (V == 1) {
      return v[0];
    } else {
      f2 s = v[0];
#pragma unroll
      for (int j = 1; j < N; ++j) s = add2(s, v[j]);
      return both(s);
    }
  }
};
template <int V>
__device__ __forceinline__ Vals<V> operator+(const Vals<V>& a, const Vals<V>& b) {
  Vals<V> r;
#pragma unroll
  for (int j = 0; j < Vals<V>::N; ++j)
    if constexpr (V == 1)
      r.v[j] = a.v[j] + b.v[j];
    else
      r.v[j] = add2(a.v[j], b.v[j]);
  return r;
}
template <int V>
__device__ __forceinline__ Vals<V> operator*(const Vals<V>& a, const Vals<V>& b) {
  Vals<V> r;
#pragma unroll
  for (int j = 0; j < Vals<V>::N; ++j)
    if constexpr (V == 1)
      r.v[j] = a.v[j] * b.v[j];
    else
      r.v[j] = mul2(a.v[j], b.v[j]);
  return r;
}
template <int V>
__device__ __forceinline__ Vals<V> fma_v(const Vals<V>& a, const Vals<V>& b, const Vals<V>& c) {
  Vals<V> r;
#pragma unroll
  for (int j = 0; j < Vals<V>::N; ++j)
    if constexpr (V == 1)
      r.v[j] = fmaf(a.v[j], b.v[j], c.v[j]);
    else
      r.v[j] = fma2(a.v[j], b.v[j], c.v[j]);
  return r;
}
template <int V>
__device__ __forceinline__ Vals<V> operator+(const Vals<V>& a, float b) { return a + Vals<V>(b); }
template <int V>
__device__ __forceinline__ Vals<V> operator*(const Vals<V>& a, float b) { return a * Vals<V>(b); }

// The gates' factors, and their derivatives.  With t = exp(-g), s = 1 / (1 + t) and 1 - s = t s, which
// does not cancel.  A t that overflows (g below -88.7) gives s = 0 and derivatives of 0: 4e-37 off.  The
// reciprocal is that of (1 + t) / 4, which is not below the least normal number.  NaNs stay.
template <int V>
__device__ __forceinline__ Vals<V> gate_of(int32_t kind, const Vals<V>& g, Vals<V>& slope) {
  if (kind == GBA_GATE_MUL) {
    slope = Vals<V>(1.f);
    return g;
  }
  float t[V], q[V];
  (g * -1.4426950408889634f).get(t);
#pragma unroll
  for (int j = 0; j < V; ++j) asm("ex2.approx.ftz.f32 %0, %0;" : "+f"(t[j]));
  fma_v(Vals<V>(t), Vals<V>(0.25f), Vals<V>(0.25f)).get(q);
#pragma unroll
  for (int j = 0; j < V; ++j) {
    asm("rcp.approx.ftz.f32 %0, %0;" : "+f"(q[j]));
    asm("min.NaN.f32 %0, %0, %1;" : "+f"(t[j]) : "f"(FLT_MAX));
  }
  const Vals<V> sig = Vals<V>(q) * 0.25f, rest = Vals<V>(t) * sig;
  if (kind == GBA_GATE_SIGMOID) {
    slope = sig * rest;
    return sig;
  }
  slope = sig * fma_v(g, rest, Vals<V>(1.f));
  return g * sig;
}
__device__ __forceinline__ float gate_of(int32_t kind, float g, float& slope) {
  Vals<1> d;
  const Vals<1> f = gate_of<1>(kind, Vals<1>(g), d);
  slope = d.v[0];
  return f.v[0];
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
    if (warps <= 8) {  // adding eight takes less than five exchanges
#pragma unroll
      for (int i = 0; i < N; ++i) {
        const float4 lo = reinterpret_cast<const float4*>(buf + i * 32)[0], hi = reinterpret_cast<const float4*>(buf + i * 32)[1];
        v[i] = ((lo.x + (warps > 1 ? lo.y : 0.f)) + ((warps > 2 ? lo.z : 0.f) + (warps > 3 ? lo.w : 0.f))) +
               (((warps > 4 ? hi.x : 0.f) + (warps > 5 ? hi.y : 0.f)) + ((warps > 6 ? hi.z : 0.f) + (warps > 7 ? hi.w : 0.f)));
      }
    } else {
#pragma unroll
      for (int i = 0; i < N; ++i) {
        v[i] = lane < warps ? buf[i * 32 + lane] : 0.f;
#pragma unroll
        for (int o = 16; o > 0; o >>= 1) v[i] += __shfl_xor_sync(0xffffffffu, v[i], o);
      }
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

template <typename T, int V>
__device__ __forceinline__ void put(T* to, const Vals<V>& v) {
  float x[V];
  v.get(x);
  Pack<T, V> o;
  o.set(x);
  o.store(to);
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
  __device__ __forceinline__ Vals<V> get(int k, const Place<BLOCK>&) const {
    float x[V];
    Pack<T, V> w;
    w.load(at + (size_t)k * blockDim.x * V);
    w.get(x);
    return Vals<V>(x);
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
  __device__ __forceinline__ Vals<1> get(int k, const Place<BLOCK>& pl) const {
    const int c = k * pl.threads + pl.t;
    return Vals<1>(c < d ? to_float(row[c]) : 0.f);
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
  __device__ __forceinline__ Vals<1> get(int k, const Place<BLOCK>&) const { return Vals<1>(v[k]); }
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
  __device__ __forceinline__ Vals<V> get(int k, int p, int c) const {
    if constexpr (V == 1) {
      return Vals<V>(held[(k * P + p) * blockDim.x]);
    } else {
      float w[V];
      params<V>(of(k), a.param_type, c, k & 1 ? 0.f : 1.f, w);
      return Vals<V>(w);
    }
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
template <typename T, int V, int P>
__host__ __device__ constexpr size_t matrix_bytes(int d, int threads, bool block) {
  if constexpr (V == 1)
    return (block ? 1 : threads / 32) * Rowed<T, 1, P, true>::bytes(d);
  else
    return (size_t)threads * V * P * sizeof(T);
}
template <typename T, typename R, int V, int P>
__host__ __device__ constexpr size_t stage_bytes(int nt, int nr, int d, int threads, bool block) {
  return nt * matrix_bytes<T, V, P>(d, threads, block) + nr * matrix_bytes<R, V, P>(d, threads, block);
}

// ---- forward -------------------------------------------------------------------------
// The mean and the reciprocal deviation of a row; value(p) gives piece p.
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
      if (V == 1 || (p * at.threads + at.t) * V < a.d) s[0] += value(p).sum();
    row_sums<1, BLOCK>(s, red, turn);
    mean = s[0] * inv;
  }
  Vals<V> q(0.f);
#pragma unroll
  for (int p = 0; p < P; ++p)
    if (V == 1 || (p * at.threads + at.t) * V < a.d) {
      Vals<V> e = value(p) + -mean;
      if (V == 1 && p * at.threads + at.t >= a.d) e = Vals<V>(0.f);
      q = fma_v(e, e, q);
    }
  float sum[1] = {q.sum()};
  row_sums<1, BLOCK>(sum, red, turn);
  return make_float2(mean, 1.f / sqrtf(sum[0] * inv + a.eps));
}

// B: the most threads of a block that holds one row; 0: a row is a warp's
template <typename T, typename R, int V, int P, int B>
__global__ void __launch_bounds__(B ? B : 256, B == 1024 ? 1 : 4) k_residual_norm(ResNormArgs a) {
  constexpr bool BLOCK = B > 0;
  extern __shared__ __align__(16) char smem[];
  __shared__ __align__(16) float red[2 * 64];
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
    const float2 sx = row_stats<V, P, BLOCK>([&](int p) { return xs.get(p, pl); }, a.post, a, pl, red, turn);
    Vals<V> z[P];
#pragma unroll
    for (int p = 0; p < P; ++p) {
      const int c = (p * pl.threads + pl.t) * V;
      z[p] = Vals<V>(0.f);
      if (V == 1 || c < a.d) {
        z[p] = (xs.get(p, pl) + -sx.x) * sx.y * par.get(0, p, c);
        if (a.post_bias) z[p] = z[p] + par.get(1, p, c);
        if (a.gate != GBA_GATE_NONE) {
          Vals<V> slope;
          z[p] = z[p] * gate_of<V>(a.gate, gs.get(p, pl), slope);
        }
        z[p] = z[p] * a.bscale;
        if (a.r.p) z[p] = fma_v(rs.get(p, pl), Vals<V>(a.rscale), z[p]);
        if (a.z.p && (V > 1 || c < a.d)) put<R, V>(at<R>(a.z, row) + c, z[p]);
      }
    }
    const float2 sz = row_stats<V, P, BLOCK>([&](int p) { return z[p]; }, a.pre, a, pl, red, turn);
    if (a.stats && pl.t == 0) a.stats[row] = make_float4(sx.x, sx.y, sz.x, sz.y);
    if (a.y.p)
#pragma unroll
      for (int p = 0; p < P; ++p) {
        const int c = (p * pl.threads + pl.t) * V;
        if (V == 1 || c < a.d) {
          z[p] = (z[p] + -sz.x) * sz.y * par.get(2, p, c);
          if (a.pre_bias) z[p] = z[p] + par.get(3, p, c);
          if (V > 1 || c < a.d) put<T, V>(at<T>(a.y, row) + c, z[p]);
        }
      }
  }
  copies_done<0>();
}

constexpr int WIDE = 1024;

// Rows of any width: a block goes over its row once for each sum and once for the outputs, the first time from HBM
// and then from L2, by single elements (bf16 4,096 x 20,000 696 us, and 1,678 backwards).
template <typename T, typename R>
__global__ void __launch_bounds__(WIDE) k_residual_norm_wide(ResNormArgs a) {
  __shared__ __align__(16) float red[2 * 64];
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
__device__ __forceinline__ void flush(const ResNormArgs& a, const Place<BLOCK>& pl, Vals<V> (&acc)[4][P],
                                      float* slot, float* joined) {
  if constexpr (BLOCK) {
#pragma unroll
    for (int k = 0; k < 4; ++k)
      if (a.sums[k])
#pragma unroll
        for (int p = 0; p < P; ++p) {
          const int c = (p * pl.threads + pl.t) * V;
          float v[V];
          acc[k][p].get(v);
#pragma unroll
          for (int j = 0; j < V; ++j)
            if (c + j < a.d) slot[(int64_t)k * a.d + c + j] = v[j];
          acc[k][p] = Vals<V>(0.f);
        }
  } else {
    const int warp = threadIdx.x >> 5, warps = blockDim.x >> 5;
    constexpr int COLS = 32 * P * V;
    for (int i = 0; i < warps; ++i) {  // the warps one after another, so the order is fixed
      if (warp == i)
#pragma unroll
        for (int k = 0; k < 4; ++k)
#pragma unroll
          for (int p = 0; p < P; ++p) {
            float v[V];
            acc[k][p].get(v);
#pragma unroll
            for (int j = 0; j < V; ++j) {
              float* q = joined + k * COLS + (p * 32 + pl.t) * V + j;
              *q = i ? *q + v[j] : v[j];
            }
            acc[k][p] = Vals<V>(0.f);
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

// Floats through which the warps of a block join their sums.
template <int V, int P, bool BLOCK>
constexpr size_t JOINED = BLOCK ? 1 : 4 * 32 * P * V;

// Blocks of an SM, by the registers: the sums of biases' gradients (BIAS) take a third.
constexpr int grad_blocks(int v, int p, int b, bool bias) {
  if (b >= 512) return 1;
  if (v == 8 && p == 2) return b == 128 ? 4 : 2;
  return bias || v == 1 ? 2 : 3;
}
template <typename T, typename R, int V, int P, int B, bool BIAS>
__global__ void __launch_bounds__(B ? B : 256, grad_blocks(V, P, B, BIAS))
    k_residual_norm_grad(ResNormArgs a, int slots) {
  constexpr bool BLOCK = B > 0;
  extern __shared__ __align__(16) char smem[];
  __shared__ __align__(16) float red[2 * 64];
  __shared__ float joined[JOINED<V, P, BLOCK>];
  int turn = 0;
  follow();
  const Place<BLOCK> pl;
  const float inv = 1.f / (float)a.d;
  Vals<V> acc[4][P];
#pragma unroll
  for (int k = 0; k < 4; ++k)
#pragma unroll
    for (int p = 0; p < P; ++p) acc[k][p] = Vals<V>(0.f);
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
      Vals<V> D[P];  // the gradient of z; first gy
      float s[2] = {0.f, 0.f};
      if (a.dy.p) {
        Vals<V> sh(0.f), sg(0.f);
#pragma unroll
        for (int p = 0; p < P; ++p) {
          const int c = (p * pl.threads + pl.t) * V;
          if (V == 1 || c < a.d) {
            const Vals<V> zh = (zs.get(p, pl) + -st.z) * st.w;
            D[p] = dys.get(p, pl);
            acc[2][p] = fma_v(D[p], zh, acc[2][p]);
            if (BIAS) acc[3][p] = acc[3][p] + D[p];
            D[p] = D[p] * par.get(2, p, c);
            sh = fma_v(D[p], zh, sh);
            sg = sg + D[p];
          }
        }
        s[0] = sh.sum(), s[1] = sg.sum();
        row_sums<2, BLOCK>(s, red, turn);
        s[0] *= -inv * st.w;
        s[1] = a.pre == GBA_NORM_LAYER ? -s[1] * inv : 0.f;
      }
      Vals<V> qh(0.f), qg(0.f);
#pragma unroll
      for (int p = 0; p < P; ++p) {
        const int c = (p * pl.threads + pl.t) * V;
        if (V == 1 || c < a.d) {
          if (a.dy.p) {
            D[p] = fma_v(zs.get(p, pl) + -st.z, Vals<V>(s[0]), D[p] + s[1]) * st.w;
            if (V == 1 && c >= a.d) D[p] = Vals<V>(0.f);
          } else {
            D[p] = Vals<V>(0.f);
          }
          if (a.dz.p) D[p] = D[p] + dzs.get(p, pl);
          if (a.dr.p && (V > 1 || c < a.d)) put<R, V>(at<R>(a.dr, row) + c, D[p] * a.rscale);
          const Vals<V> xh = (xs.get(p, pl) + -st.x) * st.y, w = par.get(0, p, c);
          D[p] = D[p] * a.bscale;
          if (a.gate != GBA_GATE_NONE) {
            Vals<V> slope;
            const Vals<V> act = gate_of<V>(a.gate, gs.get(p, pl), slope);
            const Vals<V> dg = D[p] * fma_v(xh, w, par.get(1, p, c)) * slope;
            if (V > 1 || c < a.d) put<T, V>(at<T>(a.dg, row) + c, dg);
            D[p] = D[p] * act;
          }
          acc[0][p] = fma_v(D[p], xh, acc[0][p]);
          if (BIAS) acc[1][p] = acc[1][p] + D[p];
          D[p] = D[p] * w;  // gu
          qh = fma_v(D[p], xh, qh);
          qg = qg + D[p];
        }
      }
      float q[2] = {0.f, 0.f};
      if (a.post != GBA_NORM_NONE) {
        q[0] = qh.sum(), q[1] = qg.sum();
        row_sums<2, BLOCK>(q, red, turn);
        q[0] *= -inv * st.y;
        q[1] = a.post == GBA_NORM_LAYER ? -q[1] * inv : 0.f;
      }
#pragma unroll
      for (int p = 0; p < P; ++p) {
        const int c = (p * pl.threads + pl.t) * V;
        if (V == 1 || c < a.d) {
          const Vals<V> dx = fma_v(xs.get(p, pl) + -st.x, Vals<V>(q[0]), D[p] + q[1]) * st.y;
          if (V > 1 || c < a.d) put<T, V>(at<T>(a.dx, row) + c, dx);
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
  __shared__ __align__(16) float red[2 * 64];
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
    auto param = [&](const void* p, int c, float fill) {
      float w[1];
      params<1>(p, a.param_type, c, fill, w);
      return w[0];
    };
    if (a.dy.p) {
      for (int c = threadIdx.x; c < a.d; c += WIDE) {
        const float dy = to_float(at<T>(a.dy, row)[c]), gy = dy * param(a.pre_weight, c, 1.f);
        const float zh = (to_float(at<R>(a.zin, row)[c]) - st.z) * st.w;
        s[0] = fmaf(gy, zh, s[0]);
        s[1] += gy;
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
        const float zh = (to_float(at<R>(a.zin, row)[c]) - st.z) * st.w;
        D = st.w * (to_float(at<T>(a.dy, row)[c]) * param(a.pre_weight, c, 1.f) - s[1] - zh * s[0]);
      }
      return a.dz.p ? D + to_float(at<R>(a.dz, row)[c]) : D;
    };
    // e and dg of column c, whose post weight is w
    auto e_of = [&](int c, float D, float xh, float w, float& dg) {
      float e = a.bscale * D;
      if (a.gate != GBA_GATE_NONE) {
        float slope;
        const float act = gate_of(a.gate, to_float(at<T>(a.g, row)[c]), slope);
        dg = e * fmaf(xh, w, param(a.post_bias, c, 0.f)) * slope;
        e *= act;
      }
      return e;
    };
    float dg = 0.f;
    if (a.post != GBA_NORM_NONE) {
      for (int c = threadIdx.x; c < a.d; c += WIDE) {
        const float w = param(a.post_weight, c, 1.f), xh = (to_float(at<T>(a.x, row)[c]) - st.x) * st.y;
        const float gu = e_of(c, D_of(c), xh, w, dg) * w;
        q[0] = fmaf(gu, xh, q[0]);
        q[1] += gu;
      }
      row_sums<2, true>(q, red, turn);
      q[0] *= inv;
      q[1] = a.post == GBA_NORM_LAYER ? q[1] * inv : 0.f;
    }
    // dr may be dz: an element is read for the last time before it is written
    for (int c = threadIdx.x; c < a.d; c += WIDE) {
      const float D = D_of(c), w = param(a.post_weight, c, 1.f), xh = (to_float(at<T>(a.x, row)[c]) - st.x) * st.y;
      const float e = e_of(c, D, xh, w, dg);
      if (a.sums[0]) slot[c] += e * xh;
      if (a.sums[1]) slot[(int64_t)a.d + c] += e;
      if (a.dr.p) at<R>(a.dr, row)[c] = from_float<R>(a.rscale * D);
      if (a.g.p) at<T>(a.dg, row)[c] = from_float<T>(dg);
      at<T>(a.dx, row)[c] = from_float<T>(st.y * (e * w - q[1] - xh * q[0]));
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
    for (int i = threadIdx.y; i < slots; i += 8 * SUM_LANES) {
      float v[8];  // on their way together: one after another 608 slots took 18 us
#pragma unroll
      for (int u = 0; u < 8; ++u) {
        const int j = i + u * SUM_LANES;
        v[u] = j < slots ? a.parts[((int64_t)j * 4 + k) * a.d + c] : 0.f;
      }
#pragma unroll
      for (int u = 0; u < 8; ++u) {
        const float s = sum + v[u], bb = s - sum;
        off += (sum - (s - bb)) + (v[u] - bb);
        sum = s;
      }
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
// Dynamic shared memory that a block may have; with the few hundred bytes of the kernels' own it is what
// an SM gives to one.
constexpr size_t ROOM = 226 << 10;

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
  // sixteen where registers hold them: 32,768 x 2,048 236 us, 65,536 x 1,024 235, with eight 255 and 250
  const bool biases = a.sums[1] || a.sums[3];
  const bool two = grad && s.v == 8 && type_bytes(wide) == 2 && !biases && d >= 1024 && d <= 8192;
  if (grad || s.v == 1) {  // eight elements a thread; the gradient's go with four sums of parameters' gradients
    s.packs = two ? 2 : 8 / s.v;
    s.block = d > 256;
  } else {
    s.block = vecs > 128;
    s.packs = s.block ? 2 : vecs <= 32 ? 1 : vecs <= 64 ? 2 : 4;
  }
  const int each = s.v * s.packs;
  s.threads = s.block ? ((d + each - 1) / each + 31) / 32 * 32 : 32;
  s.rows = s.block ? 1 : 8;
  // two rows of each block lie in shared memory; wider ones are read again for each sum
  const size_t b = type_bytes(type), w = type_bytes(wide);
  const size_t nt = grad ? 3 : 2, nr = grad ? 2 : 1;
  auto matrix = [&](size_t of) {  // the bytes of two rows
    if (s.v == 1) return of == 2 ? 2 * s.rows * ((size_t)d * 2 + 32) : 0;
    return 2 * (size_t)s.threads * s.rows * each * of;
  };
  const size_t held = s.v == 1 ? HELD_BYTES<1, 8> : 0;
  const size_t bytes = nt * matrix(b) + nr * matrix(w) + (size_t)s.threads * s.rows * held;
  // that registers are for
  const size_t threads = !grad ? 1024 : two ? 512 : s.v == 1 || biases ? 576 : 768;
  size_t most = 2;  // blocks of an SM
  if (s.threads > 1024 || bytes > ROOM) {
    s.packs = 0;
    s.threads = WIDE;
    s.block = true;
    s.rows = 1;
  } else {
    most = std::max<size_t>(1, std::min(ROOM / (bytes + 5120), threads / (s.threads * s.rows)));
  }
  s.grid = (unsigned)std::min<int64_t>((a.n + s.rows - 1) / s.rows, (int64_t)num_sms * (int64_t)most);
  const int64_t chain = (a.n + (int64_t)s.grid * s.rows - 1) / ((int64_t)s.grid * s.rows);
  s.slots = (int)((chain + CHAIN - 1) / CHAIN);
  return s;
}

// Two rows of each of a block's lie in shared memory.  own: what the kernel has without asking.  The limit is
// the kernel's on the device and not the call's, so it is the same each time, whatever other threads launch.
template <typename K, typename... A>
cudaError_t start(K kernel, size_t own, const Shape& h, size_t stage, size_t held, cudaStream_t s, A... args) {
  const size_t bytes = 2 * stage + held * h.threads * h.rows;
  const cudaError_t e = cudaFuncSetAttribute(kernel, cudaFuncAttributeMaxDynamicSharedMemorySize, (int)(ROOM - own));
  if (e != cudaSuccess) return e;
  return launch_following(kernel, dim3(h.grid), h.threads * h.rows, bytes, s, args...);
}

template <typename T, typename R, int V, int P>
cudaError_t forward_in(const ResNormArgs& a, const Shape& h, cudaStream_t s) {
  const size_t stage = stage_bytes<T, R, V, P>(2, 1, a.d, h.threads * h.rows, h.block);
  if (!h.block) return start(k_residual_norm<T, R, V, P, 0>, 0, h, stage, HELD_BYTES<V, P>, s, a);
  if constexpr (P <= 2 || V == 1) {  // four vectors a thread are a warp's
    if (h.threads <= 256) return start(k_residual_norm<T, R, V, P, 256>, 0, h, stage, HELD_BYTES<V, P>, s, a);
    return start(k_residual_norm<T, R, V, P, 1024>, 0, h, stage, HELD_BYTES<V, P>, s, a);
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

template <typename T, typename R, int V, int P, int B, bool BIAS>
cudaError_t backward_of(const ResNormArgs& a, const Shape& h, cudaStream_t s) {
  const size_t stage = stage_bytes<T, R, V, P>(3, 2, a.d, h.threads * h.rows, h.block);
  return start(k_residual_norm_grad<T, R, V, P, B, BIAS>, JOINED<V, P, (B > 0)> * sizeof(float), h, stage, HELD_BYTES<V, P>, s, a, h.slots);
}
template <typename T, typename R, int V, bool BIAS>
cudaError_t backward_as(const ResNormArgs& a, const Shape& h, cudaStream_t s) {
  constexpr int P = 8 / V;
  if constexpr (V == 8 && sizeof(R) == 2 && !BIAS)
    if (h.packs == 2) {
      if (h.threads <= 128) return backward_of<T, R, V, 2, 128, BIAS>(a, h, s);
      if (h.threads <= 256) return backward_of<T, R, V, 2, 256, BIAS>(a, h, s);
      return backward_of<T, R, V, 2, 512, BIAS>(a, h, s);
    }
  if (!h.block) return backward_of<T, R, V, P, 0, BIAS>(a, h, s);
  if (h.threads <= 256) return backward_of<T, R, V, P, 256, BIAS>(a, h, s);
  if (h.threads <= 512) return backward_of<T, R, V, P, 512, BIAS>(a, h, s);
  return backward_of<T, R, V, P, 1024, BIAS>(a, h, s);
}

template <typename T, typename R>
cudaError_t backward(const ResNormArgs& a, const Shape& h, cudaStream_t s) {
  constexpr int V = 16 / (int)sizeof(T);
  if (h.packs == 0) return launch_following(k_residual_norm_grad_wide<T, R>, dim3(h.grid), WIDE, 0, s, a, h.slots);
  if (h.v == 1) return backward_as<T, R, 1, true>(a, h, s);
  return a.sums[1] || a.sums[3] ? backward_as<T, R, V, true>(a, h, s) : backward_as<T, R, V, false>(a, h, s);
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

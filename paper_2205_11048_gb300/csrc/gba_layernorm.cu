// Layer norm over the columns of a row, forward and backward:
//   m = mean(x), v = mean((x - m)^2), r = 1 / sqrt(v + eps), h = (x - m) r, y = h gamma + beta
//   g = dy gamma, dx = r (g - mean(g) - h mean(g h)), dgamma = sum_rows dy h, dbeta = sum_rows dy
//
// Bound by HBM bandwidth: a row is read once, stays in registers while its statistics are
// formed (mean first, then the squares of the differences, so a large mean costs no digits),
// and is written once.  A narrow row is held by up to 32 lanes, one vector each; a wider one
// by up to 16 warps, each of which holds consecutive columns, and the loads of the next row
// are in flight while this one is reduced.  What a thread does for a row beside its columns
// (two sums over lanes and warps, a root, addresses) costs as many instructions as ten
// columns or so, so a thread of a wide row holds 64 bytes of it (backward 32 of each of the
// two), the arithmetic is done on pairs, and a warp whose columns all exist checks none of
// them.  Rows off the 16-byte boundary are read by the vectors that fit them, elements at
// worst: by aligned words and a shift, as the lookup reads them, f16 35,710 x 1,161 took 83 us
// against 49.  Backward, a block keeps its threads' shares of dgamma and dbeta in registers over
// all the rows it takes and leaves one partial row; a second kernel adds the partial rows in
// order; calls of very many rows are several such launches.  Rows too wide for a block's registers
// are read again from L2 instead.
//
// Measured, of the copy bandwidth of 6.7 TB/s: forward bf16 32,768 x 4,096 94 us (86%),
// 65,536 x 1,024 46.5 (86%), float32 16,384 x 4,096 88 (91%), f16 35,710 x 1,161 49 (50%, single
// elements); backward bf16 32,768 x 2,048 75 (80%), float32 8,192 x 4,096 68 (88%).
#include <algorithm>

#include "gba_worker.cuh"

namespace gba {

namespace {

constexpr int THREADS = 256;
constexpr int MOST_WARPS = 16;  // that hold a row
constexpr int WIDE_THREADS = 1024, WIDE_GRAD_THREADS = 512;  // of the kernels for rows of any width
constexpr uint32_t FULL = 0xffffffffu;

__device__ __forceinline__ float param_at(const void* p, int32_t type, int64_t i, float missing) {
  if (!p) return missing;
  if (type == GBA_F32) return static_cast<const float*>(p)[i];
  if (type == GBA_BF16) return to_float(static_cast<const bf16*>(p)[i]);
  return to_float(static_cast<const f16*>(p)[i]);
}

// V consecutive ones, c a multiple of V.
template <int V>
__device__ __forceinline__ void params_at(const void* p, int32_t type, int64_t c, float missing,
                                          float (&x)[V]) {
  if (p && (uintptr_t)p % 16 == 0) {
    if (type == GBA_F32) {
      Pack<float, V> w;
      w.load(static_cast<const float*>(p) + c);
      w.get(x);
    } else if (type == GBA_BF16) {
      Pack<bf16, V> w;
      w.load(static_cast<const bf16*>(p) + c);
      w.get(x);
    } else {
      Pack<f16, V> w;
      w.load(static_cast<const f16*>(p) + c);
      w.get(x);
    }
  } else {
#pragma unroll
    for (int j = 0; j < V; ++j) x[j] = param_at(p, type, c + j, missing);
  }
}

// ---- how a block's threads share rows ----------------------------------------------
// LANES: a row belongs to L lanes of a warp, and a lane's piece k of V columns is the row's
// piece k L + lane.  Otherwise it belongs to W warps, warp w holds the 32 E columns from
// 32 E w on, and a lane's piece k is the warp's piece 32 k + lane.
struct Split {
  int L, W;
};
template <int V, int E, bool LANES>
struct Place {
  int group, groups;  // of threads that hold a row: this thread's, and how many the block has
  int warp_group;     // the first group of the thread's warp: a warp's lanes go round together
  int t;              // this thread in its group
  int first;          // its first column
  int step;           // columns from one piece to the next
  bool whole;         // every column that the warp's threads hold exists
  __device__ __forceinline__ Place(const Split& s, int d) {
    const int lane = threadIdx.x & 31, warp = (int)threadIdx.x >> 5;
    if (LANES) {
      t = lane & (s.L - 1);
      group = (int)threadIdx.x / s.L;
      groups = (int)blockDim.x / s.L;
      warp_group = warp * (32 / s.L);
      first = t * V;
      step = s.L * V;
      whole = d == s.L * E;
    } else {
      const int w = warp % s.W;
      t = w * 32 + lane;
      group = warp_group = warp / s.W;
      groups = (int)blockDim.x / (32 * s.W);
      first = w * 32 * E + lane * V;
      step = 32 * V;
      whole = (w + 1) * 32 * E <= d;
    }
  }
};

// Sums of N values over the threads of a row, in every one of them.  s: N words per warp of
// the block; the caller alternates between two of them, so one barrier a sum is enough.
template <int N, bool LANES>
__device__ __forceinline__ void row_sum(float (&x)[N], const Split& sp, int group, float (*s)[N]) {
  if constexpr (LANES) {
    for (int o = 1; o < sp.L; o <<= 1)
#pragma unroll
      for (int i = 0; i < N; ++i) x[i] += __shfl_xor_sync(FULL, x[i], o);
  } else {
#pragma unroll
    for (int o = 1; o < 32; o <<= 1)
#pragma unroll
      for (int i = 0; i < N; ++i) x[i] += __shfl_xor_sync(FULL, x[i], o);
    if (sp.W == 1) return;
    const int warp = (int)threadIdx.x >> 5;
    if ((threadIdx.x & 31) == 0)
#pragma unroll
      for (int i = 0; i < N; ++i) s[warp][i] = x[i];
    asm volatile("bar.sync %0, %1;" ::"r"(group + 1), "r"(sp.W * 32) : "memory");
#pragma unroll
    for (int i = 0; i < N; ++i) x[i] = 0.f;
    for (int w = 0; w < sp.W; ++w)
#pragma unroll
      for (int i = 0; i < N; ++i) x[i] += s[group * sp.W + w][i];
  }
}

// A thread's E columns of a row, as they were loaded.  Pieces past the row's end hold zeros
// from clear() on.  left: columns from the thread's first one to the row's end.
template <typename T, int V, int E, bool WHOLE>
struct Held {
  static constexpr int K = E / V;
  Pack<T, V> p[K];
  __device__ __forceinline__ void clear() {
#pragma unroll
    for (int k = 0; k < K; ++k) p[k] = Pack<T, V>{};
  }
  static __device__ __forceinline__ bool has(int k, int step, int left) { return WHOLE || k * step < left; }
  __device__ __forceinline__ void load(const T* from, int step, int left) {
#pragma unroll
    for (int k = 0; k < K; ++k)
      if (has(k, step, left)) p[k].load(from + k * step);
  }
  __device__ __forceinline__ void get(f2 (&x)[E / 2]) const {
    float v[E];
#pragma unroll
    for (int k = 0; k < K; ++k) {
      float y[V];
      p[k].get(y);
#pragma unroll
      for (int j = 0; j < V; ++j) v[k * V + j] = y[j];
    }
#pragma unroll
    for (int i = 0; i < E / 2; ++i) x[i] = pair(v[2 * i], v[2 * i + 1]);
  }
  static __device__ __forceinline__ void store(T* to, const f2 (&x)[E / 2], int step, int left) {
    float v[E];
#pragma unroll
    for (int i = 0; i < E / 2; ++i) split(x[i], v[2 * i], v[2 * i + 1]);
#pragma unroll
    for (int k = 0; k < K; ++k) {
      if (!has(k, step, left)) continue;
      float y[V];
#pragma unroll
      for (int j = 0; j < V; ++j) y[j] = v[k * V + j];
      Pack<T, V> o;
      o.set(y);
      o.store(to + k * step);
    }
  }
};

// Columns that a thread holds: of a narrow row one vector; of a wide one, forward, 64 bytes
// (single elements of 16 bits take a register each, so 16 of those).
template <int V>
constexpr int E_LANES = V > 1 ? V : 2;
template <typename T, int V>
constexpr int E_NORM = V > 1 ? 64 / (int)sizeof(T) : 16;

// Shared memory keeps a parameter of column j of piece q, of Q pieces, where a lane's accesses
// of up to 16 bytes lie next to its neighbours'.
template <int V>
__device__ __forceinline__ int param_slot(int q, int j, int Q) {
  constexpr int H = V < 4 ? V : 4;
  return ((j / H) * Q + q) * H + j % H;
}

// One row, whose columns v holds: its statistics and output.  s_param: gamma at the thread's first
// piece; taken: called when every thread of the row has what it needs of its input.
template <typename T, int V, int E, bool LANES, bool WHOLE, int WARPS, typename F>
__device__ __forceinline__ void norm_row(const LayerNormArgs& a, const Split& sp, const Place<V, E, LANES>& at,
                                         int64_t row, f2 (&v)[E / 2], const float* gamma, int Q,
                                         float (*s_sum)[WARPS][1], F taken) {
  constexpr int K = E / V, P = E / 2, H = V < 4 ? V : 4;
  using Row = Held<T, V, E, WHOLE>;
  const int step = LANES ? at.step : 32 * V, left = a.d - at.first;
  const float inv_d = 1.f / (float)a.d;
  const bool live = row < a.n;
  f2 acc = v[0];
#pragma unroll
  for (int i = 1; i < P; ++i) acc = add2(acc, v[i]);
  float sum[1] = {both(acc)};
  row_sum<1, LANES>(sum, sp, at.group, s_sum[0]);
  taken();
  const float mean = sum[0] * inv_d;
#pragma unroll
  for (int i = 0; i < P; ++i) v[i] = add2(v[i], pair(-mean, -mean));
  if (!WHOLE) {
    float z[E];
#pragma unroll
    for (int i = 0; i < P; ++i) split(v[i], z[2 * i], z[2 * i + 1]);
#pragma unroll
    for (int e = 0; e < E; ++e) z[e] = Row::has(e / V, step, left) ? z[e] : 0.f;
#pragma unroll
    for (int i = 0; i < P; ++i) v[i] = pair(z[2 * i], z[2 * i + 1]);
  }
  acc = mul2(v[0], v[0]);
#pragma unroll
  for (int i = 1; i < P; ++i) acc = fma2(v[i], v[i], acc);
  sum[0] = both(acc);
  row_sum<1, LANES>(sum, sp, at.group, s_sum[1]);
  const float rstd = rsqrtf(sum[0] * inv_d + a.eps);
  if (live && at.t == 0) {
    if (a.mean) a.mean[row] = mean;
    if (a.rstd) a.rstd[row] = rstd;
  }
  if (!live) return;
  T* y = static_cast<T*>(a.y) + row * a.y_stride + at.first;
  float z[E];
#pragma unroll
  for (int i = 0; i < P; ++i) split(mul2(v[i], pair(rstd, rstd)), z[2 * i], z[2 * i + 1]);
#pragma unroll
  for (int k = 0; k < K; ++k) {
    if (!Row::has(k, step, left)) continue;
    float o[V];
#pragma unroll
    for (int h = 0; h < V / H; ++h) {
      Pack<float, H> g, b;
      float gj[H], bj[H];
      g.load(gamma + h * Q * H + k * (step / V) * H);
      b.load(gamma + Q * V + h * Q * H + k * (step / V) * H);
      g.get(gj);
      b.get(bj);
#pragma unroll
      for (int j = 0; j < H; ++j) o[h * H + j] = fmaf(z[k * V + h * H + j], gj[j], bj[j]);
    }
    Pack<T, V> w;
    w.set(o);
    w.store(y + k * step);
  }
}

template <typename T, int V, int E, bool LANES, bool WHOLE>
__device__ __forceinline__ void norm_rows(const LayerNormArgs& a, const Split& sp, const Place<V, E, LANES>& at,
                                          float* s_param, int Q, float (*s_sum)[MOST_WARPS][1]) {
  constexpr int H = V < 4 ? V : 4;
  const int step = LANES ? at.step : 32 * V, left = a.d - at.first;
  const int64_t per_pass = (int64_t)gridDim.x * at.groups;
  int64_t first = (int64_t)blockIdx.x * at.groups + at.warp_group;
  int64_t row = (int64_t)blockIdx.x * at.groups + at.group;
  const T* x = static_cast<const T*>(a.x) + at.first;
  const float* gamma = s_param + at.first / V * H;  // piece k of them is step / V pieces further
  Held<T, V, E, WHOLE> in;
  in.clear();
  if (row < a.n) in.load(x + row * a.x_stride, step, left);
  asm volatile("bar.sync 0;" ::: "memory");  // the parameters are there, for warps of either kind
  for (; first < a.n; first += per_pass, row += per_pass) {
    f2 v[E / 2];
    in.get(v);
    if (row + per_pass < a.n) in.load(x + (row + per_pass) * a.x_stride, step, left);
    norm_row<T, V, E, LANES, WHOLE>(a, sp, at, row, v, gamma, Q, s_sum, [] {});
  }
}

// gamma and beta (or 1 and 0) into shared memory, by the whole block.
template <int V>
__device__ __forceinline__ void fetch_params(const LayerNormArgs& a, float* s_param, int Q) {
  for (int c = threadIdx.x; c < a.d; c += blockDim.x) {
    const int o = param_slot<V>(c / V, c % V, Q);
    s_param[o] = param_at(a.gamma, a.param_type, c, 1.f);
    s_param[Q * V + o] = param_at(a.beta, a.param_type, c, 0.f);
  }
}

template <typename T, int V, int E, bool LANES>
__global__ void __launch_bounds__(LANES ? THREADS : 512) k_layer_norm(LayerNormArgs a, Split sp) {
  extern __shared__ __align__(16) float s_param[];  // gamma, beta: [2][columns held]
  __shared__ float s_sum[2][MOST_WARPS][1];
  follow();
  const Place<V, E, LANES> at(sp, a.d);
  const int Q = sp.L * sp.W * (E / V);
  fetch_params<V>(a, s_param, Q);
  if (at.whole)
    norm_rows<T, V, E, LANES, true>(a, sp, at, s_param, Q, s_sum);
  else
    norm_rows<T, V, E, LANES, false>(a, sp, at, s_param, Q, s_sum);
}

// Warps of a block.  Forward 20, or 24 for 16-bit rows of six warps and more: of eight, 24 warps
// hold three groups and 20 only two (8,192 x 8,192: 57 us against 65); others gain more from
// the registers that 20 leave a thread (16,384 x 5,120: 69 against 72.5; float32 16,384 x 4,096,
// in two groups of eight, 88 against 100.5).
constexpr int RING_WARPS = 20, RING_WARPS_MORE = 24, RING_WARPS_GRAD = 16;
constexpr int RING_ROWS = 4;     // a group takes at least
constexpr int E_GRAD_RING = 16;  // columns of a thread, backward

// ---- rows through a ring in shared memory ------------------------------------------------
// Many wide rows that start on 16 bytes come by bulk copies: a group of warps has `stages` rows
// on their way, which no register waits for.  One thread of the group issues the copies, every
// thread waits for them on the stage's barrier; a wait has a limit, after which the call's
// results are undefined, GBA_E_DEVICE_TIMEOUT is latched, and later waits are short.
struct Ring {
  uint64_t* full;  // [stages] of the group
  char* data;      // [stages][bytes] of the group
  int stages;
  uint32_t bytes;  // of a stage
  int64_t limit_ns;
  bool failed;

  __device__ __forceinline__ char* stage(int64_t i) const { return data + (size_t)(i % stages) * bytes; }
  __device__ __forceinline__ void wait(int64_t i, const ErrSink& err) {
    if (!mbar_wait(full + i % stages, (uint32_t)(i / stages) & 1u, failed ? 1000000ll : limit_ns) && !failed) {
      failed = true;
      raise_error(err, ERR_TIMEOUT);
    }
  }
};

// The block's rings, one for each group of threads, in dynamic shared memory.
__device__ __forceinline__ Ring make_ring(char* smem, int group, int groups, int stages, uint32_t bytes,
                                          int64_t limit_ns) {
  uint64_t* full = reinterpret_cast<uint64_t*>(smem);
  const size_t head = ((size_t)groups * stages * 8 + 127) / 128 * 128;
  Ring r;
  r.full = full + group * stages;
  r.data = smem + head + (size_t)group * stages * bytes;
  r.stages = stages;
  r.bytes = bytes;
  r.limit_ns = limit_ns;
  r.failed = false;
  if (threadIdx.x == 0) {
    for (int i = 0; i < groups * stages; ++i) mbar_init(full + i, 1u);
    asm volatile("fence.mbarrier_init.release.cluster;" ::: "memory");
    asm volatile("fence.proxy.async.shared::cta;" ::: "memory");
  }
  return r;
}

// A thread's pieces of a row in shared memory.
template <typename T, int V, int E, bool WHOLE>
__device__ __forceinline__ void from_stage(const char* stage, int first, int left, f2 (&x)[E / 2]) {
  Held<T, V, E, WHOLE> in;
  if (!WHOLE) in.clear();
  in.load(reinterpret_cast<const T*>(stage) + first, 32 * V, left);
  in.get(x);
}

template <typename T, int V, int E, bool WHOLE, int WARPS>
__device__ __forceinline__ void norm_ring(const LayerNormArgs& a, const Split& sp, const Place<V, E, false>& at,
                                          const float* s_param, int Q, float (*s_sum)[WARPS][1], Ring ring,
                                          const ErrSink& err) {
  constexpr int H = V < 4 ? V : 4;
  const int64_t per_pass = (int64_t)gridDim.x * at.groups, row0 = (int64_t)blockIdx.x * at.groups + at.group;
  auto issue = [&](int64_t i) {
    const int64_t row = row0 + i * per_pass;
    if (at.t != 0 || row >= a.n || ring.failed) return;  // after a failure no barrier is armed twice
    uint64_t* bar = ring.full + i % ring.stages;
    mbar_arrive_expect_tx(bar, ring.bytes);
    bulk_g2s(ring.stage(i), static_cast<const T*>(a.x) + row * a.x_stride, ring.bytes, bar);
  };
  for (int i = 0; i < ring.stages; ++i) issue(i);
  const float* gamma = s_param + at.first / V * H;
  int64_t i = 0;
  for (int64_t row = row0; row < a.n; row += per_pass, ++i) {
    ring.wait(i, err);
    f2 v[E / 2];
    from_stage<T, V, E, WHOLE>(ring.stage(i), at.first, a.d - at.first, v);
    // past the row's first sum every thread has read the stage
    norm_row<T, V, E, false, WHOLE>(a, sp, at, row, v, gamma, Q, s_sum, [&] { issue(i + ring.stages); });
  }
}

template <typename T, int V, int E, int WARPS>
__global__ void __launch_bounds__(WARPS * 32, 1)
    k_layer_norm_ring(LayerNormArgs a, Split sp, int stages, ErrSink err, int64_t limit_ns) {
  extern __shared__ __align__(128) char s_ring[];  // parameters, barriers, rows
  __shared__ float s_sum[2][WARPS][1];
  const Place<V, E, false> at(sp, a.d);
  const int Q = 32 * sp.W * (E / V);
  float* s_param = reinterpret_cast<float*>(s_ring);
  const Ring ring = make_ring(s_ring + (size_t)2 * Q * V * sizeof(float), at.group, at.groups, stages,
                              (uint32_t)(a.d * sizeof(T)), limit_ns);
  follow();
  fetch_params<V>(a, s_param, Q);
  __syncthreads();
  if (at.whole)
    norm_ring<T, V, E, true, WARPS>(a, sp, at, s_param, Q, s_sum, ring, err);
  else
    norm_ring<T, V, E, false, WARPS>(a, sp, at, s_param, Q, s_sum, ring, err);
}

// Rows of any width: one block each, read three times.
template <typename T, int V>
__global__ void __launch_bounds__(WIDE_THREADS) k_layer_norm_wide(LayerNormArgs a) {
  __shared__ float s_sum[2][32][1];
  follow();
  const float inv_d = 1.f / (float)a.d;
  const int64_t step = (int64_t)blockDim.x * V;
  for (int64_t row = blockIdx.x; row < a.n; row += gridDim.x) {
    const T* x = static_cast<const T*>(a.x) + row * a.x_stride;
    T* y = static_cast<T*>(a.y) + row * a.y_stride;
    float sum[1] = {0.f}, v[V];
    Pack<T, V> w;
    for (int64_t c = (int64_t)threadIdx.x * V; c < a.d; c += step) {
      w.load(x + c);
      w.get(v);
#pragma unroll
      for (int j = 0; j < V; ++j) sum[0] += v[j];
    }
    row_sum<1, false>(sum, Split{32, WIDE_THREADS / 32}, 0, s_sum[0]);
    const float mean = sum[0] * inv_d;
    sum[0] = 0.f;
    for (int64_t c = (int64_t)threadIdx.x * V; c < a.d; c += step) {
      w.load(x + c);
      w.get(v);
#pragma unroll
      for (int j = 0; j < V; ++j) sum[0] = fmaf(v[j] - mean, v[j] - mean, sum[0]);
    }
    row_sum<1, false>(sum, Split{32, WIDE_THREADS / 32}, 0, s_sum[1]);
    const float rstd = rsqrtf(sum[0] * inv_d + a.eps);
    if (threadIdx.x == 0) {
      if (a.mean) a.mean[row] = mean;
      if (a.rstd) a.rstd[row] = rstd;
    }
    for (int64_t c = (int64_t)threadIdx.x * V; c < a.d; c += step) {
      w.load(x + c);
      w.get(v);
      float gamma[V], beta[V];
      params_at<V>(a.gamma, a.param_type, c, 1.f, gamma);
      params_at<V>(a.beta, a.param_type, c, 0.f, beta);
#pragma unroll
      for (int j = 0; j < V; ++j) v[j] = fmaf((v[j] - mean) * rstd, gamma[j], beta[j]);
      w.set(v);
      w.store(y + c);
    }
  }
}

// Columns that a thread of the gradient holds of a wide row: as many as leave room for the
// weights, the two sums, and the loads of this row and (FETCH) the next one.
template <typename T, int V>
constexpr int E_GRAD = sizeof(T) == 2 && V > 1 ? 16 : 8;

// A thread's columns of gamma, 0 past the row's end.
template <int V, int E, bool WHOLE>
__device__ __forceinline__ void params_of(const LayerNormArgs& a, int first, int step, f2 (&gamma)[E / 2]) {
  float y[E];
#pragma unroll
  for (int k = 0; k < E / V; ++k) {
    float z[V];
#pragma unroll
    for (int j = 0; j < V; ++j) z[j] = 0.f;
    if (WHOLE || first + k * step < a.d) params_at<V>(a.gamma, a.param_type, first + k * step, 1.f, z);
#pragma unroll
    for (int j = 0; j < V; ++j) y[k * V + j] = z[j];
  }
#pragma unroll
  for (int i = 0; i < E / 2; ++i) gamma[i] = pair(y[2 * i], y[2 * i + 1]);
}

// Adds a row's share to dg and db, and gives the thread's share of the row's sums of g and g h.
// (m: the negative mean; g: dy, which is 0 past the row's end, and so are its products.)
template <int P>
__device__ __forceinline__ void grad_sums(const f2 (&x)[P], const f2 (&g)[P], f2 m, f2 r, const f2 (&gamma)[P],
                                          f2 (&dg)[P], f2 (&db)[P], float (&sum)[2]) {
  f2 s0 = pair(0.f, 0.f), s1 = s0;
#pragma unroll
  for (int i = 0; i < P; ++i) {
    const f2 h = mul2(add2(x[i], m), r);
    db[i] = add2(db[i], g[i]);
    dg[i] = fma2(g[i], h, dg[i]);
    const f2 gg = mul2(g[i], gamma[i]);
    s0 = add2(s0, gg);
    s1 = fma2(gg, h, s1);
  }
  sum[0] = both(s0);
  sum[1] = both(s1);
}

// dx of a row, in the place of dy.
template <int P>
__device__ __forceinline__ void grad_out(const f2 (&x)[P], f2 (&g)[P], f2 m, f2 r, const f2 (&gamma)[P], float mg,
                                         float mgh) {
  const f2 nmg = pair(-mg, -mg), nmgh = pair(-mgh, -mgh);
#pragma unroll
  for (int i = 0; i < P; ++i) {
    const f2 h = mul2(add2(x[i], m), r);
    g[i] = mul2(r, fma2(h, nmgh, fma2(g[i], gamma[i], nmg)));
  }
}

// dx of the rows that this thread's group takes, and its shares of dgamma and dbeta.  What a
// thread keeps of a row while its sums are formed is its loads; h and g are formed from them
// twice.
template <typename T, int V, int E, bool LANES, bool FETCH, bool WHOLE>
__device__ __forceinline__ void grad_rows(const LayerNormArgs& a, const Split& sp, const Place<V, E, LANES>& at,
                                          float (*s_sum)[MOST_WARPS][2], f2 (&dg)[E / 2], f2 (&db)[E / 2]) {
  constexpr int P = E / 2;
  using Row = Held<T, V, E, WHOLE>;
  using Next = Held<T, V, FETCH ? E : V, WHOLE>;
  const int step = LANES ? at.step : 32 * V, left = a.d - at.first;
  const int64_t per_pass = (int64_t)gridDim.x * at.groups;
  const float inv_d = 1.f / (float)a.d;
  f2 gamma[P];
  params_of<V, E, WHOLE>(a, at.first, step, gamma);
  Row xin, din;
  Next xnext, dnext;
  xin.clear();
  din.clear();
  xnext.clear();
  dnext.clear();
  float mean = 0.f, rstd = 0.f, mnext = 0.f, rnext = 0.f;
  auto fetch = [&](int64_t row, auto& xs, auto& ds, float& m, float& r) {
    if (row >= a.n) {  // adds nothing
      xs.clear();
      ds.clear();
      m = r = 0.f;
      return;
    }
    xs.load(static_cast<const T*>(a.x) + row * a.x_stride + at.first, step, left);
    ds.load(static_cast<const T*>(a.dy) + row * a.dy_stride + at.first, step, left);
    m = a.mean[row];
    r = a.rstd[row];
  };
  int64_t row = (int64_t)blockIdx.x * at.groups + at.group;
  int64_t first = (int64_t)blockIdx.x * at.groups + at.warp_group;
  if (FETCH) fetch(row, xnext, dnext, mnext, rnext);
  int flip = 0;
  for (; first < a.n; first += per_pass, row += per_pass) {
    if constexpr (FETCH) {
      xin = xnext;
      din = dnext;
      mean = mnext;
      rstd = rnext;
      fetch(row + per_pass, xnext, dnext, mnext, rnext);
    } else {
      fetch(row, xin, din, mean, rstd);
    }
    const f2 m = pair(-mean, -mean), r = pair(rstd, rstd);
    float sum[2];
    {
      f2 x[P], g[P];
      xin.get(x);
      din.get(g);
      grad_sums<P>(x, g, m, r, gamma, dg, db, sum);
    }
    row_sum<2, LANES>(sum, sp, at.group, s_sum[flip]);
    flip ^= 1;
    if (row >= a.n) continue;
    f2 x[P], g[P];
    xin.get(x);
    din.get(g);
    grad_out<P>(x, g, m, r, gamma, sum[0] * inv_d, sum[1] * inv_d);
    Row::store(static_cast<T*>(a.y) + row * a.y_stride + at.first, g, step, left);
  }
}

// One partial row of dgamma and dbeta per block, [2][blocks][d]: the block's groups of threads
// are added in order, first those within a warp, then through shared memory (s_part: a value for
// each column that the block's threads hold).
template <int V, int E, bool LANES>
__device__ __forceinline__ void write_partial(const LayerNormArgs& a, const Split& sp,
                                              const Place<V, E, LANES>& at, const f2 (&dg)[E / 2],
                                              const f2 (&db)[E / 2], float* s_part) {
  constexpr int K = E / V, P = E / 2;
  __syncwarp();
  float mine[2][E];
#pragma unroll
  for (int i = 0; i < P; ++i) {
    split(dg[i], mine[0][2 * i], mine[0][2 * i + 1]);
    split(db[i], mine[1][2 * i], mine[1][2 * i + 1]);
  }
  if (LANES)
#pragma unroll
    for (int which = 0; which < 2; ++which)
#pragma unroll
      for (int e = 0; e < E; ++e)
        for (int o = sp.L; o < 32; o <<= 1) mine[which][e] += __shfl_xor_sync(FULL, mine[which][e], o);
  const int sets = LANES ? (int)blockDim.x >> 5 : at.groups;
  const int set = LANES ? (int)threadIdx.x >> 5 : at.group, width = sp.L * sp.W * E;
  const bool one_of = !LANES || (int)(threadIdx.x & 31) < sp.L;
#pragma unroll
  for (int which = 0; which < 2; ++which) {
    float* out = a.parts + ((int64_t)which * gridDim.x + blockIdx.x) * a.d;
#pragma unroll
    for (int k = 0; k < K; ++k) {
      const int c = at.first + k * at.step;
      if (!one_of || c >= a.d) continue;
#pragma unroll
      for (int j = 0; j < V; ++j) {
        if (sets == 1)
          out[c + j] = mine[which][k * V + j];
        else
          s_part[set * width + c + j] = mine[which][k * V + j];
      }
    }
    if (sets == 1) continue;
    __syncthreads();
    for (int c = threadIdx.x; c < a.d; c += blockDim.x) {
      float x = 0.f;
      for (int g = 0; g < sets; ++g) x += s_part[g * width + c];
      out[c] = x;
    }
    __syncthreads();
  }
}

template <typename T, int V, int E, bool LANES, bool FETCH>
__global__ void __launch_bounds__(LANES ? THREADS : 512) k_layer_norm_grad(LayerNormArgs a, Split sp) {
  constexpr int P = E / 2;
  __shared__ float s_sum[2][MOST_WARPS][2];
  __shared__ float s_part[THREADS * E];
  follow();
  const Place<V, E, LANES> at(sp, a.d);
  f2 dg[P], db[P];
#pragma unroll
  for (int i = 0; i < P; ++i) dg[i] = db[i] = pair(0.f, 0.f);
  // The checks of a row's end leave no registers for the next row's loads beside 16 columns of 16
  // bits (f16 136,696 x 432: 107 us with them in flight, 79 without).
  constexpr bool AHEAD = FETCH && !(sizeof(T) == 2 && E == 16);
  if (at.whole)
    grad_rows<T, V, E, LANES, FETCH, true>(a, sp, at, s_sum, dg, db);
  else
    grad_rows<T, V, E, LANES, AHEAD, false>(a, sp, at, s_sum, dg, db);
  write_partial<V, E, LANES>(a, sp, at, dg, db, s_part);
}

// The gradient's rows through the ring, x and dy of a row in one stage.  A row's stage is read
// twice, so it is free when every thread has come to the next row's sums.
template <typename T, int V, int E, bool WHOLE>
__device__ __forceinline__ void grad_ring(const LayerNormArgs& a, const Split& sp, const Place<V, E, false>& at,
                                          float (*s_sum)[RING_WARPS_GRAD][2], Ring ring, const ErrSink& err,
                                          f2 (&dg)[E / 2], f2 (&db)[E / 2]) {
  constexpr int P = E / 2;
  using Row = Held<T, V, E, WHOLE>;
  const int left = a.d - at.first;
  const int64_t per_pass = (int64_t)gridDim.x * at.groups, row0 = (int64_t)blockIdx.x * at.groups + at.group;
  const float inv_d = 1.f / (float)a.d;
  const uint32_t half = ring.bytes / 2;
  auto issue = [&](int64_t i) {
    const int64_t row = row0 + i * per_pass;
    if (at.t != 0 || row >= a.n || ring.failed) return;  // after a failure no barrier is armed twice
    uint64_t* bar = ring.full + i % ring.stages;
    mbar_arrive_expect_tx(bar, ring.bytes);
    bulk_g2s(ring.stage(i), static_cast<const T*>(a.x) + row * a.x_stride, half, bar);
    bulk_g2s(ring.stage(i) + half, static_cast<const T*>(a.dy) + row * a.dy_stride, half, bar);
  };
  for (int i = 0; i < ring.stages; ++i) issue(i);
  f2 gamma[P];
  params_of<V, E, WHOLE>(a, at.first, 32 * V, gamma);
  float mean = row0 < a.n ? a.mean[row0] : 0.f, rstd = row0 < a.n ? a.rstd[row0] : 0.f;
  int64_t i = 0;
  for (int64_t row = row0; row < a.n; row += per_pass, ++i) {
    ring.wait(i, err);
    const char* stage = ring.stage(i);
    const f2 m = pair(-mean, -mean), r = pair(rstd, rstd);
    if (row + per_pass < a.n) {
      mean = a.mean[row + per_pass];
      rstd = a.rstd[row + per_pass];
    }
    float sum[2];
    f2 x[P], g[P];
    from_stage<T, V, E, WHOLE>(stage, at.first, left, x);
    from_stage<T, V, E, WHOLE>(stage + half, at.first, left, g);
    grad_sums<P>(x, g, m, r, gamma, dg, db, sum);
    row_sum<2, false>(sum, sp, at.group, s_sum[i & 1]);
    if (i > 0) issue(i - 1 + ring.stages);
    from_stage<T, V, E, WHOLE>(stage, at.first, left, x);
    from_stage<T, V, E, WHOLE>(stage + half, at.first, left, g);
    grad_out<P>(x, g, m, r, gamma, sum[0] * inv_d, sum[1] * inv_d);
    Row::store(static_cast<T*>(a.y) + row * a.y_stride + at.first, g, 32 * V, left);
  }
}

template <typename T, int V, int E>
__global__ void __launch_bounds__(RING_WARPS_GRAD * 32, 1)
    k_layer_norm_grad_ring(LayerNormArgs a, Split sp, int stages, ErrSink err, int64_t limit_ns) {
  constexpr int P = E / 2;
  extern __shared__ __align__(128) char s_ring[];  // barriers, rows; in the end the partial rows
  __shared__ float s_sum[2][RING_WARPS_GRAD][2];
  const Place<V, E, false> at(sp, a.d);
  const Ring ring = make_ring(s_ring, at.group, at.groups, stages, (uint32_t)(2 * a.d * sizeof(T)), limit_ns);
  follow();
  __syncthreads();
  f2 dg[P], db[P];
#pragma unroll
  for (int i = 0; i < P; ++i) dg[i] = db[i] = pair(0.f, 0.f);
  if (at.whole)
    grad_ring<T, V, E, true>(a, sp, at, s_sum, ring, err, dg, db);
  else
    grad_ring<T, V, E, false>(a, sp, at, s_sum, ring, err, dg, db);
  __syncthreads();  // no row is read any more
  write_partial<V, E, false>(a, sp, at, dg, db,
                             reinterpret_cast<float*>(s_ring + ((size_t)at.groups * stages * 8 + 127) / 128 * 128));
}

// Rows of any width: dx by one block a row, read twice.
template <typename T, int V>
__global__ void __launch_bounds__(WIDE_GRAD_THREADS) k_layer_norm_grad_wide(LayerNormArgs a) {
  __shared__ float s_sum[2][WIDE_GRAD_THREADS / 32][2];
  follow();
  const float inv_d = 1.f / (float)a.d;
  const int64_t step = (int64_t)blockDim.x * V;
  int flip = 0;
  for (int64_t row = blockIdx.x; row < a.n; row += gridDim.x) {
    const T* x = static_cast<const T*>(a.x) + row * a.x_stride;
    const T* dy = static_cast<const T*>(a.dy) + row * a.dy_stride;
    T* dx = static_cast<T*>(a.y) + row * a.y_stride;
    const float mean = a.mean[row], rstd = a.rstd[row];
    float sum[2] = {0.f, 0.f}, h[V], g[V];
    Pack<T, V> w;
    for (int64_t c = (int64_t)threadIdx.x * V; c < a.d; c += step) {
      w.load(x + c);
      w.get(h);
      w.load(dy + c);
      w.get(g);
      float gamma[V];
      params_at<V>(a.gamma, a.param_type, c, 1.f, gamma);
#pragma unroll
      for (int j = 0; j < V; ++j) {
        const float gj = g[j] * gamma[j];
        sum[0] += gj;
        sum[1] = fmaf(gj, (h[j] - mean) * rstd, sum[1]);
      }
    }
    row_sum<2, false>(sum, Split{32, WIDE_GRAD_THREADS / 32}, 0, s_sum[flip]);
    flip ^= 1;
    const float mg = sum[0] * inv_d, mgh = sum[1] * inv_d;
    for (int64_t c = (int64_t)threadIdx.x * V; c < a.d; c += step) {
      w.load(x + c);
      w.get(h);
      w.load(dy + c);
      w.get(g);
      float gamma[V];
      params_at<V>(a.gamma, a.param_type, c, 1.f, gamma);
#pragma unroll
      for (int j = 0; j < V; ++j)
        g[j] = rstd * (g[j] * gamma[j] - mg - (h[j] - mean) * rstd * mgh);
      w.set(g);
      w.store(dx + c);
    }
  }
}

// Partial rows of dgamma and dbeta of rows of any width: a thread's V columns over every
// gridDim.y-th row.  Runs before the kernel that writes dx, which may be dy.
template <typename T, int V>
__global__ void __launch_bounds__(THREADS) k_layer_norm_columns(LayerNormArgs a) {
  follow();
  const int64_t c = ((int64_t)blockIdx.x * THREADS + threadIdx.x) * V;
  if (c >= a.d) return;
  float dg[V], db[V];
#pragma unroll
  for (int j = 0; j < V; ++j) dg[j] = db[j] = 0.f;
  for (int64_t row = blockIdx.y; row < a.n; row += gridDim.y) {
    Pack<T, V> wx, wd;
    float x[V], dy[V];
    wx.load(static_cast<const T*>(a.x) + row * a.x_stride + c);
    wd.load(static_cast<const T*>(a.dy) + row * a.dy_stride + c);
    wx.get(x);
    wd.get(dy);
    const float mean = a.mean[row], rstd = a.rstd[row];
#pragma unroll
    for (int j = 0; j < V; ++j) {
      db[j] += dy[j];
      dg[j] = fmaf(dy[j], (x[j] - mean) * rstd, dg[j]);
    }
  }
#pragma unroll
  for (int j = 0; j < V; ++j) {
    a.parts[(int64_t)blockIdx.y * a.d + c + j] = dg[j];
    a.parts[((int64_t)gridDim.y + blockIdx.y) * a.d + c + j] = db[j];
  }
}

// The partial rows of a launch of `parts` blocks, [2][parts][d], or of `chunks` such launches (MANY),
// added in order: a block takes 32 columns, each of its warps a share of every launch's rows.
// blockIdx.y: dgamma or dbeta.
template <bool MANY>
__global__ void __launch_bounds__(1024) k_layer_norm_params(LayerNormArgs a, int parts, int chunks) {
  constexpr int WARPS = 32;
  __shared__ float s[WARPS][33];
  follow();
  float* out = blockIdx.y == 0 ? a.dgamma : a.dbeta;
  if (!out) return;
  const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
  const int64_t c = (int64_t)blockIdx.x * 32 + lane;
  const float* p = a.parts + (int64_t)blockIdx.y * parts * a.d;
  const int each = (parts + WARPS - 1) / WARPS;
  const int lo = min(parts, warp * each), hi = min(parts, lo + each);
  float x = 0.f;
  if (c < a.d)
#pragma unroll 8
    for (int i = lo; i < hi; ++i) x += p[(int64_t)i * a.d + c];
  if (MANY)
    for (int k = 1; k < chunks; ++k) {
      p += (int64_t)2 * parts * a.d;
      float y = 0.f;
      if (c < a.d)
#pragma unroll 8
        for (int i = lo; i < hi; ++i) y += p[(int64_t)i * a.d + c];
      x += y;
    }
  s[warp][lane] = x;
  __syncthreads();
  if (warp == 0 && c < a.d) {
#pragma unroll 8
    for (int w = 1; w < WARPS; ++w) x += s[w][lane];
    out[c] = x;
  }
}

// ---- launches ------------------------------------------------------------------------

constexpr int64_t WIDE_SPLIT = 64;  // rows of blocks of k_layer_norm_columns, at least
// The most rows that a thread adds to its share of dgamma and dbeta, one after the other in float32.
// Calls of more rows are several launches, whose partial rows are added in the end, so that what
// the sums lose does not grow with the rows (dbeta of 5 10^6 x 1,003 equal float32: off by 2.2e-6 of
// itself, and by 4.6e-5 in one launch; 10^6 x 1,040 float32 2.06 ms, and 2.00 in one).
constexpr int64_t CHAIN = 512;

// The lanes of a narrow row of d columns, E to a lane.
Split lanes_of(int32_t d, int E) {
  Split s{1, 1};
  while (s.L * E < d) s.L <<= 1;
  return s;
}

// The warps of a wide row, E columns to a lane, and the threads of a block of such rows.
Split warps_of(int32_t d, int E, int* threads) {
  const Split s{32, (d + 32 * E - 1) / (32 * E)};
  *threads = 32 * s.W * std::max(1, THREADS / (32 * s.W));
  return s;
}

// Lets launches of a kernel on the current device use `most` bytes of dynamic shared memory.  The
// attribute belongs to a device and a process may use several, so each launch of more than
// SMEM_FREE sets it (48 KB are allowed without, the kernel's own included).
constexpr size_t SMEM_FREE = 47 * 1024;
template <typename F>
cudaError_t allow_smem(F* kernel, size_t most) {
  return cudaFuncSetAttribute(kernel, cudaFuncAttributeMaxDynamicSharedMemorySize, (int)most);
}

// Blocks of a kernel for wide rows that an SM holds, for each number of warps of a row.  The answers
// depend on the attribute, which comes first, and are those of any device that runs this
// architecture's code.
struct Residency {
  int blocks[MOST_WARPS + 1];
  template <typename F, typename S>
  Residency(F* kernel, int E, S smem_of) {
    if (smem_of(MOST_WARPS) > SMEM_FREE) allow_smem(kernel, smem_of(MOST_WARPS));
    for (int w = 1; w <= MOST_WARPS; ++w) {
      int threads;
      warps_of(w * 32 * E, E, &threads);
      const size_t smem = smem_of(w);
      blocks[w] = 0;
      if (cudaOccupancyMaxActiveBlocksPerMultiprocessor(&blocks[w], kernel, threads, smem) != cudaSuccess ||
          blocks[w] < 1)
        blocks[w] = 1;
    }
  }
};
// And of one for narrow rows.
template <typename F>
int resident(F* kernel, size_t smem) {
  int blocks = 0;
  return cudaOccupancyMaxActiveBlocksPerMultiprocessor(&blocks, kernel, THREADS, smem) == cudaSuccess && blocks > 0
             ? blocks
             : 1;
}

unsigned grid_of(int64_t n, const Split& s, int threads, int num_sms, int per_sm) {
  const int64_t rows = threads / (s.L * s.W);  // a block's
  return (unsigned)std::min<int64_t>((n + rows - 1) / rows, (int64_t)num_sms * per_sm);
}

// A block of a ring kernel: one per SM, of up to `most` warps, with as many stages (up to
// four) as 200 KB of shared memory leave room for beside `fixed` bytes.
struct RingShape {
  Split split;
  int groups, stages;
  size_t smem;
};
RingShape ring_of(int32_t d, int E, int most, size_t stage_bytes, size_t fixed) {
  RingShape r;
  int threads;
  r.split = warps_of(d, E, &threads);
  r.groups = std::max(1, most / r.split.W);
  const size_t room = 200 * 1024 - fixed;
  r.stages = (int)std::min<size_t>(4, room / ((size_t)r.groups * stage_bytes));
  while (r.stages < 2 && r.groups > 1) {
    --r.groups;
    r.stages = (int)std::min<size_t>(4, room / ((size_t)r.groups * stage_bytes));
  }
  r.smem = fixed + ((size_t)r.groups * r.stages * 8 + 127) / 128 * 128 + (size_t)r.groups * r.stages * stage_bytes;
  return r;
}
// Does a ring serve n rows?  With a few rows a group its setting up costs more than it saves.
bool ring_serves(const RingShape& r, int64_t n, int num_sms) {
  return r.split.W >= 2 && r.stages >= 2 && n >= (int64_t)RING_ROWS * r.groups * num_sms;
}
template <typename F>
cudaError_t launch_ring(F* kernel, const RingShape& r, const LayerNormArgs& a, const RingWait& w, unsigned grid,
                        cudaStream_t s) {
  const cudaError_t e = allow_smem(kernel, 220 * 1024);
  if (e != cudaSuccess) return e;
  return launch_following(kernel, dim3(grid), 32 * r.split.W * r.groups, r.smem, s, a, r.split, r.stages, w.err, w.limit_ns);
}

template <typename T, int V, int E>
cudaError_t norm_wide(const LayerNormArgs& a, int num_sms, cudaStream_t s) {
  auto smem_of = [](int w) { return (size_t)w * 32 * E * 2 * sizeof(float); };
  static const Residency held(k_layer_norm<T, V, E, false>, E, smem_of);
  int threads;
  const Split sp = warps_of(a.d, E, &threads);
  if (smem_of(sp.W) > SMEM_FREE) {  // the same limit each time, whatever other threads launch
    const cudaError_t e = allow_smem(k_layer_norm<T, V, E, false>, smem_of(MOST_WARPS));
    if (e != cudaSuccess) return e;
  }
  return launch_following(k_layer_norm<T, V, E, false>,
                          dim3(grid_of(a.n, sp, threads, num_sms, held.blocks[sp.W])), threads, smem_of(sp.W), s, a,
                          sp);
}

template <typename T, int V>
cudaError_t norm_as(const LayerNormArgs& a, const RingWait& w, int num_sms, cudaStream_t s) {
  constexpr int EL = E_LANES<V>, E = E_NORM<T, V>;
  if constexpr (V * sizeof(T) == 16)
    if (a.d > 32 * E && a.d <= MOST_WARPS * 32 * E) {
      int threads;
      const size_t params = (size_t)warps_of(a.d, E, &threads).W * 32 * E * 2 * sizeof(float);
      const bool more = sizeof(T) == 2 && warps_of(a.d, E, &threads).W >= 6;
      const RingShape r = ring_of(a.d, E, more ? RING_WARPS_MORE : RING_WARPS, (size_t)a.d * sizeof(T), params);
      if (ring_serves(r, a.n, num_sms)) {
        auto kernel = k_layer_norm_ring<T, V, E, RING_WARPS>;
        if constexpr (sizeof(T) == 2)
          if (more) kernel = k_layer_norm_ring<T, V, E, RING_WARPS_MORE>;
        return launch_ring(kernel, r, a, w, (unsigned)std::min<int64_t>(num_sms, (a.n + r.groups - 1) / r.groups), s);
      }
    }
  if (a.d <= 32 * EL) {
    constexpr size_t smem = (size_t)32 * EL * 2 * sizeof(float);
    static const int held = resident(k_layer_norm<T, V, EL, true>, smem);
    const Split sp = lanes_of(a.d, EL);
    return launch_following(k_layer_norm<T, V, EL, true>, dim3(grid_of(a.n, sp, THREADS, num_sms, held)), THREADS,
                            smem, s, a, sp);
  }
  if (a.d > MOST_WARPS * 32 * E)
    return launch_following(k_layer_norm_wide<T, V>, dim3((unsigned)std::min<int64_t>(a.n, num_sms * 2)),
                            WIDE_THREADS, 0, s, a);
  // rows of one warp and two or three vectors a lane hold no more than that (bf16 100,000 x 400:
  // 33 us, and 52 with four)
  if constexpr (E > 2 * V && V > 1) {
    if (a.d <= 64 * V) return norm_wide<T, V, 2 * V>(a, num_sms, s);
    if (a.d <= 96 * V) return norm_wide<T, V, 3 * V>(a, num_sms, s);
  }
  return norm_wide<T, V, E>(a, num_sms, s);
}

// How a gradient's rows are held: a vector a lane, with the next row's loads in flight, without
// (rows of up to 8,192 columns that are read by 8 columns a thread), or not at all.
enum class Way { LANES, FETCH, PLAIN, WIDE, RING };
struct GradShape {
  Way way;
  RingShape ring;
  Split split;
  int threads;
  int parts;  // blocks of a launch, and its partial rows
  int chunks;    // launches
  int64_t rows;  // of each
  // A block holds `groups` rows at a time.
  void split_rows(int64_t n, int groups) {
    const int64_t per_pass = (int64_t)parts * groups, passes = (n + per_pass - 1) / per_pass;
    chunks = (int)((passes + CHAIN - 1) / CHAIN);
    rows = (passes + chunks - 1) / chunks * per_pass;
  }
};

// float32 rows come through the ring (4,096 x 8,192: 82 us from registers, 69 this way).  16-bit ones
// do not: what bounds them is the instructions that widen them, twice in either way, and
// reading shared memory adds to those (32,768 x 2,048: 75 us from registers, 87 this way, 82
// with the loads kept in registers between the two).
template <typename T, int V>
constexpr bool GRAD_RING = sizeof(T) == 4 && V == 4;

template <typename T, int V>
GradShape grad_shape(const LayerNormArgs& a, int num_sms) {
  constexpr int EL = E_LANES<V>, E = E_GRAD<T, V>;
  GradShape g{};
  if (a.d <= 32 * EL) {
    static const int held = resident(k_layer_norm_grad<T, V, EL, true, true>, 0);
    g.way = Way::LANES;
    g.split = lanes_of(a.d, EL);
    g.threads = THREADS;
    g.parts = (int)grid_of(a.n, g.split, g.threads, num_sms, held);
    g.split_rows(a.n, g.threads / g.split.L);
    return g;
  }
  if constexpr (GRAD_RING<T, V>)
    if (a.d <= RING_WARPS_GRAD * 32 * E_GRAD_RING) {
      // (the partial rows take the stages' place in the end)
      g.ring = ring_of(a.d, E_GRAD_RING, RING_WARPS_GRAD, (size_t)2 * a.d * sizeof(T), 0);
      if (ring_serves(g.ring, a.n, num_sms)) {
        g.way = Way::RING;
        g.parts = (int)std::min<int64_t>(num_sms, (a.n + g.ring.groups - 1) / g.ring.groups);
        g.split_rows(a.n, g.ring.groups);
        return g;
      }
    }
  if (a.d <= MOST_WARPS * 32 * E) {
    static const Residency held(k_layer_norm_grad<T, V, E, false, true>, E, [](int) { return (size_t)0; });
    g.way = Way::FETCH;
    g.split = warps_of(a.d, E, &g.threads);
    g.parts = (int)grid_of(a.n, g.split, g.threads, num_sms, held.blocks[g.split.W]);
    g.split_rows(a.n, g.threads / (32 * g.split.W));
  } else if (E < 16 && a.d <= MOST_WARPS * 32 * 16) {
    g.way = Way::PLAIN;
    g.split = warps_of(a.d, 16, &g.threads);
    g.parts = (int)grid_of(a.n, g.split, g.threads, num_sms, 1);
    g.split_rows(a.n, g.threads / (32 * g.split.W));
  } else {
    g.way = Way::WIDE;
    g.parts = (int)std::min(a.n, std::min<int64_t>(65535, std::max(WIDE_SPLIT, (a.n + CHAIN - 1) / CHAIN)));
    g.chunks = 1;
    g.rows = a.n;
  }
  return g;
}

template <typename T, int V>
cudaError_t grad_as(const LayerNormArgs& a, const RingWait& w, int num_sms, cudaStream_t s) {
  constexpr int EL = E_LANES<V>, E = E_GRAD<T, V>;
  const GradShape g = grad_shape<T, V>(a, num_sms);
  cudaError_t e = cudaSuccess;
  if (g.way == Way::WIDE) {
    const int64_t per = (int64_t)THREADS * V;
    e = launch_following(k_layer_norm_columns<T, V>, dim3((unsigned)((a.d + per - 1) / per), (unsigned)g.parts),
                         THREADS, 0, s, a);
    if (e == cudaSuccess)
      e = launch_following(k_layer_norm_grad_wide<T, V>, dim3((unsigned)std::min<int64_t>(a.n, num_sms * 4)),
                           WIDE_GRAD_THREADS, 0, s, a);
  } else {
    auto kernel = g.way == Way::LANES ? k_layer_norm_grad<T, V, EL, true, true> : k_layer_norm_grad<T, V, E, false, true>;
    if constexpr (E < 16)
      if (g.way == Way::PLAIN) kernel = k_layer_norm_grad<T, V, 16, false, false>;
    LayerNormArgs c = a;
    for (int k = 0; k < g.chunks; ++k) {
      const int64_t first = k * g.rows;
      c.x = static_cast<const T*>(a.x) + first * a.x_stride;
      c.dy = static_cast<const T*>(a.dy) + first * a.dy_stride;
      c.y = static_cast<T*>(a.y) + first * a.y_stride;
      c.mean = a.mean + first;
      c.rstd = a.rstd + first;
      c.n = std::min(g.rows, a.n - first);
      c.parts = a.parts + (size_t)k * 2 * g.parts * a.d;
      e = cudaErrorInvalidValue;
      if (g.way != Way::RING)
        e = launch_following(kernel, dim3(g.parts), g.threads, 0, s, c, g.split);
      else if constexpr (GRAD_RING<T, V>)
        e = launch_ring(k_layer_norm_grad_ring<T, V, E_GRAD_RING>, g.ring, c, w, (unsigned)g.parts, s);
      if (e != cudaSuccess) return e;
    }
  }
  if (e != cudaSuccess || (!a.dgamma && !a.dbeta)) return e;
  return launch_following(g.chunks > 1 ? k_layer_norm_params<true> : k_layer_norm_params<false>, dim3((unsigned)((a.d + 31) / 32), 2), 1024, 0, s, a, g.parts, g.chunks);
}

// Calls f with the vector width of a's matrices.
template <typename T, typename F>
auto with_vector(const LayerNormArgs& a, F f) {
  constexpr int most = 16 / (int)sizeof(T);
  int v = std::min(vector_of(most, a.x, a.x_stride, a.d, sizeof(T)),
                   vector_of(most, a.y, a.y_stride, a.d, sizeof(T)));
  if (a.dy) v = std::min(v, vector_of(most, a.dy, a.dy_stride, a.d, sizeof(T)));
  if constexpr (most == 8)
    if (v == 8) return f(std::integral_constant<int, 8>());
  if (v == 4) return f(std::integral_constant<int, 4>());
  if (v == 2) return f(std::integral_constant<int, 2>());
  return f(std::integral_constant<int, 1>());
}

template <typename F>
auto with_type(int32_t type, const LayerNormArgs& a, F f) {
  if (type == GBA_F32) return with_vector<float>(a, [&](auto v) { return f(float(), v); });
  if (type == GBA_BF16) return with_vector<bf16>(a, [&](auto v) { return f(bf16(), v); });
  return with_vector<f16>(a, [&](auto v) { return f(f16(), v); });
}

}  // namespace

cudaError_t launch_layer_norm(const LayerNormArgs& a, int32_t type, const RingWait& w, int num_sms,
                              cudaStream_t s) {
  return with_type(type, a, [&](auto x, auto v) { return norm_as<decltype(x), v()>(a, w, num_sms, s); });
}

size_t layer_norm_grad_workspace(const LayerNormArgs& a, int32_t type, int num_sms) {
  const size_t parts = with_type(type, a, [&](auto x, auto v) {
    const GradShape g = grad_shape<decltype(x), v()>(a, num_sms);
    return (size_t)g.parts * g.chunks;
  });
  return parts * 2 * (size_t)a.d * sizeof(float);
}

cudaError_t launch_layer_norm_grad(const LayerNormArgs& a, int32_t type, const RingWait& w, int num_sms,
                                   cudaStream_t s) {
  return with_type(type, a, [&](auto x, auto v) { return grad_as<decltype(x), v()>(a, w, num_sms, s); });
}

}  // namespace gba

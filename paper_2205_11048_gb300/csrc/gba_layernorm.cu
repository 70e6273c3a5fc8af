// Layer norm over the columns of a row, forward and backward:
//   m = mean(x), v = mean((x - m)^2), r = 1 / sqrt(v + eps), h = (x - m) r, y = h gamma + beta
//   g = dy gamma, dx = r (g - mean(g) - h mean(g h)), dgamma = sum_rows dy h, dbeta = sum_rows dy
//
// Bound by HBM bandwidth: a row is read once, stays in registers while its statistics are
// formed (mean first, then the squares of the differences, so a large mean costs no digits),
// and is written once.  A row is held by 1 << lg threads of up to 16 columns each.  Backward,
// a block keeps its threads' shares of dgamma and dbeta in registers over all the rows it
// takes and leaves one partial row; a second kernel adds the partial rows in order.  Rows too wide for a block's registers are read again from L2 instead.
#include <algorithm>

#include "gba_worker.cuh"

namespace gba {

namespace {

constexpr int THREADS = 256;
constexpr int EPT = 16;      // columns a thread holds, forward
constexpr int MOST_LG = 10;  // so rows of up to 16,384 columns stay in registers
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

// Sums of N values over the 1 << lg threads of a row, in every one of them.  s: a word per
// warp and value; the caller alternates two of them, so one barrier is enough.
template <int N>
__device__ __forceinline__ void row_sum(float (&x)[N], int lg, float (*s)[N]) {
  const int in_warp = lg < 5 ? lg : 5;
#pragma unroll
  for (int i = 0; i < N; ++i)
    for (int o = 1; o < 1 << in_warp; o <<= 1) x[i] += __shfl_xor_sync(FULL, x[i], o);
  if (lg <= 5) return;
  const int warp = threadIdx.x >> 5;
  if ((threadIdx.x & 31) == 0)
#pragma unroll
    for (int i = 0; i < N; ++i) s[warp][i] = x[i];
  __syncthreads();
  const int warps = 1 << (lg - 5), first = warp & ~(warps - 1);
#pragma unroll
  for (int i = 0; i < N; ++i) x[i] = 0.f;
  for (int w = 0; w < warps; ++w)
#pragma unroll
    for (int i = 0; i < N; ++i) x[i] += s[first + w][i];
}

// KEEP: a thread's parameters stay in registers over all the rows its block takes.  The next
// row's loads are in flight while this one is reduced.
template <typename T, int V, bool KEEP>
__global__ void __launch_bounds__(KEEP ? 512 : 1024) k_layer_norm(LayerNormArgs a, int lg) {
  constexpr int K = EPT / V;
  __shared__ float s_sum[2][32][1];
  follow();
  const int tpr = 1 << lg, t = threadIdx.x & (tpr - 1);
  const int64_t per_pass = (int64_t)gridDim.x * ((int)blockDim.x >> lg);
  const float inv_d = 1.f / (float)a.d;
  float gamma[KEEP ? K : 1][V], beta[KEEP ? K : 1][V];
  if (KEEP)
#pragma unroll
    for (int k = 0; k < K; ++k) {
      const int c = (k * tpr + t) * V;
      if (c < a.d) {
        params_at<V>(a.gamma, a.param_type, c, 1.f, gamma[k]);
        params_at<V>(a.beta, a.param_type, c, 0.f, beta[k]);
      }
    }
  Pack<T, V> in[K];
  auto fetch = [&](int64_t row) {
    const T* x = static_cast<const T*>(a.x) + row * a.x_stride;
#pragma unroll
    for (int k = 0; k < K; ++k) {
      const int c = (k * tpr + t) * V;
      if (row < a.n && c < a.d) in[k].load(x + c);
    }
  };
  int64_t row = (int64_t)blockIdx.x * ((int)blockDim.x >> lg) + (threadIdx.x >> lg);
  // all threads of a block go round equally often: they meet in the sums
  int64_t first = (int64_t)blockIdx.x * ((int)blockDim.x >> lg);
  fetch(row);
  for (; first < a.n; first += per_pass, row += per_pass) {
    const bool live = row < a.n;
    T* y = static_cast<T*>(a.y) + row * a.y_stride;
    float v[K][V];
    float sum[1] = {0.f};
#pragma unroll
    for (int k = 0; k < K; ++k) {
      const int c = (k * tpr + t) * V;
      if (live && c < a.d)
        in[k].get(v[k]);
      else
#pragma unroll
        for (int j = 0; j < V; ++j) v[k][j] = 0.f;
#pragma unroll
      for (int j = 0; j < V; ++j) sum[0] += v[k][j];
    }
    fetch(row + per_pass);
    row_sum<1>(sum, lg, s_sum[0]);
    const float mean = sum[0] * inv_d;
    sum[0] = 0.f;
#pragma unroll
    for (int k = 0; k < K; ++k) {
      const int c = (k * tpr + t) * V;
      if (c < a.d)
#pragma unroll
        for (int j = 0; j < V; ++j) {
          v[k][j] -= mean;
          sum[0] = fmaf(v[k][j], v[k][j], sum[0]);
        }
    }
    row_sum<1>(sum, lg, s_sum[1]);
    const float rstd = 1.f / sqrtf(sum[0] * inv_d + a.eps);
    if (live && t == 0) {
      if (a.mean) a.mean[row] = mean;
      if (a.rstd) a.rstd[row] = rstd;
    }
#pragma unroll
    for (int k = 0; k < K; ++k) {
      const int c = (k * tpr + t) * V;
      if (!live || c >= a.d) continue;
      float* gk = gamma[KEEP ? k : 0];
      float* bk = beta[KEEP ? k : 0];
      if (!KEEP) {
        params_at<V>(a.gamma, a.param_type, c, 1.f, gamma[0]);
        params_at<V>(a.beta, a.param_type, c, 0.f, beta[0]);
      }
#pragma unroll
      for (int j = 0; j < V; ++j) v[k][j] = fmaf(v[k][j] * rstd, gk[j], bk[j]);
      Pack<T, V> o;
      o.set(v[k]);
      o.store(y + c);
    }
  }
}

// Rows of any width: one block each, read three times.
template <typename T, int V>
__global__ void __launch_bounds__(1024) k_layer_norm_wide(LayerNormArgs a) {
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
    row_sum<1>(sum, 10, s_sum[0]);
    const float mean = sum[0] * inv_d;
    sum[0] = 0.f;
    for (int64_t c = (int64_t)threadIdx.x * V; c < a.d; c += step) {
      w.load(x + c);
      w.get(v);
#pragma unroll
      for (int j = 0; j < V; ++j) sum[0] = fmaf(v[j] - mean, v[j] - mean, sum[0]);
    }
    row_sum<1>(sum, 10, s_sum[1]);
    const float rstd = 1.f / sqrtf(sum[0] * inv_d + a.eps);
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

// Columns that a thread of the gradient holds: as many as leave room for the weights, the two
// sums, and the loads of this row and the next one.
template <typename T, int V>
constexpr int EPT_GRAD = sizeof(T) == 2 && V > 1 ? 16 : 8;

// One partial row of dgamma and dbeta per block: [2][blocks][d].  What a thread keeps of a row
// while its sums are formed is its loads; h and g are formed from them twice.  FETCH: the
// next row's loads are in flight meanwhile.
template <typename T, int V, bool FETCH>
__global__ void __launch_bounds__(FETCH ? 512 : 1024) k_layer_norm_grad(LayerNormArgs a, int lg) {
  constexpr int EPT_ = EPT_GRAD<T, V>, K = EPT_ / V;
  __shared__ float s_sum[2][32][2];
  __shared__ float s_part[THREADS * EPT_];
  follow();
  const int tpr = 1 << lg, t = threadIdx.x & (tpr - 1);
  const int per_block = (int)blockDim.x >> lg;
  const int64_t per_pass = (int64_t)gridDim.x * per_block;
  const float inv_d = 1.f / (float)a.d;
  float gamma[K][V], dg[K][V], db[K][V];
#pragma unroll
  for (int k = 0; k < K; ++k) {
    const int c = (k * tpr + t) * V;
    if (c < a.d) params_at<V>(a.gamma, a.param_type, c, 1.f, gamma[k]);
#pragma unroll
    for (int j = 0; j < V; ++j) dg[k][j] = db[k][j] = 0.f;
  }
  Pack<T, V> xin[K], din[K], xnext[FETCH ? K : 1], dnext[FETCH ? K : 1];
  float mean = 0.f, rstd = 0.f, mnext = 0.f, rnext = 0.f;
  auto fetch = [&](int64_t row, Pack<T, V>* xs, Pack<T, V>* ds, float& m, float& r) {
    if (row >= a.n) return;
    const T* x = static_cast<const T*>(a.x) + row * a.x_stride;
    const T* dy = static_cast<const T*>(a.dy) + row * a.dy_stride;
#pragma unroll
    for (int k = 0; k < K; ++k) {
      const int c = (k * tpr + t) * V;
      if (c < a.d) {
        xs[k].load(x + c);
        ds[k].load(dy + c);
      }
    }
    m = a.mean[row];
    r = a.rstd[row];
  };
  int64_t first = (int64_t)blockIdx.x * per_block;
  int64_t row = first + ((int)threadIdx.x >> lg);
  if (FETCH) fetch(row, xnext, dnext, mnext, rnext);
  int flip = 0;
  for (; first < a.n; first += per_pass, row += per_pass) {
    const bool live = row < a.n;
    if constexpr (FETCH) {
#pragma unroll
      for (int k = 0; k < K; ++k) {
        xin[k] = xnext[k];
        din[k] = dnext[k];
      }
      mean = mnext;
      rstd = rnext;
      fetch(row + per_pass, xnext, dnext, mnext, rnext);
    } else {
      fetch(row, xin, din, mean, rstd);
    }
    float sum[2] = {0.f, 0.f};
#pragma unroll
    for (int k = 0; k < K; ++k) {
      const int c = (k * tpr + t) * V;
      if (!live || c >= a.d) continue;
      float x[V], g[V];
      xin[k].get(x);
      din[k].get(g);
#pragma unroll
      for (int j = 0; j < V; ++j) {
        const float h = (x[j] - mean) * rstd;
        db[k][j] += g[j];
        dg[k][j] = fmaf(g[j], h, dg[k][j]);
        g[j] *= gamma[k][j];
        sum[0] += g[j];
        sum[1] = fmaf(g[j], h, sum[1]);
      }
    }
    row_sum<2>(sum, lg, s_sum[flip]);
    flip ^= 1;
    const float mg = sum[0] * inv_d, mgh = sum[1] * inv_d;
    T* dx = static_cast<T*>(a.y) + row * a.y_stride;
#pragma unroll
    for (int k = 0; k < K; ++k) {
      const int c = (k * tpr + t) * V;
      if (!live || c >= a.d) continue;
      float x[V], g[V];
      xin[k].get(x);
      din[k].get(g);
#pragma unroll
      for (int j = 0; j < V; ++j) {
        const float h = (x[j] - mean) * rstd;
        g[j] = rstd * (g[j] * gamma[k][j] - mg - h * mgh);
      }
      Pack<T, V> o;
      o.set(g);
      o.store(dx + c);
    }
  }
  // the block's groups of threads, in order: first those within a warp, then through shared memory
#pragma unroll
  for (int k = 0; k < K; ++k)
#pragma unroll
    for (int j = 0; j < V; ++j)
      for (int o = tpr; o < 32; o <<= 1) {
        dg[k][j] += __shfl_xor_sync(FULL, dg[k][j], o);
        db[k][j] += __shfl_xor_sync(FULL, db[k][j], o);
      }
  const int lgw = lg < 5 ? 5 : lg;
  const int groups = (int)blockDim.x >> lgw, group = (int)threadIdx.x >> lgw, width = tpr * EPT_;
  const bool one_of = lg >= 5 || (threadIdx.x & 31) < tpr;
#pragma unroll
  for (int which = 0; which < 2; ++which) {
    float* out = a.parts + ((int64_t)which * gridDim.x + blockIdx.x) * a.d;
    float(*mine)[V] = which == 0 ? dg : db;
#pragma unroll
    for (int k = 0; k < K; ++k) {
      const int c = (k * tpr + t) * V;
      if (!one_of || c >= a.d) continue;
#pragma unroll
      for (int j = 0; j < V; ++j) {
        if (groups == 1)
          out[c + j] = mine[k][j];
        else
          s_part[group * width + c + j] = mine[k][j];
      }
    }
    if (groups == 1) continue;
    __syncthreads();
    for (int c = threadIdx.x; c < a.d; c += blockDim.x) {
      float x = 0.f;
      for (int g = 0; g < groups; ++g) x += s_part[g * width + c];
      out[c] = x;
    }
    __syncthreads();
  }
}

// Rows of any width: dx by one block a row, read twice.
template <typename T, int V>
__global__ void __launch_bounds__(512) k_layer_norm_grad_wide(LayerNormArgs a) {
  __shared__ float s_sum[2][16][2];
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
    row_sum<2>(sum, 9, s_sum[flip]);
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

// The partial rows, added in order: a block takes 32 columns, each of its warps a share of
// the rows.  blockIdx.y: dgamma or dbeta.
__global__ void __launch_bounds__(1024) k_layer_norm_params(LayerNormArgs a, int parts) {
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
  s[warp][lane] = x;
  __syncthreads();
  if (warp == 0 && c < a.d) {
#pragma unroll 8
    for (int w = 1; w < WARPS; ++w) x += s[w][lane];
    out[c] = x;
  }
}

int lg_of(int32_t d, int ept) {
  int lg = 0;
  while (((int64_t)ept << lg) < d) ++lg;
  return lg;
}

// Blocks of the register kernels, and threads of each.
struct Shape {
  unsigned grid, threads;
};
Shape shape_of(int64_t n, int lg, int num_sms, int threads_per_sm) {
  const unsigned threads = std::max(THREADS, 1 << lg);
  const int64_t blocks = (n + (threads >> lg) - 1) / (threads >> lg);
  return Shape{(unsigned)std::min<int64_t>(blocks, (int64_t)num_sms * (threads_per_sm / (int)threads)), threads};
}
// Threads of a kernel that an SM holds, in blocks of so many.
template <typename F>
int threads_per_sm(F* kernel, int threads) {
  int blocks = 0;
  if (cudaOccupancyMaxActiveBlocksPerMultiprocessor(&blocks, kernel, threads, 0) != cudaSuccess || blocks < 1)
    blocks = 1;
  return blocks * threads;
}
constexpr int64_t WIDE_SPLIT = 64;  // rows of blocks of k_layer_norm_columns

template <typename T, int V>
cudaError_t norm_as(const LayerNormArgs& a, int num_sms, cudaStream_t s) {
  const int lg = lg_of(a.d, EPT);
  if (lg > MOST_LG)
    return launch_following(k_layer_norm_wide<T, V>, dim3((unsigned)std::min<int64_t>(a.n, num_sms * 2)), 1024,
                            0, s, a);
  if (lg == MOST_LG) {
    const Shape sh = shape_of(a.n, lg, num_sms, 1024);
    return launch_following(k_layer_norm<T, V, false>, dim3(sh.grid), sh.threads, 0, s, a, lg);
  }
  static const int held[2] = {threads_per_sm(k_layer_norm<T, V, true>, THREADS),
                              threads_per_sm(k_layer_norm<T, V, true>, 2 * THREADS)};
  const Shape sh = shape_of(a.n, lg, num_sms, held[lg == 9]);
  return launch_following(k_layer_norm<T, V, true>, dim3(sh.grid), sh.threads, 0, s, a, lg);
}

// The kernel of a gradient: rows of up to 8,192 columns stay in registers.
enum class Way { FETCH, PLAIN, WIDE };
struct GradShape {
  Way way;
  int lg;
  Shape shape;
  int parts;  // partial rows
};

template <typename T, int V>
GradShape grad_shape(const LayerNormArgs& a, int num_sms) {
  GradShape g{};
  g.lg = lg_of(a.d, EPT_GRAD<T, V>);
  if (a.d > 8192) {
    g.way = Way::WIDE;
    g.parts = (int)std::min(a.n, WIDE_SPLIT);
    return g;
  }
  g.way = g.lg <= 9 ? Way::FETCH : Way::PLAIN;
  static const int held[2] = {threads_per_sm(k_layer_norm_grad<T, V, true>, THREADS),
                              threads_per_sm(k_layer_norm_grad<T, V, true>, 2 * THREADS)};
  g.shape = shape_of(a.n, g.lg, num_sms, g.way == Way::PLAIN ? 1024 : held[g.lg == 9]);
  g.parts = (int)g.shape.grid;
  return g;
}

template <typename T, int V>
cudaError_t grad_as(const LayerNormArgs& a, int num_sms, cudaStream_t s) {
  const GradShape g = grad_shape<T, V>(a, num_sms);
  cudaError_t e;
  if (g.way == Way::WIDE) {
    const int64_t per = (int64_t)THREADS * V;
    e = launch_following(k_layer_norm_columns<T, V>, dim3((unsigned)((a.d + per - 1) / per), (unsigned)g.parts),
                         THREADS, 0, s, a);
    if (e == cudaSuccess)
      e = launch_following(k_layer_norm_grad_wide<T, V>, dim3((unsigned)std::min<int64_t>(a.n, num_sms * 4)),
                           512, 0, s, a);
  } else {
    auto kernel = k_layer_norm_grad<T, V, true>;
    if constexpr (EPT_GRAD<T, V> == 8)  // the others hold 8,192 columns in 512 threads
      if (g.way == Way::PLAIN) kernel = k_layer_norm_grad<T, V, false>;
    e = launch_following(kernel, dim3(g.shape.grid), g.shape.threads, 0, s, a, g.lg);
  }
  if (e != cudaSuccess || (!a.dgamma && !a.dbeta)) return e;
  return launch_following(k_layer_norm_params, dim3((unsigned)((a.d + 31) / 32), 2), 1024, 0, s, a, g.parts);
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

cudaError_t launch_layer_norm(const LayerNormArgs& a, int32_t type, int num_sms, cudaStream_t s) {
  return with_type(type, a, [&](auto x, auto v) { return norm_as<decltype(x), v()>(a, num_sms, s); });
}

size_t layer_norm_grad_workspace(const LayerNormArgs& a, int32_t type, int num_sms) {
  const int parts = with_type(type, a, [&](auto x, auto v) { return grad_shape<decltype(x), v()>(a, num_sms).parts; });
  return (size_t)parts * 2 * (size_t)a.d * sizeof(float);
}

cudaError_t launch_layer_norm_grad(const LayerNormArgs& a, int32_t type, int num_sms,
                                   cudaStream_t s) {
  return with_type(type, a, [&](auto x, auto v) { return grad_as<decltype(x), v()>(a, num_sms, s); });
}

}  // namespace gba

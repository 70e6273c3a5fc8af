// Layer norm over the columns of a row, forward and backward:
//   m = mean(x), v = mean((x - m)^2), r = 1 / sqrt(v + eps), h = (x - m) r, y = h gamma + beta
//   g = dy gamma, dx = r (g - mean(g) - h mean(g h)), dgamma = sum_rows dy h, dbeta = sum_rows dy
//
// Bound by HBM bandwidth: a row is read once, stays in registers while its statistics are
// formed (mean first, then the squares of the differences, so a large mean costs no digits),
// and is written once.  A row is held by 1 << lg threads of 16 columns each.  Backward, a
// block keeps its threads' shares of dgamma and dbeta in registers over all the rows it
// takes and leaves one partial row per group of threads; a second kernel adds the partial
// rows in order.  Rows too wide for a block's registers are read again from L2 instead.
#include <algorithm>

#include "gba_worker.cuh"

namespace gba {

namespace {

constexpr int THREADS = 256;
constexpr int EPT = 16;          // columns a thread holds
constexpr int MOST_LG = 10;      // forward: rows of up to 16,384 columns in registers
constexpr int MOST_LG_GRAD = 9;  // backward: 8,192
constexpr uint32_t FULL = 0xffffffffu;

__device__ __forceinline__ float param_at(const void* p, int32_t type, int64_t i, float missing) {
  if (!p) return missing;
  if (type == GBA_F32) return static_cast<const float*>(p)[i];
  if (type == GBA_BF16) return to_float(static_cast<const bf16*>(p)[i]);
  return to_float(static_cast<const f16*>(p)[i]);
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

template <typename T, int V>
__global__ void __launch_bounds__(1024) k_layer_norm(LayerNormArgs a, int lg) {
  constexpr int K = EPT / V;
  __shared__ float s_sum[2][32][1];
  follow();
  const int tpr = 1 << lg, t = threadIdx.x & (tpr - 1);
  const int per_block = (int)blockDim.x >> lg;
  const float inv_d = 1.f / (float)a.d;
  for (int64_t r0 = (int64_t)blockIdx.x * per_block; r0 < a.n; r0 += (int64_t)gridDim.x * per_block) {
    const int64_t row = r0 + (threadIdx.x >> lg);
    const bool live = row < a.n;
    const T* x = static_cast<const T*>(a.x) + row * a.x_stride;
    T* y = static_cast<T*>(a.y) + row * a.y_stride;
    Pack<T, V> in[K];
#pragma unroll
    for (int k = 0; k < K; ++k) {
      const int c = (k * tpr + t) * V;
      if (live && c < a.d) in[k].load(x + c);
    }
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
#pragma unroll
      for (int j = 0; j < V; ++j)
        v[k][j] = fmaf(v[k][j] * rstd, param_at(a.gamma, a.param_type, c + j, 1.f),
                       param_at(a.beta, a.param_type, c + j, 0.f));
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
#pragma unroll
      for (int j = 0; j < V; ++j)
        v[j] = fmaf((v[j] - mean) * rstd, param_at(a.gamma, a.param_type, c + j, 1.f),
                    param_at(a.beta, a.param_type, c + j, 0.f));
      w.set(v);
      w.store(y + c);
    }
  }
}

// Partial rows of dgamma and dbeta: [2][parts][d].
template <typename T, int V>
__global__ void __launch_bounds__(512) k_layer_norm_grad(LayerNormArgs a, int lg) {
  constexpr int K = EPT / V;
  __shared__ float s_sum[2][16][2];
  follow();
  const int tpr = 1 << lg, t = threadIdx.x & (tpr - 1), group = (int)threadIdx.x >> lg;
  const int per_block = (int)blockDim.x >> lg;
  const float inv_d = 1.f / (float)a.d;
  float gamma[K][V], dg[K][V], db[K][V];
#pragma unroll
  for (int k = 0; k < K; ++k)
#pragma unroll
    for (int j = 0; j < V; ++j) {
      const int c = (k * tpr + t) * V + j;
      gamma[k][j] = c < a.d ? param_at(a.gamma, a.param_type, c, 1.f) : 0.f;
      dg[k][j] = db[k][j] = 0.f;
    }
  int flip = 0;
  for (int64_t r0 = (int64_t)blockIdx.x * per_block; r0 < a.n; r0 += (int64_t)gridDim.x * per_block) {
    const int64_t row = r0 + group;
    const bool live = row < a.n;
    const T* x = static_cast<const T*>(a.x) + row * a.x_stride;
    const T* dy = static_cast<const T*>(a.dy) + row * a.dy_stride;
    T* dx = static_cast<T*>(a.y) + row * a.y_stride;
    Pack<T, V> xin[K], din[K];
#pragma unroll
    for (int k = 0; k < K; ++k) {
      const int c = (k * tpr + t) * V;
      if (live && c < a.d) {
        xin[k].load(x + c);
        din[k].load(dy + c);
      }
    }
    const float mean = live ? a.mean[row] : 0.f, rstd = live ? a.rstd[row] : 0.f;
    float h[K][V], g[K][V];
    float sum[2] = {0.f, 0.f};
#pragma unroll
    for (int k = 0; k < K; ++k) {
      const int c = (k * tpr + t) * V;
      if (live && c < a.d) {
        xin[k].get(h[k]);
        din[k].get(g[k]);
#pragma unroll
        for (int j = 0; j < V; ++j) {
          h[k][j] = (h[k][j] - mean) * rstd;
          db[k][j] += g[k][j];
          dg[k][j] = fmaf(g[k][j], h[k][j], dg[k][j]);
          g[k][j] *= gamma[k][j];
          sum[0] += g[k][j];
          sum[1] = fmaf(g[k][j], h[k][j], sum[1]);
        }
      }
    }
    row_sum<2>(sum, lg, s_sum[flip]);
    flip ^= 1;
    const float mg = sum[0] * inv_d, mgh = sum[1] * inv_d;
#pragma unroll
    for (int k = 0; k < K; ++k) {
      const int c = (k * tpr + t) * V;
      if (!live || c >= a.d) continue;
#pragma unroll
      for (int j = 0; j < V; ++j) g[k][j] = rstd * (g[k][j] - mg - h[k][j] * mgh);
      Pack<T, V> o;
      o.set(g[k]);
      o.store(dx + c);
    }
  }
  const int64_t part = (int64_t)blockIdx.x * per_block + group, parts = (int64_t)gridDim.x * per_block;
#pragma unroll
  for (int k = 0; k < K; ++k) {
    const int c = (k * tpr + t) * V;
    if (c >= a.d) continue;
#pragma unroll
    for (int j = 0; j < V; ++j) {
      a.parts[part * a.d + c + j] = dg[k][j];
      a.parts[(parts + part) * a.d + c + j] = db[k][j];
    }
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
#pragma unroll
      for (int j = 0; j < V; ++j) {
        const float gj = g[j] * param_at(a.gamma, a.param_type, c + j, 1.f);
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
#pragma unroll
      for (int j = 0; j < V; ++j)
        g[j] = rstd * (g[j] * param_at(a.gamma, a.param_type, c + j, 1.f) - mg - (h[j] - mean) * rstd * mgh);
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

// The partial rows, added in order: a block takes 32 columns, its 8 warps a share of the rows
// each.  blockIdx.y: dgamma or dbeta.
__global__ void __launch_bounds__(THREADS) k_layer_norm_params(LayerNormArgs a, int64_t parts) {
  constexpr int WARPS = THREADS / 32;
  __shared__ float s[WARPS][33];
  follow();
  float* out = blockIdx.y == 0 ? a.dgamma : a.dbeta;
  if (!out) return;
  const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
  const int64_t c = (int64_t)blockIdx.x * 32 + lane;
  const float* p = a.parts + (int64_t)blockIdx.y * parts * a.d;
  const int64_t each = (parts + WARPS - 1) / WARPS;
  const int64_t lo = warp * each, hi = lo + each < parts ? lo + each : parts;
  float x = 0.f;
  if (c < a.d)
#pragma unroll 8
    for (int64_t i = lo; i < hi; ++i) x += p[i * a.d + c];
  s[warp][lane] = x;
  __syncthreads();
  if (warp == 0 && c < a.d) {
    for (int w = 1; w < WARPS; ++w) x += s[w][lane];
    out[c] = x;
  }
}

int lg_of(int32_t d) {
  int lg = 0;
  while (((int64_t)EPT << lg) < d) ++lg;
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
constexpr int GRAD_THREADS_PER_SM = 512;
constexpr int64_t WIDE_SPLIT = 64;  // rows of blocks of k_layer_norm_columns

template <typename T, int V>
cudaError_t norm_as(const LayerNormArgs& a, int num_sms, cudaStream_t s) {
  const int lg = lg_of(a.d);
  if (lg > MOST_LG)
    return launch_following(k_layer_norm_wide<T, V>, dim3((unsigned)std::min<int64_t>(a.n, num_sms * 2)), 1024,
                            0, s, a);
  const Shape sh = shape_of(a.n, lg, num_sms, 2048);
  return launch_following(k_layer_norm<T, V>, dim3(sh.grid), sh.threads, 0, s, a, lg);
}

template <typename T, int V>
cudaError_t grad_as(const LayerNormArgs& a, int num_sms, cudaStream_t s) {
  const int lg = lg_of(a.d);
  int64_t parts;
  cudaError_t e;
  if (lg > MOST_LG_GRAD) {
    parts = std::min(a.n, WIDE_SPLIT);
    const int64_t per = (int64_t)THREADS * V;
    e = launch_following(k_layer_norm_columns<T, V>, dim3((unsigned)((a.d + per - 1) / per), (unsigned)parts),
                         THREADS, 0, s, a);
    if (e == cudaSuccess)
      e = launch_following(k_layer_norm_grad_wide<T, V>, dim3((unsigned)std::min<int64_t>(a.n, num_sms * 4)),
                           512, 0, s, a);
  } else {
    const Shape sh = shape_of(a.n, lg, num_sms, GRAD_THREADS_PER_SM);
    parts = (int64_t)sh.grid * (sh.threads >> lg);
    e = launch_following(k_layer_norm_grad<T, V>, dim3(sh.grid), sh.threads, 0, s, a, lg);
  }
  if (e != cudaSuccess || (!a.dgamma && !a.dbeta)) return e;
  return launch_following(k_layer_norm_params, dim3((unsigned)((a.d + 31) / 32), 2), THREADS, 0, s, a, parts);
}

template <typename T>
int vector_for(const LayerNormArgs& a) {
  constexpr int most = 16 / (int)sizeof(T);
  int v = std::min(vector_of(most, a.x, a.x_stride, a.d, sizeof(T)),
                   vector_of(most, a.y, a.y_stride, a.d, sizeof(T)));
  return a.dy ? std::min(v, vector_of(most, a.dy, a.dy_stride, a.d, sizeof(T))) : v;
}

template <typename T>
cudaError_t norm_type(const LayerNormArgs& a, int num_sms, cudaStream_t s) {
  const int v = vector_for<T>(a);
  if constexpr (sizeof(T) == 2)
    if (v == 8) return norm_as<T, 8>(a, num_sms, s);
  if (v == 4) return norm_as<T, 4>(a, num_sms, s);
  if (v == 2) return norm_as<T, 2>(a, num_sms, s);
  return norm_as<T, 1>(a, num_sms, s);
}

template <typename T>
cudaError_t grad_type(const LayerNormArgs& a, int num_sms, cudaStream_t s) {
  const int v = vector_for<T>(a);
  if constexpr (sizeof(T) == 2)
    if (v == 8) return grad_as<T, 8>(a, num_sms, s);
  if (v == 4) return grad_as<T, 4>(a, num_sms, s);
  if (v == 2) return grad_as<T, 2>(a, num_sms, s);
  return grad_as<T, 1>(a, num_sms, s);
}

}  // namespace

cudaError_t launch_layer_norm(const LayerNormArgs& a, int32_t type, int num_sms, cudaStream_t s) {
  if (type == GBA_F32) return norm_type<float>(a, num_sms, s);
  if (type == GBA_BF16) return norm_type<bf16>(a, num_sms, s);
  return norm_type<f16>(a, num_sms, s);
}

size_t layer_norm_grad_workspace(const LayerNormArgs& a, int num_sms) {
  const int lg = lg_of(a.d);
  int64_t parts = std::min(a.n, WIDE_SPLIT);
  if (lg <= MOST_LG_GRAD) {
    const Shape sh = shape_of(a.n, lg, num_sms, GRAD_THREADS_PER_SM);
    parts = (int64_t)sh.grid * (sh.threads >> lg);
  }
  return (size_t)parts * 2 * (size_t)a.d * sizeof(float);
}

cudaError_t launch_layer_norm_grad(const LayerNormArgs& a, int32_t type, int num_sms,
                                   cudaStream_t s) {
  if (type == GBA_F32) return grad_type<float>(a, num_sms, s);
  if (type == GBA_BF16) return grad_type<bf16>(a, num_sms, s);
  return grad_type<f16>(a, num_sms, s);
}

}  // namespace gba

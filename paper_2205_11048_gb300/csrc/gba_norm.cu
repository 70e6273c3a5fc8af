// The global norm of many gradient tensors, and clipping by it:
//   N = sqrt(sum of g^2 over all of them),  out = min(1, M / (N + 1e-6)) * g.
//
// Bound by HBM bandwidth, or by the launches when the tensors are small.  The first kernel
// sums the squares, the second scales.  Both cut the tensors into the same pieces; the
// scaling takes them from the last to the first, so that it starts with what the norm left
// in L2.
//
// The squares of 16 or 32 elements are added in float32, the sums of those in double.
// Where such a sum leaves the range in which float32 squares are exact to their last bits,
// its elements are squared in double instead: the norm is right over all of float32.
// Blocks take pieces in a fixed order and the last block to finish adds the blocks' sums
// in order: the same tensors give the same bits.
//
// Measured: the norm of 89M float32 in 82 tensors 58 us (6.1 TB/s), of 64M bf16 in 148 30 us
// (4.3 TB/s: a piece of 16 KB is one round of loads); scaling those into float32 65 us (384 MB,
// 5.9 TB/s, the reads partly from L2).  A message of 306,496 float32: 6.4 and 9.2 us, launches.
#include <algorithm>

#include "gba_worker.cuh"

namespace gba {

namespace {

constexpr int THREADS = 256;
constexpr int NORM_BLOCKS = 5, CLIP_BLOCKS = 4;  // that an SM holds
constexpr int MOST_V = 8;  // elements of a vector of 16 bytes, at most

struct Part {
  const void* grad;
  void* out;
  int64_t n;
  uint32_t first;  // its first piece
  int16_t type, out_type;
};

template <int CAP>
struct PartList {
  int32_t count;
  int32_t unit;     // elements per piece
  uint32_t pieces;
  Part part[CAP];
};

struct NormOut {
  double* sums;      // of the blocks, those of earlier launches first
  uint32_t first;    // of this launch
  uint32_t last;     // this launch is the last: its last block forms the norm
  uint32_t* ticket;  // zero, and zero again afterwards
  float* norm;       // may be null
  float* coef;
  float max_norm;
};

template <int CAP>
__device__ __forceinline__ int part_of(const PartList<CAP>& l, uint32_t piece) {
  int lo = 0, hi = l.count;
  while (hi - lo > 1) {
    const int mid = (lo + hi) >> 1;
    if (l.part[mid].first <= piece)
      lo = mid;
    else
      hi = mid;
  }
  return lo;
}

// A part's elements: `head` single ones up to the first 16-byte boundary, `vecs` vectors of
// V, and the rest.
template <typename T>
struct Layout {
  static constexpr int V = 16 / (int)sizeof(T);
  int64_t head, vecs;
  __device__ __forceinline__ Layout(const Part& p) {
    const uint32_t off = (uint32_t)((uintptr_t)p.grad & 15u);
    head = off ? (16u - off) / (uint32_t)sizeof(T) : 0u;
    if (head > p.n) head = p.n;
    vecs = (p.n - head) / V;
  }
  // The single elements, numbered from 0: those of the head, then those of the tail.
  __device__ __forceinline__ int singles(int64_t n) const { return (int)(n - vecs * V); }
  __device__ __forceinline__ int64_t single(int i) const { return i < head ? i : vecs * V + i; }
};

// Adds the squares of x to sum.
template <int N>
__device__ __forceinline__ void add_squares(double& sum, const float (&x)[N]) {
  float q = 0.f;
#pragma unroll
  for (int i = 0; i < N; ++i) q = fmaf(x[i], x[i], q);
  if (q < 0x1p120f && q > 0x1p-80f) {
    sum += (double)q;
  } else {  // zeros, or squares that leave float32's range, or an infinity or NaN
    bool any = false;
#pragma unroll
    for (int i = 0; i < N; ++i) any = any || x[i] != 0.f;
    if (any)
#pragma unroll
      for (int i = 0; i < N; ++i) sum += (double)x[i] * (double)x[i];
  }
}

template <typename T>
__device__ __forceinline__ void piece_squares(const Part& p, uint32_t k, int unit, double& sum) {
  constexpr int V = Layout<T>::V, U = 4;
  const Layout<T> lay(p);
  const T* g = static_cast<const T*>(p.grad);
  const T* gv = g + lay.head;
  const int64_t per = unit / V, lo = (int64_t)k * per;
  const int64_t hi = lo + per < lay.vecs ? lo + per : lay.vecs;
  int64_t i = lo + threadIdx.x;
  for (; i + (U - 1) * THREADS < hi; i += U * THREADS) {
    Pack<T, V> w[U];
#pragma unroll
    for (int u = 0; u < U; ++u) w[u].load(gv + (i + u * THREADS) * V);
    float x[U * V];
#pragma unroll
    for (int u = 0; u < U; ++u) {
      float y[V];
      w[u].get(y);
#pragma unroll
      for (int j = 0; j < V; ++j) x[u * V + j] = y[j];
    }
    add_squares(sum, x);
  }
  for (; i < hi; i += THREADS) {
    Pack<T, V> w;
    float x[V];
    w.load(gv + i * V);
    w.get(x);
    add_squares(sum, x);
  }
  if (k == 0 && (int)threadIdx.x < lay.singles(p.n)) {
    const float x[1] = {to_float(g[lay.single(threadIdx.x)])};
    add_squares(sum, x);
  }
}

// The block's sum, in every thread of warp 0.
__device__ __forceinline__ double block_sum(double x) {
  __shared__ double s[THREADS / 32];
#pragma unroll
  for (int o = 16; o > 0; o >>= 1) x += __shfl_xor_sync(0xffffffffu, x, o);
  __syncthreads();
  if ((threadIdx.x & 31) == 0) s[threadIdx.x >> 5] = x;
  __syncthreads();
  double y = 0.0;
  if (threadIdx.x < 32)
#pragma unroll
    for (int w = 0; w < THREADS / 32; ++w) y += s[w];
  return y;
}

template <int CAP>
__global__ void __launch_bounds__(THREADS, NORM_BLOCKS)
    k_grad_norm(const __grid_constant__ PartList<CAP> l, NormOut o) {
  __shared__ bool s_last;
  follow();
  double sum = 0.0;
  for (uint32_t c = blockIdx.x; c < l.pieces; c += gridDim.x) {
    const Part& p = l.part[part_of(l, c)];
    const uint32_t k = c - p.first;
    if (p.type == GBA_F32)
      piece_squares<float>(p, k, l.unit, sum);
    else if (p.type == GBA_BF16)
      piece_squares<bf16>(p, k, l.unit, sum);
    else
      piece_squares<f16>(p, k, l.unit, sum);
  }
  sum = block_sum(sum);
  if (threadIdx.x == 0) {
    o.sums[o.first + blockIdx.x] = sum;
    __threadfence();
    s_last = o.last && atomicAdd(o.ticket, 1u) + 1u == gridDim.x;
  }
  __syncthreads();
  if (!s_last) return;
  __threadfence();
  const uint32_t n = o.first + gridDim.x;
  sum = 0.0;
  for (uint32_t i = threadIdx.x; i < n; i += THREADS) sum += *(const volatile double*)(o.sums + i);
  sum = block_sum(sum);
  if (threadIdx.x == 0) {
    const double norm = sqrt(sum);
    const double c = (double)o.max_norm / (norm + 1e-6);
    if (o.norm) *o.norm = (float)norm;
    *o.coef = c > 1.0 ? 1.f : (float)c;
    *o.ticket = 0u;
  }
}

// A warp's vectors leave in the order of the outputs.  Where an output does not start on the
// boundary that its vectors need (a tensor packed behind others of odd sizes), the lanes'
// values change places through shared memory, so that neighbouring lanes still store
// neighbouring elements.
template <typename T, typename TO>
__device__ __forceinline__ void clip_piece(const Part& p, uint32_t k, int unit, float c, float* swap) {
  constexpr int V = Layout<T>::V, U = 4;
  const Layout<T> lay(p);
  const T* g = static_cast<const T*>(p.grad);
  TO* out = static_cast<TO*>(p.out);
  const T* gv = g + lay.head;
  TO* ov = out + lay.head;
  constexpr uintptr_t A = V * sizeof(TO) < 16 ? V * sizeof(TO) : 16;
  const bool aligned = (uintptr_t)ov % A == 0;
  const int64_t per = unit / V, lo = (int64_t)k * per;
  const int64_t hi = lo + per < lay.vecs ? lo + per : lay.vecs;
  const int lane = threadIdx.x & 31;
  // the warp's, the same for every type: another warp may be at a piece of another type
  float* mine = swap + (threadIdx.x >> 5) * (32 * MOST_V);
  // first: the warp's first vector, of which `count` are left
  auto scaled = [&](const Pack<T, V>& w, int64_t first, int count) {
    float x[V];
    w.get(x);
#pragma unroll
    for (int j = 0; j < V; ++j) x[j] *= c;
    if (aligned) {
      Pack<TO, V> y;
      y.set(x);
      if (lane < count) y.store(ov + (first + lane) * V);
    } else {
      __syncwarp();
#pragma unroll
      for (int j = 0; j < V; j += 4)
        *reinterpret_cast<float4*>(mine + lane * V + j) = make_float4(x[j], x[j + 1], x[j + 2], x[j + 3]);
      __syncwarp();
#pragma unroll
      for (int j = 0; j < V; ++j) {
        const int e = j * 32 + lane;
        if (e < count * V) ov[first * V + e] = from_float<TO>(mine[e]);
      }
    }
  };
  int64_t first = lo + (threadIdx.x & ~31u);  // a warp's lanes go round together
  for (; first + (U - 1) * THREADS + 32 <= hi; first += U * THREADS) {
    Pack<T, V> w[U];
#pragma unroll
    for (int u = 0; u < U; ++u) w[u].load(gv + (first + u * THREADS + lane) * V);
#pragma unroll
    for (int u = 0; u < U; ++u) scaled(w[u], first + u * THREADS, 32);
  }
  for (; first < hi; first += THREADS) {
    const int count = hi - first < 32 ? (int)(hi - first) : 32;
    Pack<T, V> w{};
    if (lane < count) w.load(gv + (first + lane) * V);
    scaled(w, first, count);
  }
  if (k == 0 && (int)threadIdx.x < lay.singles(p.n)) {
    const int64_t e = lay.single(threadIdx.x);
    out[e] = from_float<TO>(to_float(g[e]) * c);
  }
}

template <typename T>
__device__ __forceinline__ void clip_out(const Part& p, uint32_t k, int unit, float c, float* swap) {
  if (p.out_type == GBA_F32)
    clip_piece<T, float>(p, k, unit, c, swap);
  else if (p.out_type == GBA_BF16)
    clip_piece<T, bf16>(p, k, unit, c, swap);
  else
    clip_piece<T, f16>(p, k, unit, c, swap);
}

template <int CAP>
__global__ void __launch_bounds__(THREADS, CLIP_BLOCKS)
    k_grad_clip(const __grid_constant__ PartList<CAP> l, const float* coef) {
  __shared__ __align__(16) float swap[THREADS * MOST_V];
  follow();
  const float c = *(const volatile float*)coef;
  for (uint32_t b = blockIdx.x; b < l.pieces; b += gridDim.x) {
    const uint32_t piece = l.pieces - 1u - b;
    const Part& p = l.part[part_of(l, piece)];
    if (p.out == p.grad && c == 1.f) continue;
    const uint32_t k = piece - p.first;
    if (p.type == GBA_F32)
      clip_out<float>(p, k, l.unit, c, swap);
    else if (p.type == GBA_BF16)
      clip_out<bf16>(p, k, l.unit, c, swap);
    else
      clip_out<f16>(p, k, l.unit, c, swap);
  }
}

// The list's kernels take up to CAP parts as a parameter; longer lists take several launches.
constexpr int CAP_MOST = 960;
static_assert(sizeof(PartList<CAP_MOST>) + sizeof(NormOut) <= 32764, "the limit of a kernel's parameters");

template <int CAP>
PartList<CAP> list_of(const gba_grad_part* parts, int32_t count, int unit) {
  PartList<CAP> l;
  l.count = 0;
  l.unit = unit;
  uint64_t pieces = 0;
  for (int32_t i = 0; i < count; ++i) {
    const gba_grad_part& p = parts[i];
    if (p.n == 0) continue;
    l.part[l.count++] = Part{p.grad, p.out, p.n, (uint32_t)pieces, (int16_t)p.type, (int16_t)p.out_type};
    pieces += (uint64_t)std::max<int64_t>(1, (p.n + unit - 1) / unit);
  }
  l.pieces = (uint32_t)pieces;
  return l;
}

template <int CAP>
cudaError_t run_as(const gba_grad_part* parts, int32_t n_parts, bool clip, int unit, NormOut o,
                   int num_sms, cudaStream_t s) {
  o.first = 0;
  for (int32_t at = 0; at == 0 || at < n_parts; at += CAP) {
    const int32_t count = std::min(CAP, n_parts - at);
    const PartList<CAP> l = list_of<CAP>(parts + at, count, unit);
    const unsigned grid = std::min(std::max(l.pieces, 1u), (unsigned)(num_sms * NORM_BLOCKS));
    o.last = at + CAP >= n_parts;
    const cudaError_t e = launch_following(k_grad_norm<CAP>, dim3(grid), THREADS, 0, s, l, o);
    if (e != cudaSuccess) return e;
    o.first += grid;
  }
  if (!clip) return cudaSuccess;
  for (int32_t at = (n_parts - 1) / CAP * CAP; at >= 0 && n_parts > 0; at -= CAP) {
    const PartList<CAP> l = list_of<CAP>(parts + at, std::min(CAP, n_parts - at), unit);
    if (l.pieces == 0) continue;
    const unsigned grid = std::min(l.pieces, (unsigned)(num_sms * CLIP_BLOCKS));
    const cudaError_t e = launch_following(k_grad_clip<CAP>, dim3(grid), THREADS, 0, s, l, (const float*)o.coef);
    if (e != cudaSuccess) return e;
  }
  return cudaSuccess;
}

}  // namespace

constexpr int MOST_UNIT = 8192;

size_t norm_workspace(int64_t n_parts, int num_sms) {
  const size_t launches = (size_t)(n_parts / CAP_MOST + 1);
  return 256 + launches * (size_t)(num_sms * NORM_BLOCKS) * sizeof(double);
}

cudaError_t launch_norm(const gba_grad_part* parts, int32_t n_parts, bool clip, float max_norm,
                        float* norm, char* ws, uint32_t* ticket, int num_sms, cudaStream_t s) {
  // pieces that give every block several, of 2,048 to 8,192 elements
  uint64_t total = 0;
  for (int32_t i = 0; i < n_parts; ++i) total += (uint64_t)parts[i].n;
  int unit = 2048;
  while (unit < MOST_UNIT && total / (uint64_t)unit > (uint64_t)num_sms * 16) unit *= 2;
  // and no more of them than 2^31
  const uint64_t most = (total / (uint64_t)unit) + (uint64_t)n_parts;
  if (most >= (1ull << 31)) return cudaErrorInvalidValue;
  NormOut o{};
  o.sums = reinterpret_cast<double*>(ws + 256);
  o.ticket = ticket;
  o.norm = norm;
  o.coef = reinterpret_cast<float*>(ws);
  o.max_norm = max_norm;
  if (n_parts <= 16) return run_as<16>(parts, n_parts, clip, unit, o, num_sms, s);
  if (n_parts <= 240) return run_as<240>(parts, n_parts, clip, unit, o, num_sms, s);
  return run_as<CAP_MOST>(parts, n_parts, clip, unit, o, num_sms, s);
}

}  // namespace gba

// One step of AdamW over many tensors:
//   g = c grad,  m = b1 m + (1 - b1) g,  v = b2 v + (1 - b2) g^2,
//   w = (1 - lr wd) w - lr / (1 - b1^t) m / (sqrt(v) / sqrt(1 - b2^t) + eps),
// with c = min(1, max_norm / (norm + 1e-6)), and the reading of its 8-bit states.
//
// Bound by HBM bandwidth: each element's weight, gradient and states are read once and written
// once.  A warp takes blocks of 256 elements, eight a lane, because 8-bit states share their
// scales over 256.  The moments are formed by one IEEE operation after another (no fused
// multiply-add), so that which code a moment is rounded to follows from its formula; the weight
// is rounded once.
// 64 10^6 float32 weights in 148 tensors with bf16 gradients and copies: 315 us, 5.70 TB/s; with 8-bit
// states 179 us, 5.74 TB/s, and 147 us for reading them as float32 (4.4 TB/s: 128 MB in, 512 MB out).
// States rounded by chance: 244 us (in 64 tensors 239, against 176 to the nearest), for a counter's hash an
// element: 107 instructions an element in place of 67 bound it then.
// 306,496 weights: 6 us, a launch.  Four blocks an SM: three took 323 us,
// five 312 and, in 8 bits, 198.
#include <cuda_fp8.h>

#include <algorithm>

#include "gba_worker.cuh"

namespace gba {

namespace {

constexpr int THREADS = 256;
constexpr int BLOCK = 256;  // elements that share the scales of 8-bit states
constexpr int V = 8;        // elements of a lane
constexpr int BLOCKS = 4;   // of an SM
static_assert(BLOCK == 32 * V, "a warp holds the elements that share a scale");

struct Part {
  void* w;
  const void* grad;
  void* m;
  void* v;
  float* m_scale;
  float* v_scale;
  void* copy;
  int64_t n;
  uint32_t first;  // its first piece
  float decay;
  int8_t type, grad_type, copy_type, vec;  // vec: every array lies on 16-byte boundaries
  uint32_t number;  // its place in the caller's list
};

template <int CAP>
struct PartList {
  int32_t count;
  uint32_t pieces;
  Part part[CAP];
};

// The part that a piece belongs to, from that of an earlier one on: a block's pieces ascend, so all of
// them together pass each part once.
template <typename L>
__device__ __forceinline__ void advance(const L& l, uint32_t piece, int& i) {
  while (i + 1 < l.count && l.part[i + 1].first <= piece) ++i;
}

// Eight elements of a type known at run time, as they lie in memory; `n` of them exist, at
// `step` elements from one another (1 where they are read as vectors).
struct Raw {
  uint4 w[2];
};
__device__ __forceinline__ Raw load_raw(const void* p, int type, int64_t i) {
  Raw r;
  if (type == GBA_F32) {
    r.w[0] = reinterpret_cast<const uint4*>(static_cast<const float*>(p) + i)[0];
    r.w[1] = reinterpret_cast<const uint4*>(static_cast<const float*>(p) + i)[1];
  } else {
    r.w[0] = reinterpret_cast<const uint4*>(static_cast<const uint16_t*>(p) + i)[0];
  }
  return r;
}
__device__ __forceinline__ void get_raw(const Raw& r, int type, float (&x)[V]) {
  if (type == GBA_F32) {
    Pack<float, V> k;
    k.w[0] = r.w[0], k.w[1] = r.w[1];
    k.get(x);
  } else if (type == GBA_BF16) {
    Pack<bf16, V> k;
    k.w[0] = r.w[0];
    k.get(x);
  } else {
    Pack<f16, V> k;
    k.w[0] = r.w[0];
    k.get(x);
  }
}
__device__ __forceinline__ void store_as(void* p, int type, int64_t i, const float (&x)[V]) {
  if (type == GBA_F32) {
    Pack<float, V> k;
    k.set(x);
    k.store(static_cast<float*>(p) + i);
  } else if (type == GBA_BF16) {
    Pack<bf16, V> k;
    k.set(x);
    k.store(static_cast<bf16*>(p) + i);
  } else {
    Pack<f16, V> k;
    k.set(x);
    k.store(static_cast<f16*>(p) + i);
  }
}
__device__ __forceinline__ float load_one(const void* p, int type, int64_t i) {
  if (type == GBA_F32) return static_cast<const float*>(p)[i];
  return type == GBA_BF16 ? to_float(static_cast<const bf16*>(p)[i]) : to_float(static_cast<const f16*>(p)[i]);
}
__device__ __forceinline__ void store_one(void* p, int type, int64_t i, float x) {
  if (type == GBA_F32)
    static_cast<float*>(p)[i] = x;
  else if (type == GBA_BF16)
    static_cast<bf16*>(p)[i] = from_float<bf16>(x);
  else
    static_cast<f16*>(p)[i] = from_float<f16>(x);
}

// ---- states in 8 bits -------------------------------------------------------------------
// The first moment: e4m3, the largest of a block as 448.  The second: 5 exponent and 3 mantissa
// bits, no sign; code c > 0 has the bits (c + 768) << 20 of a float32, 255 is 1.875, the largest
// of a block.  A block's largest counts as at least 2^-100, so that no scale is 0.
__device__ __forceinline__ float m_of(uint32_t code) {
  return __half2float(__half(__nv_cvt_fp8_to_halfraw((__nv_fp8_storage_t)code, __NV_E4M3)));
}
__device__ __forceinline__ float v_of(uint32_t code) { return code ? __uint_as_float((code + 768u) << 20) : 0.f; }
// Eight codes at once.
__device__ __forceinline__ void m_of_8(uint2 c, float (&m)[V]) {
  const uint32_t w[2] = {c.x, c.y};
#pragma unroll
  for (int j = 0; j < V; j += 2) {
    const __half2_raw h = __nv_cvt_fp8x2_to_halfraw2((__nv_fp8x2_storage_t)(w[j / 4] >> (j % 4 * 8) & 0xFFFFu), __NV_E4M3);
    const float2 f = __half22float2(__half2(h));
    m[j] = f.x, m[j + 1] = f.y;
  }
}
__device__ __forceinline__ void v_of_8(uint2 c, float (&v)[V]) {
  const uint32_t w[2] = {c.x, c.y};
#pragma unroll
  for (int j = 0; j < V; ++j) v[j] = v_of(w[j / 4] >> (j % 4 * 8) & 255u);
}
__device__ __forceinline__ uint2 m_codes(const float (&q)[V]) {
  uint32_t w[4];
#pragma unroll
  for (int j = 0; j < V; j += 2)
    w[j / 2] = __nv_cvt_float2_to_fp8x2(make_float2(q[j], q[j + 1]), __NV_SATFINITE, __NV_E4M3);
  return make_uint2(w[0] | w[1] << 16, w[2] | w[3] << 16);
}
__device__ __forceinline__ uint32_t m_code(float q) { return __nv_cvt_float_to_fp8(q, __NV_SATFINITE, __NV_E4M3); }
__device__ __forceinline__ uint32_t v_code(float q) {
  const uint32_t b = __float_as_uint(q);
  const int c = (int)((b + 0x7FFFFu + ((b >> 20) & 1u)) >> 20) - 768;
  return q > 0.f ? (uint32_t)min(max(c, 1), 255) : 0u;
}
// To one of the two codes next to a value, up or down, so that it is the value on average: a code's step is
// added `by` 2^20ths and what is left over is cut off.  Below 2^-6 the steps of m are 2^-9; what is above its
// largest value, infinite or no number is left to m_code.
__device__ __forceinline__ float m_cut(float q, uint32_t by) {
  const float a = fabsf(q);
  float x = a;
  if (a < 0x1p-6f)
    x = floorf(fmaf((float)by, 0x1p-20f, a * 512.f)) * 0x1p-9f;
  else if (a <= 448.f)
    x = __uint_as_float((__float_as_uint(a) + by) & ~0xFFFFFu);
  return copysignf(x, q);
}
__device__ __forceinline__ uint32_t v_code_cut(float q, uint32_t by) {
  const int c = (int)((__float_as_uint(q) + by) >> 20) - 768;
  return q > 0.f ? (uint32_t)min(max(c, 1), 255) : 0u;
}
__device__ __forceinline__ float block_scale(float most, float share) {
#pragma unroll
  for (int o = 16; o > 0; o >>= 1) most = fmaxf(most, __shfl_xor_sync(0xffffffffu, most, o));
  return __fmul_rn(fmaxf(most, 0x1p-100f), share);
}

struct Step {
  float c, size, root, eps, lr;
  float beta1, rest1, beta2, rest2;
  uint64_t key;  // of this step's chances
};

// The chances of element i of a part, 20 bits for m and for v: by counters, so a call has no state of its own.
__device__ __forceinline__ void chances(const Step& h, const Part& p, int64_t i, uint32_t& m, uint32_t& v) {
  const uint64_t r = splitmix64(h.key ^ ((uint64_t)p.number << 40 | (uint64_t)i));
  m = (uint32_t)r & 0xFFFFFu;
  v = (uint32_t)(r >> 44);
}

__device__ __forceinline__ void moments(const Step& h, float g, float& m, float& v) {
  g = __fmul_rn(g, h.c);
  m = __fadd_rn(__fmul_rn(m, h.beta1), __fmul_rn(g, h.rest1));
  v = __fadd_rn(__fmul_rn(v, h.beta2), __fmul_rn(__fmul_rn(g, g), h.rest2));
}
// The root and the quotient by the hardware's approximations (2^-23 and 2^-22 of themselves, with a
// denominator of at least eps, which is a normal number): what the moments round to does not depend on
// them.  A v below the normal numbers has its root, because eps may be smaller than that.
__device__ __forceinline__ float moved(const Step& h, float keep, float w, float m, float v) {
  float root;
  asm("sqrt.approx.f32 %0, %1;" : "=f"(root) : "f"(v));
  return fmaf(keep, w, -h.size * __fdividef(m, fmaf(root, h.root, h.eps)));
}

// A warp's block of 256 elements from `at` on, all of them there and in vectors.
template <int BITS, bool CHANCE>
__device__ __forceinline__ void whole_block(const Part& p, const Step& h, int64_t at) {
  const int lane = threadIdx.x & 31;
  const int64_t i = at + lane * V;
  const Raw rw = load_raw(p.w, p.type, i), rg = load_raw(p.grad, p.grad_type, i);
  float w[V], g[V], m[V], v[V];
  float ms = 0.f, vs = 0.f;
  if constexpr (BITS == 32) {
    Pack<float, V> km, kv;
    km.load(static_cast<const float*>(p.m) + i);
    kv.load(static_cast<const float*>(p.v) + i);
    km.get(m);
    kv.get(v);
  } else {
    const uint2 cm = *reinterpret_cast<const uint2*>(static_cast<const uint8_t*>(p.m) + i);
    const uint2 cv = *reinterpret_cast<const uint2*>(static_cast<const uint8_t*>(p.v) + i);
    ms = p.m_scale[at / BLOCK];
    vs = p.v_scale[at / BLOCK];
    m_of_8(cm, m);
    v_of_8(cv, v);
#pragma unroll
    for (int j = 0; j < V; ++j) m[j] = __fmul_rn(m[j], ms), v[j] = __fmul_rn(v[j], vs);
  }
  get_raw(rw, p.type, w);
  get_raw(rg, p.grad_type, g);
  const float keep = fmaf(-h.lr, p.decay, 1.f);
#pragma unroll
  for (int j = 0; j < V; ++j) {
    moments(h, g[j], m[j], v[j]);
    w[j] = moved(h, keep, w[j], m[j], v[j]);
  }
  store_as(p.w, p.type, i, w);
  if (p.copy) store_as(p.copy, p.copy_type, i, w);
  if constexpr (BITS == 32) {
    store_as(p.m, GBA_F32, i, m);
    store_as(p.v, GBA_F32, i, v);
  } else {
    float mm = 0.f, mv = 0.f;
#pragma unroll
    for (int j = 0; j < V; ++j) mm = fmaxf(mm, fabsf(m[j])), mv = fmaxf(mv, v[j]);
    ms = block_scale(mm, (float)(1.0 / 448.0));
    vs = block_scale(mv, (float)(1.0 / 1.875));
    const float mi = __frcp_rn(ms), vi = __frcp_rn(vs);
    uint32_t cv[2] = {0u, 0u};
#pragma unroll
    for (int j = 0; j < V; ++j) {
      m[j] = __fmul_rn(m[j], mi);
      v[j] = __fmul_rn(v[j], vi);
      uint32_t c;
      if constexpr (CHANCE) {
        uint32_t bm, bv;
        chances(h, p, i + j, bm, bv);
        m[j] = m_cut(m[j], bm);
        c = v_code_cut(v[j], bv);
      } else {
        c = v_code(v[j]);
      }
      cv[j / 4] |= c << (j % 4 * 8);
    }
    *reinterpret_cast<uint2*>(static_cast<uint8_t*>(p.m) + i) = m_codes(m);
    *reinterpret_cast<uint2*>(static_cast<uint8_t*>(p.v) + i) = make_uint2(cv[0], cv[1]);
    if (lane == 0) p.m_scale[at / BLOCK] = ms, p.v_scale[at / BLOCK] = vs;
  }
}

// The same of a part's last elements, and of parts that lie anywhere: element by element,
// neighbouring lanes at neighbouring ones.
template <int BITS, bool CHANCE>
__device__ __forceinline__ void loose_block(const Part& p, const Step& h, int64_t at) {
  const int lane = threadIdx.x & 31;
  const float keep = fmaf(-h.lr, p.decay, 1.f);
  float m[V], v[V];
  float ms = 0.f, vs = 0.f, mm = 0.f, mv = 0.f;
  if constexpr (BITS == 8) ms = p.m_scale[at / BLOCK], vs = p.v_scale[at / BLOCK];
#pragma unroll
  for (int j = 0; j < V; ++j) {
    const int64_t i = at + j * 32 + lane;
    m[j] = v[j] = 0.f;
    if (i < p.n) {
      if constexpr (BITS == 32) {
        m[j] = static_cast<const float*>(p.m)[i];
        v[j] = static_cast<const float*>(p.v)[i];
      } else {
        m[j] = __fmul_rn(m_of(static_cast<const uint8_t*>(p.m)[i]), ms);
        v[j] = __fmul_rn(v_of(static_cast<const uint8_t*>(p.v)[i]), vs);
      }
      moments(h, load_one(p.grad, p.grad_type, i), m[j], v[j]);
      const float w = moved(h, keep, load_one(p.w, p.type, i), m[j], v[j]);
      store_one(p.w, p.type, i, w);
      if (p.copy) store_one(p.copy, p.copy_type, i, w);
      mm = fmaxf(mm, fabsf(m[j])), mv = fmaxf(mv, v[j]);
    }
  }
  if constexpr (BITS == 8) {
    ms = block_scale(mm, (float)(1.0 / 448.0));
    vs = block_scale(mv, (float)(1.0 / 1.875));
    if (lane == 0) p.m_scale[at / BLOCK] = ms, p.v_scale[at / BLOCK] = vs;
  }
  const float mi = BITS == 8 ? __frcp_rn(ms) : 0.f, vi = BITS == 8 ? __frcp_rn(vs) : 0.f;
#pragma unroll
  for (int j = 0; j < V; ++j) {
    const int64_t i = at + j * 32 + lane;
    if (i < p.n) {
      if constexpr (BITS == 32) {
        static_cast<float*>(p.m)[i] = m[j];
        static_cast<float*>(p.v)[i] = v[j];
      } else {
        m[j] = __fmul_rn(m[j], mi);
        v[j] = __fmul_rn(v[j], vi);
        uint32_t bm = 0u, bv = 0u;
        if constexpr (CHANCE) {
          chances(h, p, i, bm, bv);
          m[j] = m_cut(m[j], bm);
        }
        static_cast<uint8_t*>(p.m)[i] = (uint8_t)m_code(m[j]);
        static_cast<uint8_t*>(p.v)[i] = (uint8_t)(CHANCE ? v_code_cut(v[j], bv) : v_code(v[j]));
      }
    }
  }
}

constexpr int PIECE = THREADS * V;  // elements of a block of threads

// last: the last launch of the call, whose last block counts the step
template <int CAP, int BITS, bool CHANCE>
__global__ void __launch_bounds__(THREADS, BLOCKS)
    k_adamw(const __grid_constant__ PartList<CAP> l, AdamWArgs a, bool last) {
  __shared__ Step s_step;
  __shared__ int s_skip;
  follow();
  if (threadIdx.x == 0) {
    const float norm = a.norm ? *(const volatile float*)a.norm : 0.f;
    const int64_t t = *(const volatile int64_t*)a.step + 1;
    s_skip = !isfinite(norm);
    Step h;
    h.lr = a.lr_now ? *(const volatile float*)a.lr_now : a.lr;
    h.c = a.norm ? fminf(__fdiv_rn(a.max_norm, __fadd_rn(norm, 1e-6f)), 1.f) : 1.f;
    // 1 - b^t = -expm1(t log b)
    h.size = h.lr / -expm1f((float)((double)t * a.log1));
    h.root = 1.f / sqrtf(-expm1f((float)((double)t * a.log2)));
    h.eps = a.eps;
    h.beta1 = a.beta1, h.rest1 = a.rest1, h.beta2 = a.beta2, h.rest2 = a.rest2;
    h.key = CHANCE ? splitmix64((uint64_t)t) : 0u;
    s_step = h;
  }
  __syncthreads();
  if (s_skip) return;
  const Step h = s_step;
  int i = 0;
  for (uint32_t c = blockIdx.x; c < l.pieces; c += gridDim.x) {
    advance(l, c, i);
    const Part& p = l.part[i];
    const int64_t at = (int64_t)(c - p.first) * PIECE + (threadIdx.x >> 5) * BLOCK;
    if (at >= p.n) continue;
    if (p.vec && at + BLOCK <= p.n)
      whole_block<BITS, CHANCE>(p, h, at);
    else
      loose_block<BITS, CHANCE>(p, h, at);
  }
  if (!last) return;
  __syncthreads();
  if (threadIdx.x == 0 && atomicAdd(a.ticket, 1u) + 1u == gridDim.x) {  // the others have read the step
    *a.step += 1;
    *a.ticket = 0u;
  }
}

template <int CAP>
struct ValueList {
  int32_t count;
  uint32_t pieces;
  struct {
    const void* m;
    const void* v;
    const float* m_scale;
    const float* v_scale;
    float* m_out;
    float* v_out;
    int64_t n;
    uint32_t first;
    int16_t bits, vec;  // vec: every array lies on its vectors' boundary
  } part[CAP];
};

// A thread takes V elements that follow one another; past a part's last vector, or where an array does
// not lie on its vectors' boundary, they go one by one.
template <int CAP>
__global__ void __launch_bounds__(THREADS) k_adamw_values(const __grid_constant__ ValueList<CAP> l) {
  follow();
  int part = 0;
  for (uint32_t c = blockIdx.x; c < l.pieces; c += gridDim.x) {
    advance(l, c, part);
    const auto& p = l.part[part];
    const int64_t at = (int64_t)(c - p.first) * PIECE;
    const int64_t i = at + threadIdx.x * V;
    if (p.vec && i + V <= p.n) {
      if (p.bits == 32) {
        Pack<float, V> m, v;
        m.load(static_cast<const float*>(p.m) + i);
        v.load(static_cast<const float*>(p.v) + i);
        m.store(p.m_out + i);
        v.store(p.v_out + i);
      } else {
        const uint2 cm = *reinterpret_cast<const uint2*>(static_cast<const uint8_t*>(p.m) + i);
        const uint2 cv = *reinterpret_cast<const uint2*>(static_cast<const uint8_t*>(p.v) + i);
        const float ms = p.m_scale[i / BLOCK], vs = p.v_scale[i / BLOCK];
        float m[V], v[V];
        m_of_8(cm, m);
        v_of_8(cv, v);
#pragma unroll
        for (int j = 0; j < V; ++j) m[j] = __fmul_rn(m[j], ms), v[j] = __fmul_rn(v[j], vs);
        store_as(p.m_out, GBA_F32, i, m);
        store_as(p.v_out, GBA_F32, i, v);
      }
      continue;
    }
    for (int64_t e = i; e < i + V && e < p.n; ++e) {
      if (p.bits == 32) {
        p.m_out[e] = static_cast<const float*>(p.m)[e];
        p.v_out[e] = static_cast<const float*>(p.v)[e];
      } else {
        p.m_out[e] = __fmul_rn(m_of(static_cast<const uint8_t*>(p.m)[e]), p.m_scale[e / BLOCK]);
        p.v_out[e] = __fmul_rn(v_of(static_cast<const uint8_t*>(p.v)[e]), p.v_scale[e / BLOCK]);
      }
    }
  }
}

constexpr int CAP_MOST = 384;
static_assert(sizeof(Part) == 80, "no more than an aligned one has to be");
static_assert(sizeof(PartList<CAP_MOST>) + sizeof(AdamWArgs) + 16 <= 32764, "the limit of a kernel's parameters");
static_assert(sizeof(ValueList<CAP_MOST>) <= 32764, "the limit of a kernel's parameters");

bool on(const void* q, size_t to) { return (uintptr_t)q % to == 0; }
bool aligned(const gba_adamw_part& p) {
  return on(p.weight, 16) && on(p.grad, 16) && on(p.copy, 16) && on(p.m, p.bits == 32 ? 16 : 8) &&
         on(p.v, p.bits == 32 ? 16 : 8);
}

// The parts of `bits` from parts[at] on, as many as fit; at: the first that is left.
template <int CAP>
PartList<CAP> list_of(const gba_adamw_part* parts, int32_t n_parts, int32_t bits, int32_t& at) {
  PartList<CAP> l;
  l.count = 0;
  uint64_t pieces = 0;
  for (; at < n_parts; ++at) {
    const gba_adamw_part& p = parts[at];
    if (p.n == 0 || p.bits != bits) continue;
    const uint64_t more = (uint64_t)((p.n + PIECE - 1) / PIECE);
    if (l.count == CAP || (l.count > 0 && pieces + more >= (1ull << 31))) break;
    l.part[l.count++] = Part{p.weight, p.grad, p.m, p.v, p.m_scale, p.v_scale, p.copy, p.n, (uint32_t)pieces,
                             p.weight_decay, (int8_t)p.type, (int8_t)p.grad_type, (int8_t)p.copy_type,
                             (int8_t)aligned(p), (uint32_t)at};
    pieces += more;
  }
  l.pieces = (uint32_t)pieces;
  return l;
}

bool any_left(const gba_adamw_part* parts, int32_t n_parts, int32_t bits, int32_t at) {
  for (; at < n_parts; ++at)
    if (parts[at].n > 0 && parts[at].bits == bits) return true;
  return false;
}

template <int CAP, int BITS, bool CHANCE>
cudaError_t run_as(const gba_adamw_part* parts, int32_t n_parts, const AdamWArgs& a, bool last, int num_sms,
                   cudaStream_t s) {
  int32_t at = 0;
  do {
    const PartList<CAP> l = list_of<CAP>(parts, n_parts, BITS, at);
    const unsigned grid = std::min(std::max(l.pieces, 1u), (unsigned)(num_sms * BLOCKS));
    const bool end = last && !any_left(parts, n_parts, BITS, at);
    const cudaError_t e = launch_following(k_adamw<CAP, BITS, CHANCE>, dim3(grid), THREADS, 0, s, l, a, end);
    if (e != cudaSuccess) return e;
  } while (any_left(parts, n_parts, BITS, at));
  return cudaSuccess;
}

template <int BITS, bool CHANCE>
cudaError_t run(const gba_adamw_part* parts, int32_t n_parts, const AdamWArgs& a, bool last, int num_sms,
                cudaStream_t s) {
  return n_parts <= 16 ? run_as<16, BITS, CHANCE>(parts, n_parts, a, last, num_sms, s)
                       : n_parts <= 160 ? run_as<160, BITS, CHANCE>(parts, n_parts, a, last, num_sms, s)
                                        : run_as<CAP_MOST, BITS, CHANCE>(parts, n_parts, a, last, num_sms, s);
}

template <int CAP>
cudaError_t values_as(const gba_adamw_part* parts, int32_t n_parts, float* const* m_out, float* const* v_out,
                      int num_sms, cudaStream_t s) {
  for (int32_t at = 0; at < n_parts;) {
    ValueList<CAP> l;
    l.count = 0;
    uint64_t pieces = 0;
    for (; at < n_parts && l.count < CAP; ++at) {
      const gba_adamw_part& p = parts[at];
      if (p.n == 0) continue;
      const uint64_t more = (uint64_t)((p.n + PIECE - 1) / PIECE);
      if (l.count > 0 && pieces + more >= (1ull << 31)) break;
      auto& q = l.part[l.count++];
      q.m = p.m, q.v = p.v, q.m_scale = p.m_scale, q.v_scale = p.v_scale;
      q.m_out = m_out[at], q.v_out = v_out[at], q.n = p.n, q.first = (uint32_t)pieces, q.bits = (int16_t)p.bits;
      q.vec = on(p.m, p.bits == 32 ? 16 : 8) && on(p.v, p.bits == 32 ? 16 : 8) && on(m_out[at], 16) && on(v_out[at], 16);
      pieces += more;
    }
    l.pieces = (uint32_t)pieces;
    if (l.count == 0) continue;
    const unsigned grid = std::min(l.pieces, (unsigned)(num_sms * 8));
    const cudaError_t e = launch_following(k_adamw_values<CAP>, dim3(grid), THREADS, 0, s, l);
    if (e != cudaSuccess) return e;
  }
  return cudaSuccess;
}

}  // namespace

cudaError_t launch_adamw(const gba_adamw_part* parts, int32_t n_parts, AdamWArgs a, int num_sms, cudaStream_t s) {
  const bool wide = any_left(parts, n_parts, 32, 0), narrow = any_left(parts, n_parts, 8, 0);
  if (wide || !narrow) {
    const cudaError_t e = run<32, false>(parts, n_parts, a, !narrow, num_sms, s);
    if (e != cudaSuccess) return e;
  }
  if (!narrow) return cudaSuccess;
  return a.rounding == GBA_ROUND_CHANCE ? run<8, true>(parts, n_parts, a, true, num_sms, s)
                                        : run<8, false>(parts, n_parts, a, true, num_sms, s);
}

cudaError_t launch_adamw_values(const gba_adamw_part* parts, int32_t n_parts, float* const* m_out,
                                float* const* v_out, int num_sms, cudaStream_t s) {
  return n_parts <= 160 ? values_as<160>(parts, n_parts, m_out, v_out, num_sms, s)
                        : values_as<CAP_MOST>(parts, n_parts, m_out, v_out, num_sms, s);
}

}  // namespace gba

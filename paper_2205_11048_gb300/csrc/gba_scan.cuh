// What the gated scan (gba_scan.cu) and its gradient (gba_scan_grad.cu) share: segments, the pairs
// through which they are joined, the gates, and the copies of rows into shared memory.
#pragma once

#include <algorithm>

#include "gba_worker.cuh"

namespace gba {

constexpr int SCAN_THREADS = 128;
constexpr int V = 4;  // channels of a thread

// The mark of a row: sequence * 4 + FIRST + LAST, or where it belongs to none, below zero: minus how
// many such rows follow one another from it on.
constexpr int32_t FIRST = 1, LAST = 2;

struct ScanPlan {
  const int32_t* marks;  // of the rows; null: sequences of `each` rows
  uint64_t* words;       // a pair for each segment and channel
  int64_t rows;          // positions of a segment
  uint32_t n_segs, n_cols;
  uint32_t pad;          // channels of a row of words
  uint32_t each;
  int32_t chained;       // something may come into a segment
  int32_t steps;         // positions of a thread
  int32_t tx;            // threads along the channels
  int32_t loose;         // rows that do not lie on a vector's boundary
  int32_t num_sms;
};

// ---- elements ----------------------------------------------------------------------------
// The V channels of a thread, two to an operation.
struct Vec {
  f2 v[V / 2];
  __device__ __forceinline__ void get(float (&x)[V]) const {
#pragma unroll
    for (int j = 0; j < V; j += 2) split(v[j / 2], x[j], x[j + 1]);
  }
  __device__ __forceinline__ void set(const float (&x)[V]) {
#pragma unroll
    for (int j = 0; j < V; j += 2) v[j / 2] = pair(x[j], x[j + 1]);
  }
  __device__ __forceinline__ void fill(float x) {
#pragma unroll
    for (int j = 0; j < V / 2; ++j) v[j] = pair(x, x);
  }
};
__device__ __forceinline__ Vec operator*(const Vec& a, const Vec& b) {
  Vec r;
#pragma unroll
  for (int j = 0; j < V / 2; ++j) r.v[j] = mul2(a.v[j], b.v[j]);
  return r;
}
__device__ __forceinline__ Vec operator+(const Vec& a, const Vec& b) {
  Vec r;
#pragma unroll
  for (int j = 0; j < V / 2; ++j) r.v[j] = add2(a.v[j], b.v[j]);
  return r;
}
__device__ __forceinline__ Vec fma_v(const Vec& a, const Vec& b, const Vec& c) {
  Vec r;
#pragma unroll
  for (int j = 0; j < V / 2; ++j) r.v[j] = fma2(a.v[j], b.v[j], c.v[j]);
  return r;
}
__device__ __forceinline__ float exp2_fast(float x) {
  float y;
  asm("ex2.approx.ftz.f32 %0, %1;" : "=f"(y) : "f"(x));
  return y;
}
__device__ __forceinline__ float rcp_fast(float x) {
  float y;
  asm("rcp.approx.ftz.f32 %0, %1;" : "=f"(y) : "f"(x));
  return y;
}
__device__ __forceinline__ float max_nan(float x, float y) {
  float z;
  asm("max.NaN.f32 %0, %1, %2;" : "=f"(z) : "f"(x), "f"(y));
  return z;
}
__device__ __forceinline__ float min_nan(float x, float y) {
  float z;
  asm("min.NaN.f32 %0, %1, %2;" : "=f"(z) : "f"(x), "f"(y));
  return z;
}

constexpr float LOG2E = 1.4426950408889634f;

// The decay a of a forget gate f as a sigmoid, and 1 - a without cancellation: 1 / (1 + t) and
// t / (1 + t) with t = exp(-f); below -87 f counts as -87, where a is 1.6e-38.  exp by the
// hardware's power of two (off by 2^-22 of itself, and by the rounding of its argument and of that
// constant, 1.23 |f| U); the reciprocal by one Newton step, because a decay near one is multiplied with itself for as
// long as the memory lasts.
// What takes a constant is done one by one: the instructions for pairs take none, and registers
// for them cost more than the pairs save.
__device__ __forceinline__ void sigmoid_gates(const Vec& forget, Vec& a, Vec& rest) {
  float f[V], t[V], q[V], e[V];
  forget.get(f);
#pragma unroll
  for (int j = 0; j < V; ++j) {
    t[j] = exp2_fast(max_nan(f[j], -87.f) * -LOG2E);
    const float s = t[j] + 1.f;
    q[j] = rcp_fast(s);
    e[j] = fmaf(-s, q[j], 1.f);
  }
  Vec tv, qv, ev;
  tv.set(t), qv.set(q), ev.set(e);
  a = fma_v(qv, ev, qv);
  rest = tv * a;
}
// The same of its logarithm g = min(f, 0).  By the hardware's power of two alone, off by 2^-22 of itself, a decay near
// one forgets its memory by up to 1.6 U (U = 2^-24) more or less a row, and it and one minus it do not add up to one.
// With RESTS (tied): down to -0.69 from e = exp(g) - 1 = g / (1 - g/2 + g^2/12 - g^4/720 + g^6/30240) (the series of
// Bernoulli's numbers, of which g^8 / 1,209,600 is left out: 0.5 U).  One minus the decay is -e, within 5.2 U of itself
// (2.1 for the denominator, 2 for the hardware's reciprocal, 1 for the product), and the decay 1 + e, rounded once.
// Without: down to -1/16 exp's own series up to g^4, within 3 U of 1 - a, and rounded.
// Further down the power of two is enough: what it is off adds up to 66 U at most.
// bf16, with the power of two alone (and a polynomial of ten terms for one minus the decay) and so: 64 sequences of
// 1,024 x 2,048 untied 135 and 134 us, tied 158 and 154; one of 262,144 x 256 128 and 130, 152 and 151.  The tied form
// for both took 141 and 138 untied; RESTS asked for at run time 8 us more; single floats instead of pairs 3.
template <bool RESTS>
__device__ __forceinline__ void log_gates(const Vec& forget, Vec& a, Vec& rest) {
  constexpr float NEAR = RESTS ? -0.69f : -0.0625f;
  float f[V], e[V], g[V];
  forget.get(f);
#pragma unroll
  for (int j = 0; j < V; ++j) f[j] = min_nan(f[j], 0.f);
#pragma unroll
  for (int j = 0; j < V; j += 2) {
    const f2 x = pair(f[j], f[j + 1]);
    f2 p;
    if constexpr (RESTS) {
      const f2 s = mul2(x, x);
      p = fma2(s, pair(1.f / 30240.f, 1.f / 30240.f), pair(-1.f / 720.f, -1.f / 720.f));
      p = fma2(s, p, pair(1.f / 12.f, 1.f / 12.f));
      p = fma2(s, p, pair(1.f, 1.f));
      p = fma2(x, pair(-0.5f, -0.5f), p);
    } else {
      p = fma2(x, pair(1.f / 24.f, 1.f / 24.f), pair(1.f / 6.f, 1.f / 6.f));
      p = fma2(x, p, pair(0.5f, 0.5f));
      p = fma2(x, p, pair(1.f, 1.f));
      p = fma2(x, p, pair(1.f, 1.f));
    }
    split(p, e[j], e[j + 1]);
  }
#pragma unroll
  for (int j = 0; j < V; ++j) {
    const float far = exp2_fast(f[j] * LOG2E);
    if constexpr (RESTS) {
      e[j] = f[j] * rcp_fast(e[j]);
      g[j] = f[j] < NEAR ? far : 1.f + e[j];
      e[j] = f[j] < NEAR ? 1.f - far : -e[j];
    } else {
      g[j] = f[j] < NEAR ? far : e[j];
    }
  }
  a.set(g);
  if constexpr (RESTS) rest.set(e);
}

__device__ __forceinline__ void gates(int32_t decay, const Vec& forget, Vec& a, Vec& rest) {
  if (decay == GBA_DECAY_SIGMOID)
    sigmoid_gates(forget, a, rest);
  else
    log_gates<true>(forget, a, rest);
}

// ---- pairs -------------------------------------------------------------------------------
// A stretch of positions stands for v -> A v + h, or where an entry lies within (cut) for v -> h.
// As a word: -A (so a zero has its sign bit set), or 1 for a cut, and h.
struct Pairs {
  Vec A, h;
  bool cut;
  __device__ __forceinline__ void clear() {
    A.fill(1.f);
    h.fill(0.f);
    cut = false;
  }
  // then the stretch (a, b) that follows
  __device__ __forceinline__ void then(const Vec& a, const Vec& b, bool c) {
    if (c) {
      cut = true;
      h = b;
    } else {
      A = A * a;
      h = fma_v(a, h, b);
    }
  }
  __device__ __forceinline__ void put(uint64_t* p) const {
    float a[V], b[V];
    A.get(a), h.get(b);
#pragma unroll
    for (int j = 0; j < V; ++j)
      p[j] = (uint64_t)__float_as_uint(cut ? 1.f : -a[j]) << 32 | __float_as_uint(b[j]);
  }
  __device__ __forceinline__ void then(const uint64_t* p) {
    float a[V], b[V];
#pragma unroll
    for (int j = 0; j < V; ++j) {
      const uint64_t w = p[j];
      a[j] = -__uint_as_float((uint32_t)(w >> 32)), b[j] = __uint_as_float((uint32_t)w);
    }
    Vec av, bv;
    av.set(a), bv.set(b);
    then(av, bv, a[0] < 0.f);  // a segment's channels are cut together
  }
};

// V elements as they lie in memory.
template <typename T>
__device__ __forceinline__ Vec vec_of(const Pack<T, V>& k) {
  float x[V];
  k.get(x);
  Vec r;
  r.set(x);
  return r;
}
template <typename T>
__device__ __forceinline__ Pack<T, V> pack_of(const Vec& v) {
  float x[V];
  v.get(x);
  Pack<T, V> k;
  k.set(x);
  return k;
}

// ---- rows in shared memory ---------------------------------------------------------------
// (Pieces of 16 bytes pass L1 by: float32 32,768 x 2,048 in 151 us instead of 185.)
template <int BYTES>
__device__ __forceinline__ void copy_async(void* to, const void* from) {
  if constexpr (BYTES == 16)
    asm volatile("cp.async.cg.shared.global [%0], [%1], 16;" ::"r"(smem_addr(to)), "l"(from) : "memory");
  else
    asm volatile("cp.async.ca.shared.global [%0], [%1], %2;" ::"r"(smem_addr(to)), "l"(from), "n"(BYTES) : "memory");
}
__device__ __forceinline__ void copies_begun() { asm volatile("cp.async.commit_group;" ::: "memory"); }
template <int N>  // all but the last N groups of this thread
__device__ __forceinline__ void copies_done() {
  asm volatile("cp.async.wait_group %0;" ::"n"(N) : "memory");
}

// Where a thread stands: its channels, and its stretch of a tile's positions.  A block walks over
// the tiles of one segment of the positions and one group of channels.
template <int TX, int STEPS>
struct Spot {
  static constexpr int TY = SCAN_THREADS / TX, ROWS = TY * STEPS, COLS = TX * V;
  uint32_t seg, col;
  int tx, ty, c;  // c: the thread's first channel; the others follow it, or at TX from one another if loose
  __device__ __forceinline__ explicit Spot(const ScanPlan& plan) {
    seg = blockIdx.x / plan.n_cols;
    col = blockIdx.x - seg * plan.n_cols;
    tx = threadIdx.x % TX;
    ty = threadIdx.x / TX;
    c = (int)col * COLS + (plan.loose ? tx : tx * V);
  }
};

// Waits for the lanes that share a row; others of the warp may be elsewhere.
template <int TX>
__device__ __forceinline__ void sync_row() {
  if constexpr (TX == 32)
    __syncwarp();
  else
    __syncwarp(((1u << TX) - 1u) << (threadIdx.x & 31u & ~(unsigned)(TX - 1)));
}

__device__ __forceinline__ bool inside(int64_t row, int64_t lo, int64_t hi) { return row >= lo && row < hi; }

// V channels at STEPS positions for each thread.  LOOSE: of rows that do not lie on a vector's
// boundary a thread has channels that are TX apart, so that neighbouring lanes are still at
// neighbouring elements.
template <typename T, int TX, int STEPS, bool LOOSE, bool HALVES = LOOSE && sizeof(T) == 2>
struct Stage {
  static constexpr int B = V * (int)sizeof(T);
  T at[STEPS][SCAN_THREADS][V];
  // BACK: of the rows row, row - 1, ...; else row, row + 1, ...; those within [lo, hi)
  template <bool BACK>
  __device__ __forceinline__ void fetch(const Rows& m, const Spot<TX, STEPS>& s, int64_t row, int64_t lo, int64_t hi,
                                        int d, int64_t) {
    const int64_t step = BACK ? -m.stride : m.stride;
    const bool whole = BACK ? row < hi && row - (STEPS - 1) >= lo : row >= lo && row + STEPS <= hi;
    const T* p = static_cast<const T*>(m.p) + row * m.stride;
    if constexpr (!LOOSE) {
      if (s.c >= d) return;
      p += s.c;
      if (whole) {
#pragma unroll
        for (int i = 0; i < STEPS; ++i, p += step) copy_async<B>(at[i][threadIdx.x], p);
      } else {
#pragma unroll
        for (int i = 0; i < STEPS; ++i, p += step)
          if (inside(BACK ? row - i : row + i, lo, hi)) copy_async<B>(at[i][threadIdx.x], p);
      }
    } else {
      p += s.c;
#pragma unroll
      for (int i = 0; i < STEPS; ++i, p += step)
        if (whole || inside(BACK ? row - i : row + i, lo, hi))
#pragma unroll
          for (int k = 0; k < V; ++k)
            if (s.c + k * TX < d) copy_async<sizeof(T)>(&at[i][threadIdx.x][k], p + k * TX);
    }
  }
  __device__ __forceinline__ Vec get(int i, const Spot<TX, STEPS>&) const {
    Pack<T, V> k;
    memcpy(&k, __builtin_assume_aligned(at[i][threadIdx.x], B), B);
    return vec_of(k);
  }
};

// Rows of 16-bit elements that start at any of them: the aligned words that hold a row's share,
// with the half word that it starts at; words that are not wholly in the matrix come by halves.
template <typename T, int TX, int STEPS>
struct Stage<T, TX, STEPS, true, true> {
  static constexpr int WORDS = TX * V / 2 + 1;  // of a row's share
  uint32_t at[STEPS][SCAN_THREADS / TX][WORDS + 1];  // the last: the half word
  template <bool BACK>
  __device__ __forceinline__ void fetch(const Rows& m, const Spot<TX, STEPS>& s, int64_t row, int64_t lo, int64_t hi,
                                        int d, int64_t n) {
    const int first = s.c - s.tx, many = d - first < TX * V ? d - first : TX * V;
    if (many <= 0) return;
    const uintptr_t base = (uintptr_t)m.p, end = base + ((n - 1) * m.stride + d) * 2;
#pragma unroll
    for (int i = 0; i < STEPS; ++i) {
      const int64_t r = BACK ? row - i : row + i;
      if (!inside(r, lo, hi)) continue;
      const uintptr_t b = base + (r * m.stride + first) * 2, w = b & ~(uintptr_t)3;
      const int odd = (int)(b & 2), words = (odd + many * 2 + 3) >> 2;
      uint32_t* to = at[i][s.ty];
#pragma unroll
      for (int k = 0; k < 3; ++k) {
        const int e = k * TX + s.tx;
        if (e >= words) continue;
        const uintptr_t from = w + 4 * e;
        if (from >= base && from + 4 <= end) {
          copy_async<4>(to + e, (const void*)from);
        } else {
          uint16_t* h = reinterpret_cast<uint16_t*>(to + e);
          if (from >= base) h[0] = *(const uint16_t*)from;
          if (from + 2 >= base && from + 4 <= end) h[1] = *(const uint16_t*)(from + 2);
        }
      }
      if (s.tx == 0) to[WORDS] = odd;
    }
  }
  __device__ __forceinline__ Vec get(int i, const Spot<TX, STEPS>& s) const {
    // a row that was not fetched left anything there: whatever it is, the elements lie in the row's words
    const T* q = reinterpret_cast<const T*>(at[i][s.ty]) + (at[i][s.ty][WORDS] >> 1 & 1) + s.tx;
    T t[V];
#pragma unroll
    for (int j = 0; j < V; ++j) t[j] = q[j * TX];
    Pack<T, V> k;
    memcpy(&k, t, sizeof k);
    return vec_of(k);
  }
};

// Stores V channels of a row.
template <typename T, int TX, int STEPS, bool LOOSE>
__device__ __forceinline__ void put_row(const OutRows& m, const Spot<TX, STEPS>& s, int64_t row, int d, const Vec& x) {
  const Pack<T, V> k = pack_of<T>(x);
  T* p = static_cast<T*>(m.p) + row * m.stride + s.c;
  if constexpr (!LOOSE) {
    k.store(p);
  } else {
    T t[V];
    memcpy(t, &k, sizeof t);
#pragma unroll
    for (int j = 0; j < V; ++j)
      if (s.c + j * TX < d) p[j * TX] = t[j];
  }
}

// V values of a row of states; they need no alignment where LOOSE.
template <int TX, bool LOOSE>
__device__ __forceinline__ Vec state_row(const float* p, int64_t stride, int32_t mark, int c, int d) {
  Vec r;
  r.fill(0.f);
  if (!p) return r;
  p += (int64_t)(mark >> 2) * stride + c;
  if constexpr (LOOSE) {
    float v[V];
#pragma unroll
    for (int j = 0; j < V; ++j) v[j] = c + j * TX < d ? p[j * TX] : 0.f;
    r.set(v);
  } else {
    Pack<float, V> k;
    k.load(p);
    r = vec_of(k);
  }
  return r;
}
template <int TX, bool LOOSE>
__device__ __forceinline__ void keep_row(float* p, int64_t stride, int32_t mark, int c, int d, const Vec& x) {
  p += (int64_t)(mark >> 2) * stride + c;
  if constexpr (LOOSE) {
    float v[V];
    x.get(v);
#pragma unroll
    for (int j = 0; j < V; ++j)
      if (c + j * TX < d) p[j * TX] = v[j];
  } else {
    pack_of<float>(x).store(p);
  }
}

// ---- marks ---------------------------------------------------------------------------------
// The marks of a thread's positions, fetched with its rows.
template <int TX, int STEPS>
struct Marks {
  static_assert(STEPS <= TX, "a lane of the row for each position");
  int32_t at[SCAN_THREADS / TX][STEPS];
  template <bool BACK>
  __device__ __forceinline__ void fetch(const ScanPlan& plan, const Spot<TX, STEPS>& s, int64_t row, int64_t lo,
                                        int64_t hi) {
    if (!plan.marks || s.tx >= STEPS) return;
    const int64_t r = BACK ? row - s.tx : row + s.tx;
    if (inside(r, lo, hi)) copy_async<4>(&at[s.ty][s.tx], plan.marks + r);
  }
  // Whether one of them is more than a row within a sequence.  pos: the place of the lowest in its
  // sequence, of those that have one length.
  template <bool BACK>
  __device__ __forceinline__ bool mixed(const ScanPlan& plan, const Spot<TX, STEPS>& s, int64_t row, int64_t lo,
                                        int64_t hi, uint32_t pos) const {
    if (BACK ? row >= hi || row - (STEPS - 1) < lo : row < lo || row + STEPS > hi) return true;
    if (!plan.marks) return pos == 0 || pos + STEPS >= plan.each;
    sync_row<TX>();
    bool special = false;
#pragma unroll
    for (int i = 0; i < STEPS; ++i) {
      const int32_t m = at[s.ty][i];
      special = special || m < 0 || (m & (FIRST | LAST));
    }
    return special;
  }
  // Whether none of them belongs to a sequence, where it matters: rows that were not fetched.
  template <bool BACK>
  __device__ __forceinline__ bool none(const ScanPlan& plan, const Spot<TX, STEPS>& s, int64_t row, int64_t lo,
                                       int64_t hi) const {
    const int64_t low = BACK ? row - (STEPS - 1) : row;
    return plan.marks && inside(low, lo, hi) && at[s.ty][BACK ? STEPS - 1 : 0] <= -STEPS;
  }
  // The marks of all positions, of which those outside the segment are no rows.
  template <bool BACK>
  __device__ __forceinline__ void all(const ScanPlan& plan, const Spot<TX, STEPS>& s, int64_t row, int64_t lo,
                                      int64_t hi, int32_t (&m)[STEPS]) const {
#pragma unroll
    for (int i = 0; i < STEPS; ++i) {
      const int64_t r = BACK ? row - i : row + i;
      m[i] = inside(r, lo, hi) ? get(plan, s, i, r) : -1;
    }
  }
  // The mark of position i, whose row is in the segment.
  __device__ __forceinline__ int32_t get(const ScanPlan& plan, const Spot<TX, STEPS>& s, int i, int64_t row) const {
    if (plan.marks) return at[s.ty][i];
    const uint32_t seq = (uint32_t)row / plan.each, p = (uint32_t)row - seq * plan.each;
    return (int32_t)seq * 4 + (p == 0 ? FIRST : 0) + (p + 1 == plan.each ? LAST : 0);
  }
};

// A row's place in its sequence, of those that have one length, and the same `by` rows on or back.
__device__ __forceinline__ uint32_t place_of(const ScanPlan& plan, int64_t row) {
  return plan.marks || row < 0 ? 0u : (uint32_t)row % plan.each;
}
template <bool BACK>
__device__ __forceinline__ uint32_t moved(const ScanPlan& plan, uint32_t pos, uint32_t by) {
  if (plan.marks) return 0u;
  if (BACK) return pos >= by ? pos - by : plan.each - 1 - (by - 1 - pos) % plan.each;
  pos += by;
  return pos < plan.each ? pos : pos % plan.each;
}

// The mark of the lowest row of a stretch that is to be fetched, asked for a turn ahead.
template <int STEPS, bool BACK>
__device__ __forceinline__ int32_t coming(const ScanPlan& plan, int64_t row, int64_t lo, int64_t hi) {
  const int64_t low = BACK ? row - (STEPS - 1) : row;
  return plan.marks && inside(low, lo, hi) ? plan.marks[low] : 0;
}

// The mark of one row.
__device__ __forceinline__ int32_t mark_of(const ScanPlan& plan, int64_t row) {
  if (plan.marks) return plan.marks[row];
  const uint32_t seq = (uint32_t)row / plan.each, pos = (uint32_t)row - seq * plan.each;
  return (int32_t)seq * 4 + (pos == 0 ? FIRST : 0) + (pos + 1 == plan.each ? LAST : 0);
}

// ---- the threads' pairs ----------------------------------------------------------------------
template <int TX, int STEPS>
struct Joint {
  static constexpr int TY = SCAN_THREADS / TX, COLS = TX * V;
  __align__(16) float A[2][TY][COLS];  // of the tile at hand and the one before
  __align__(16) float h[2][TY][COLS];
  int32_t cut[2][TY];

  __device__ __forceinline__ void put(int half, const Spot<TX, STEPS>& s, const Pairs& r) {
    pack_of<float>(r.A).store(&A[half][s.ty][s.tx * V]);
    pack_of<float>(r.h).store(&h[half][s.ty][s.tx * V]);
    if (s.tx == 0) cut[half][s.ty] = r.cut;
  }
  // Joins all threads' pairs to r; mine: r as it is before the thread's own.
  __device__ __forceinline__ void then(int half, const Spot<TX, STEPS>& s, Pairs& r, Vec& mine) const {
#pragma unroll
    for (int k = 0; k < TY; ++k) {
      if (k == s.ty) mine = r.h;
      Pack<float, V> a, b;
      a.load(&A[half][k][s.tx * V]);
      b.load(&h[half][k][s.tx * V]);
      r.then(vec_of(a), vec_of(b), cut[half][k]);
    }
  }
};

// What comes into the block's segment: the segments before it joined in order, each thread's
// share of them first.  Uses half 0 of the joint; ends with a barrier.
template <int TX, int STEPS>
__device__ __forceinline__ void into_segment(Joint<TX, STEPS>& j, const ScanPlan& plan, const Spot<TX, STEPS>& s,
                                             Pairs& r) {
  constexpr int TY = SCAN_THREADS / TX;
  r.clear();
  const uint32_t share = (s.seg + TY - 1) / TY, lo = s.ty * share, hi = lo + share < s.seg ? lo + share : s.seg;
  const uint64_t* p = plan.words + (size_t)s.col * (TX * V) + s.tx * V;
#pragma unroll 4
  for (uint32_t k = lo; k < hi; ++k) r.then(p + (size_t)k * plan.pad);
  j.put(0, s, r);
  __syncthreads();
  Vec mine;
  r.clear();
  j.then(0, s, r, mine);
  r.cut = false;
  __syncthreads();
}

// at_least, at_most: the shared memory of this launch, where it is more than S, and of any of the kernel's.  The limit is
// the kernel's on the device and not the call's, so it is the same each time, whatever other threads launch.
template <typename S, typename K>
inline cudaError_t start_scan(K kernel, unsigned blocks, const ScanArgs& a, const ScanPlan& p, cudaStream_t s,
                              size_t at_least = 0, size_t at_most = 0) {
  const size_t bytes = std::max(at_least, sizeof(S)), limit = std::max(at_most, sizeof(S));
  const cudaError_t e = cudaFuncSetAttribute(kernel, cudaFuncAttributeMaxDynamicSharedMemorySize, (int)limit);
  if (e != cudaSuccess) return e;
  return launch_following(kernel, dim3(blocks), SCAN_THREADS, bytes, s, a, p);
}

constexpr int SCAN_STEPS = 8;  // positions of a thread; few where there is little work
constexpr int SCAN_FEW = 2;
constexpr int SCAN_WIDE = 4;   // backwards, of float32 rows of many sequences
constexpr int SCAN_BLOCKS = 4, GRAD_BLOCKS = 3;  // of an SM

cudaError_t start_scan_grad(const ScanArgs& a, int32_t type, int32_t out_type, const ScanPlan& p, cudaStream_t s);

}  // namespace gba

// A gated linear recurrence over sequences, h_t = a_t h_(t-1) + b_t for every channel, and its
// gradient: with S the gradient that leaves a row towards the row before it,
//   G_t = dy_t + S_(t+1),  S_t = a_t G_t,  dx = G (1 - a) or G,  da = G (h_(t-1) - x) or G h_(t-1).
// Both are one scan, of the rows in order or from the last to the first; here a position is a
// row's place in that order, an entry a row before which the scan starts anew (from a state or
// zero), an exit one after which its value is kept.
//
// Bound by HBM bandwidth: each input is read once and each output written once.  A tile is a
// stretch of positions times a group of channels.  A thread holds a few consecutive positions
// of a few channels; stretches are joined as pairs (A, h) that stand for v -> A v + h, or for
// v -> h where an entry lies within: first the threads of a tile, then the tiles of a group of
// 16, then the groups of 16 groups, then those one after another.  A tile waits for tiles
// before it only; tiles are taken by ticket, so those run or have run.  The pairs are joined
// in an order that the sizes fix, whichever tile is first: equal calls give equal bits.
#include <algorithm>

#include "gba_worker.cuh"

namespace gba {

namespace {

constexpr int THREADS = 256;
constexpr int GROUP = 16;  // tiles of a group, groups of a span

constexpr int32_t NONE = -1;  // the mark of a row that belongs to no sequence; else sequence * 4 +
constexpr int32_t FIRST = 1, LAST = 2;

struct Plan {
  uint32_t* ticket;
  uint64_t* tiles;   // a word for each tile and channel, then for each group, then for each span
  uint64_t* groups;
  uint64_t* spans;
  const int32_t* marks;  // of the rows; null: sequences of `each` rows
  int64_t wait_ns;
  uint32_t n_tiles;  // along the positions
  uint32_t n_cols;   // along the channels
  uint32_t pad;      // channels of a row of words
  uint32_t each;
  int32_t chained;   // a tile may need what comes out of the tile before
};

// ---- marks -----------------------------------------------------------------------------
// Marks every row, checks offsets and lengths, clears the words, and passes the states of empty
// sequences on.
__global__ void __launch_bounds__(THREADS)
    k_scan_marks(ScanArgs a, int32_t* marks, uint4* words, int64_t n_words, int64_t each) {
  follow();
  const int64_t id = (int64_t)blockIdx.x * THREADS + threadIdx.x, all = (int64_t)gridDim.x * THREADS;
  for (int64_t i = id; i < n_words; i += all) words[i] = make_uint4(0u, 0u, 0u, 0u);
  if (marks)
    for (int64_t t = id; t < a.n; t += all) {
      int32_t m = NONE;
      if (a.offsets) {
        int64_t lo = -1, hi = a.n_seq + 1;  // offsets[lo] <= t < offsets[hi]
        while (hi - lo > 1) {
          const int64_t mid = (lo + hi) >> 1;
          if (a.offsets[mid] <= t)
            lo = mid;
          else
            hi = mid;
        }
        if (lo >= 0 && lo < a.n_seq)
          m = (int32_t)lo * 4 + (a.offsets[lo] == t ? FIRST : 0) + (a.offsets[lo + 1] == t + 1 ? LAST : 0);
      } else {
        const int64_t seq = t / each, pos = t - seq * each, len = a.lengths[seq];
        if (pos < len) m = (int32_t)seq * 4 + (pos == 0 ? FIRST : 0) + (pos + 1 == len || pos + 1 == each ? LAST : 0);
      }
      marks[t] = m;
    }
  const int lane = threadIdx.x & 31;
  for (int64_t s = id >> 5; s < a.n_seq; s += all >> 5) {
    int64_t len = each;
    bool good = true;
    if (a.offsets) {
      const int64_t from = a.offsets[s], to = a.offsets[s + 1];
      good = from >= 0 && from <= to && to <= a.n;
      len = to - from;
    } else if (a.lengths) {
      len = a.lengths[s];
      good = len >= 0 && len <= each;
    }
    if (!good && lane == 0) raise_error(a.err, ERR_SEQUENCES);
    if (len == 0 && a.last)
      for (int c = lane; c < a.d; c += 32)
        a.last[s * a.last_stride + c] = a.state ? a.state[s * a.state_stride + c] : 0.f;
  }
}

// ---- words -------------------------------------------------------------------------------
// A pair as one word that is never 0: -A (so a zero has its sign bit set) and h; where an entry
// lies within, 1 in the place of -A.
struct Pair {
  float minus, h;
};
__device__ __forceinline__ float through(const Pair& p, float v) { return p.minus > 0.f ? p.h : fmaf(-p.minus, v, p.h); }
// First p, then q.
__device__ __forceinline__ Pair joined(const Pair& p, const Pair& q) {
  if (q.minus > 0.f) return q;
  return Pair{p.minus > 0.f ? 1.f : -(p.minus * q.minus), fmaf(-q.minus, p.h, q.h)};
}
__device__ __forceinline__ uint64_t word_of(const Pair& p) {
  return (uint64_t)__float_as_uint(p.minus) << 32 | __float_as_uint(p.h);
}
__device__ __forceinline__ Pair pair_of(uint64_t w) {
  return Pair{__uint_as_float((uint32_t)(w >> 32)), __uint_as_float((uint32_t)w)};
}

template <int V>
__device__ __forceinline__ void put_words(uint64_t* p, const uint64_t (&w)[V]) {
  if constexpr (V == 1) {
    asm volatile("st.relaxed.gpu.global.u64 [%0], %1;" ::"l"(p), "l"(w[0]) : "memory");
  } else {
#pragma unroll
    for (int j = 0; j < V; j += 2)
      asm volatile("st.relaxed.gpu.global.v2.u64 [%0], {%1, %2};" ::"l"(p + j), "l"(w[j]), "l"(w[j + 1]) : "memory");
  }
}
template <int V>
__device__ __forceinline__ bool get_words(const uint64_t* p, uint64_t (&w)[V]) {
  bool all = true;
  if constexpr (V == 1) {
    asm volatile("ld.relaxed.gpu.global.u64 %0, [%1];" : "=l"(w[0]) : "l"(p) : "memory");
    all = w[0] != 0;
  } else {
#pragma unroll
    for (int j = 0; j < V; j += 2) {
      asm volatile("ld.relaxed.gpu.global.v2.u64 {%0, %1}, [%2];" : "=l"(w[j]), "=l"(w[j + 1]) : "l"(p + j) : "memory");
      all = all && w[j] != 0 && w[j + 1] != 0;
    }
  }
  return all;
}
// Waits for the words of an earlier tile; after the limit they count as zeros.
template <int V>
__device__ __forceinline__ void wait_words(const uint64_t* p, uint64_t (&w)[V], const Plan& plan, const ErrSink& err) {
  if (get_words<V>(p, w)) return;
  const uint64_t t0 = globaltimer_ns();
  while (!get_words<V>(p, w)) {
    __nanosleep(32);
    if ((int64_t)(globaltimer_ns() - t0) > plan.wait_ns) {
      raise_error(err, ERR_TIMEOUT);
      return;
    }
  }
}

// ---- gates -------------------------------------------------------------------------------
// The decay of a forget gate, and one minus it without cancellation.
__device__ __forceinline__ float2 decay_of(int32_t kind, float f) {
  if (kind == GBA_DECAY_LOG) {
    const float g = f > 0.f ? 0.f : f;
    return make_float2(expf(g), -expm1f(g));
  }
  // 1 / (1 + t) and t / (1 + t) with t = exp(-|f|); the quotient by one Newton step, because a
  // decay near one is multiplied with itself for as long as the memory lasts
  const float t = expf(-fabsf(f)), s = 1.f + t;
  float q = __fdividef(1.f, s);
  q = fmaf(q, fmaf(-s, q, 1.f), q);
  const float r = t * q;
  return f >= 0.f ? make_float2(q, r) : make_float2(r, q);
}
__device__ __forceinline__ float log_decay(float f) { return expf(f > 0.f ? 0.f : f); }

// ---- the scan ------------------------------------------------------------------------------
template <int V, int TX, int STEPS>
struct Tile {
  static constexpr int TY = THREADS / TX, ROWS = TY * STEPS, COLS = TX * V;
  int32_t mark[ROWS];
  Pair pairs[TY][COLS];          // of the threads
  Pair before[2 * GROUP][COLS];  // of the tiles before in the group, then of the groups before in the span
  float carry[COLS];
  uint32_t at;
};

// The value that comes into each thread's stretch.  own: the thread's pairs; the tile's marks are set.
// skip: nothing comes into the tile (its first position is an entry, or belongs to no sequence).
template <int V, int TX, int STEPS>
__device__ __forceinline__ void incoming(Tile<V, TX, STEPS>& s, const Plan& plan, const ErrSink& err, uint32_t ti,
                                         uint32_t col, bool skip, const Pair (&own)[V], float (&v)[V]) {
  constexpr int TY = THREADS / TX;
  const int tx = threadIdx.x % TX, ty = threadIdx.x / TX, c0 = tx * V;
#pragma unroll
  for (int j = 0; j < V; ++j) s.pairs[ty][c0 + j] = own[j];
  __syncthreads();
  if (plan.chained) {
    const uint32_t j_in = ti % GROUP, g = ti / GROUP, g_in = g % GROUP, sp = g / GROUP;
    const size_t ch = (size_t)col * (TX * V) + c0;
    Pair tile[V];
    bool cut = false;  // an entry lies within the tile: the same for all channels
    if (ty == 0) {
#pragma unroll
      for (int j = 0; j < V; ++j) {
        tile[j] = s.pairs[0][c0 + j];
        for (int k = 1; k < TY; ++k) tile[j] = joined(tile[j], s.pairs[k][c0 + j]);
      }
      cut = tile[0].minus > 0.f;
      if (j_in + 1 < GROUP && ti + 1 < plan.n_tiles) {
        uint64_t w[V];
#pragma unroll
        for (int j = 0; j < V; ++j) w[j] = word_of(tile[j]);
        put_words<V>(plan.tiles + (size_t)ti * plan.pad + ch, w);
      }
    }
    const bool closes = j_in + 1 == GROUP && ti + 1 < plan.n_tiles;  // the last tile of its group
    const bool ends = closes && g_in + 1 == GROUP;                   // and of its span
    // the tiles before, in the group
    if (!skip || closes)
      for (int e = ty; e < (int)j_in; e += TY) {
        uint64_t w[V];
        wait_words<V>(plan.tiles + (size_t)(ti - j_in + e) * plan.pad + ch, w, plan, err);
#pragma unroll
        for (int j = 0; j < V; ++j) s.before[e][c0 + j] = pair_of(w[j]);
      }
    __syncthreads();
    Pair group[V];  // of the tiles before
    if (ty == 0 && (!skip || closes)) {
#pragma unroll
      for (int j = 0; j < V; ++j) {
        group[j] = Pair{-1.f, 0.f};
        for (int e = 0; e < (int)j_in; ++e) group[j] = joined(group[j], s.before[e][c0 + j]);
      }
      if (closes && !ends) {
        uint64_t w[V];
#pragma unroll
        for (int j = 0; j < V; ++j) w[j] = word_of(cut ? tile[j] : joined(group[j], tile[j]));
        put_words<V>(plan.groups + (size_t)g * plan.pad + ch, w);
      }
    }
    // the groups before, in the span, and what comes out of the span before
    if (!skip || ends)
      for (int e = ty; e < (int)g_in; e += TY) {
        uint64_t w[V];
        wait_words<V>(plan.groups + (size_t)(g - g_in + e) * plan.pad + ch, w, plan, err);
#pragma unroll
        for (int j = 0; j < V; ++j) s.before[GROUP + e][c0 + j] = pair_of(w[j]);
      }
    __syncthreads();
    if (ty == 0 && (!skip || ends)) {
      float in[V];
#pragma unroll
      for (int j = 0; j < V; ++j) in[j] = 0.f;
      if (sp > 0) {
        uint64_t w[V];
        wait_words<V>(plan.spans + (size_t)(sp - 1) * plan.pad + ch, w, plan, err);
#pragma unroll
        for (int j = 0; j < V; ++j) in[j] = pair_of(w[j]).h;
      }
#pragma unroll
      for (int j = 0; j < V; ++j) {
        for (int e = 0; e < (int)g_in; ++e) in[j] = through(s.before[GROUP + e][c0 + j], in[j]);
        in[j] = through(group[j], in[j]);
        s.carry[c0 + j] = in[j];
      }
      if (ends) {
        uint64_t w[V];
#pragma unroll
        for (int j = 0; j < V; ++j) w[j] = word_of(Pair{1.f, through(tile[j], in[j])});
        put_words<V>(plan.spans + (size_t)sp * plan.pad + ch, w);
      }
    }
    __syncthreads();
  }
#pragma unroll
  for (int j = 0; j < V; ++j) {
    v[j] = plan.chained && !skip ? s.carry[c0 + j] : 0.f;
    for (int k = 0; k < ty; ++k) v[j] = through(s.pairs[k][c0 + j], v[j]);
  }
}

// The block's tile and its marks.
template <int V, int TX, int STEPS>
__device__ __forceinline__ void begin(Tile<V, TX, STEPS>& s, const ScanArgs& a, const Plan& plan, bool back,
                                      uint32_t& ti, uint32_t& col) {
  constexpr int ROWS = Tile<V, TX, STEPS>::ROWS;
  uint32_t at = blockIdx.x;
  if (plan.chained) {
    if (threadIdx.x == 0) s.at = atomicAdd(plan.ticket, 1u);
    __syncthreads();
    at = s.at;
  }
  ti = at / plan.n_cols;
  col = at - ti * plan.n_cols;
  for (int i = threadIdx.x; i < ROWS; i += THREADS) {
    const int64_t p = (int64_t)ti * ROWS + i, row = back ? a.n - 1 - p : p;
    int32_t m = NONE;
    if (p < a.n) {
      if (plan.marks) {
        m = plan.marks[row];
      } else {
        const uint32_t seq = (uint32_t)row / plan.each, pos = (uint32_t)row - seq * plan.each;
        m = (int32_t)seq * 4 + (pos == 0 ? FIRST : 0) + (pos + 1 == plan.each ? LAST : 0);
      }
    }
    s.mark[i] = m;
  }
}

template <int V>
__device__ __forceinline__ void state_row(const float* p, int64_t stride, int32_t mark, int c, float (&v)[V]) {
  if (!p) {
#pragma unroll
    for (int j = 0; j < V; ++j) v[j] = 0.f;
    return;
  }
  Pack<float, V> k;
  k.load(p + (int64_t)(mark >> 2) * stride + c);
  k.get(v);
}

template <typename T, typename O, int V, int TX, int STEPS>
__global__ void __launch_bounds__(THREADS, 2) k_scan(ScanArgs a, Plan plan) {
  __shared__ Tile<V, TX, STEPS> s;
  constexpr int ROWS = Tile<V, TX, STEPS>::ROWS;
  follow();
  uint32_t ti, col;
  begin(s, a, plan, false, ti, col);
  const int tx = threadIdx.x % TX, ty = threadIdx.x / TX;
  const int c = (int)col * (TX * V) + tx * V;
  const bool in = c < a.d;
  const int64_t row0 = (int64_t)ti * ROWS + ty * STEPS;
  Pack<T, V> px[STEPS], pf[STEPS];
#pragma unroll
  for (int i = 0; i < STEPS; ++i)
    if (in && row0 + i < a.n) {
      px[i].load(static_cast<const T*>(a.x.p) + (row0 + i) * a.x.stride + c);
      pf[i].load(static_cast<const T*>(a.f.p) + (row0 + i) * a.f.stride + c);
    }
  __syncthreads();
  float A[STEPS][V], B[STEPS][V];  // h -> A h + B, or B at an entry
  Pair own[V];
#pragma unroll
  for (int j = 0; j < V; ++j) own[j] = Pair{-1.f, 0.f};
#pragma unroll
  for (int i = 0; i < STEPS; ++i) {
    const int32_t m = s.mark[ty * STEPS + i];
    float x[V], f[V];
    px[i].get(x);
    pf[i].get(f);
#pragma unroll
    for (int j = 0; j < V; ++j) {
      if (a.tied || a.decay == GBA_DECAY_SIGMOID) {
        const float2 g = decay_of(a.decay, f[j]);
        A[i][j] = g.x;
        B[i][j] = a.tied ? g.y * x[j] : x[j];
      } else {
        A[i][j] = log_decay(f[j]);
        B[i][j] = x[j];
      }
    }
    if (m == NONE || !in) {
#pragma unroll
      for (int j = 0; j < V; ++j) A[i][j] = 0.f, B[i][j] = 0.f, own[j] = Pair{1.f, 0.f};
    } else if (m & FIRST) {
      float h0[V];
      state_row<V>(a.state, a.state_stride, m, c, h0);
#pragma unroll
      for (int j = 0; j < V; ++j) {
        if (a.state) B[i][j] = fmaf(A[i][j], h0[j], B[i][j]);
        own[j] = Pair{1.f, B[i][j]};
      }
    } else {
#pragma unroll
      for (int j = 0; j < V; ++j) {
        own[j].h = fmaf(A[i][j], own[j].h, B[i][j]);
        if (own[j].minus <= 0.f || own[j].minus != own[j].minus) own[j].minus *= A[i][j];
      }
    }
  }
  float h[V];
  const int32_t m0 = s.mark[0];
  incoming<V, TX, STEPS>(s, plan, a.err, ti, col, m0 == NONE || (m0 & FIRST), own, h);
  if (!in) return;
#pragma unroll
  for (int i = 0; i < STEPS; ++i) {
    const int32_t m = s.mark[ty * STEPS + i];
    if (row0 + i >= a.n) break;
#pragma unroll
    for (int j = 0; j < V; ++j) h[j] = m == NONE || (m & FIRST) ? B[i][j] : fmaf(A[i][j], h[j], B[i][j]);
    Pack<O, V> y;
    y.set(h);
    y.store(static_cast<O*>(a.out.p) + (row0 + i) * a.out.stride + c);
    if (a.last && m != NONE && (m & LAST)) {
      Pack<float, V> k;
      k.set(h);
      k.store(a.last + (int64_t)(m >> 2) * a.last_stride + c);
    }
  }
}

template <typename T, typename O, int V, int TX, int STEPS>
__global__ void __launch_bounds__(THREADS, 2) k_scan_grad(ScanArgs a, Plan plan) {
  __shared__ Tile<V, TX, STEPS> s;
  constexpr int ROWS = Tile<V, TX, STEPS>::ROWS;
  follow();
  uint32_t ti, col;
  begin(s, a, plan, true, ti, col);
  const int tx = threadIdx.x % TX, ty = threadIdx.x / TX;
  const int c = (int)col * (TX * V) + tx * V;
  const bool in = c < a.d;
  const int64_t p0 = (int64_t)ti * ROWS + ty * STEPS, row0 = a.n - 1 - p0;
  Pack<T, V> px[STEPS], pf[STEPS];
  Pack<O, V> pd[STEPS], py[STEPS];
#pragma unroll
  for (int i = 0; i < STEPS; ++i)
    if (in && row0 - i >= 0) {
      pd[i].load(static_cast<const O*>(a.dy.p) + (row0 - i) * a.dy.stride + c);
      pf[i].load(static_cast<const T*>(a.f.p) + (row0 - i) * a.f.stride + c);
      if (a.tied) px[i].load(static_cast<const T*>(a.x.p) + (row0 - i) * a.x.stride + c);
      if (row0 - i > 0) py[i].load(static_cast<const O*>(a.y.p) + (row0 - i - 1) * a.y.stride + c);
    }
  __syncthreads();
  Pair own[V];
#pragma unroll
  for (int j = 0; j < V; ++j) own[j] = Pair{-1.f, 0.f};
#pragma unroll
  for (int i = 0; i < STEPS; ++i) {
    const int32_t m = s.mark[ty * STEPS + i];
    if (m == NONE || !in) {
#pragma unroll
      for (int j = 0; j < V; ++j) own[j] = Pair{1.f, 0.f};
      continue;
    }
    float f[V], dy[V];
    pf[i].get(f);
    pd[i].get(dy);
    float s0[V];
    if (m & LAST) state_row<V>(a.state, a.state_stride, m, c, s0);
#pragma unroll
    for (int j = 0; j < V; ++j) {
      const float g = a.decay == GBA_DECAY_LOG ? log_decay(f[j]) : decay_of(a.decay, f[j]).x;
      if (m & LAST) {
        own[j] = Pair{1.f, g * (a.state ? dy[j] + s0[j] : dy[j])};
      } else {
        own[j].h = g * (dy[j] + own[j].h);
        if (own[j].minus <= 0.f || own[j].minus != own[j].minus) own[j].minus *= g;
      }
    }
  }
  float v[V];
  const int32_t m0 = s.mark[0];
  incoming<V, TX, STEPS>(s, plan, a.err, ti, col, m0 == NONE || (m0 & LAST), own, v);
  if (!in) return;
#pragma unroll
  for (int i = 0; i < STEPS; ++i) {
    const int32_t m = s.mark[ty * STEPS + i];
    const int64_t row = row0 - i;
    if (row < 0) break;
    float dx[V], df[V];
    if (m == NONE) {
#pragma unroll
      for (int j = 0; j < V; ++j) dx[j] = df[j] = v[j] = 0.f;
    } else {
      float x[V], f[V], dy[V], h[V];
      pf[i].get(f);
      pd[i].get(dy);
      if (m & FIRST)
        state_row<V>(a.h0, a.h0_stride, m, c, h);
      else
        py[i].get(h);
      if (a.tied) px[i].get(x);
      if (m & LAST) state_row<V>(a.state, a.state_stride, m, c, v);
#pragma unroll
      for (int j = 0; j < V; ++j) {
        const float G = dy[j] + v[j];
        float2 g;
        if (a.tied || a.decay == GBA_DECAY_SIGMOID)
          g = decay_of(a.decay, f[j]);
        else
          g = make_float2(log_decay(f[j]), 0.f);
        const float da = a.tied ? G * (h[j] - x[j]) : G * h[j];
        dx[j] = a.tied ? G * g.y : G;
        df[j] = a.decay == GBA_DECAY_SIGMOID ? da * (g.x * g.y) : f[j] > 0.f ? 0.f : da * g.x;
        v[j] = g.x * G;
      }
      if (a.last && (m & FIRST)) {
        Pack<float, V> k;
        k.set(v);
        k.store(a.last + (int64_t)(m >> 2) * a.last_stride + c);
      }
    }
    Pack<T, V> o;
    o.set(dx);
    o.store(static_cast<T*>(a.out.p) + row * a.out.stride + c);
    o.set(df);
    o.store(static_cast<T*>(a.df.p) + row * a.df.stride + c);
  }
}

// ---- launches ------------------------------------------------------------------------------
struct Shape {
  int v, tx, steps;
  uint32_t rows, cols;  // of a tile
  uint32_t n_tiles, n_cols;
  int64_t each;
  bool marks, chained;
  size_t words;  // 16-byte words to clear, the ticket's first
  size_t bytes;
};

Shape shape_of(const ScanArgs& a, int32_t type, int32_t out_type, bool grad, int num_sms) {
  Shape s{};
  auto fits = [&](const void* p, int64_t stride, size_t bytes) {
    return !p || vector_of(4, p, stride, a.d, bytes) == 4;
  };
  const size_t b = type_bytes(type), ob = type_bytes(out_type);
  bool ok = fits(a.x.p, a.x.stride, b) && fits(a.f.p, a.f.stride, b) && fits(a.state, a.state_stride, 4) &&
            fits(a.last, a.last_stride, 4) && fits(a.h0, a.h0_stride, 4) &&
            fits(a.out.p, a.out.stride, grad ? b : ob);
  if (grad) ok = ok && fits(a.y.p, a.y.stride, ob) && fits(a.dy.p, a.dy.stride, ob) && fits(a.df.p, a.df.stride, b);
  s.v = ok ? 4 : 1;
  s.tx = a.d <= 16 * s.v ? 8 : 32;
  s.cols = (uint32_t)(s.tx * s.v);
  s.n_cols = (uint32_t)((a.d + s.cols - 1) / s.cols);
  s.each = a.n_seq > 0 ? a.n / a.n_seq : 0;
  s.marks = a.offsets || a.lengths;
  // a few positions a thread where there are few of them
  const int ty = THREADS / s.tx, most = grad ? 4 : 8;
  const int64_t tiles = ((a.n + ty * most - 1) / (ty * most)) * s.n_cols;
  s.steps = tiles >= num_sms ? most : 2;
  s.rows = (uint32_t)(ty * s.steps);
  s.n_tiles = (uint32_t)((a.n + s.rows - 1) / s.rows);
  s.chained = s.n_tiles > 1 && (s.marks || s.rows % s.each != 0);
  size_t words = 16;
  if (s.chained) {
    const size_t pad = (size_t)s.n_cols * s.cols, groups = (s.n_tiles + GROUP - 1) / GROUP;
    words += (s.n_tiles + groups + (groups + GROUP - 1) / GROUP) * pad * 8;
  }
  s.words = s.chained ? (words + 15) / 16 : 0;
  s.bytes = (words + 255) / 256 * 256 + (s.marks ? (size_t)a.n * 4 : 0);
  return s;
}

template <typename T, typename O, int V, int TX, int STEPS, bool GRAD>
cudaError_t start(const ScanArgs& a, const Plan& p, cudaStream_t s) {
  const dim3 grid(p.n_tiles * p.n_cols);
  if constexpr (GRAD)
    return launch_following(k_scan_grad<T, O, V, TX, STEPS>, grid, THREADS, 0, s, a, p);
  else
    return launch_following(k_scan<T, O, V, TX, STEPS>, grid, THREADS, 0, s, a, p);
}

template <typename T, typename O, bool GRAD>
cudaError_t launch_as(const ScanArgs& a, const Shape& h, const Plan& p, cudaStream_t s) {
  constexpr int MOST = GRAD ? 4 : 8;
  if (h.v == 4) {
    if (h.tx == 32)
      return h.steps == MOST ? start<T, O, 4, 32, MOST, GRAD>(a, p, s) : start<T, O, 4, 32, 2, GRAD>(a, p, s);
    return h.steps == MOST ? start<T, O, 4, 8, MOST, GRAD>(a, p, s) : start<T, O, 4, 8, 2, GRAD>(a, p, s);
  }
  if (h.tx == 32)
    return h.steps == MOST ? start<T, O, 1, 32, MOST, GRAD>(a, p, s) : start<T, O, 1, 32, 2, GRAD>(a, p, s);
  return h.steps == MOST ? start<T, O, 1, 8, MOST, GRAD>(a, p, s) : start<T, O, 1, 8, 2, GRAD>(a, p, s);
}

template <bool GRAD>
cudaError_t launch_typed(const ScanArgs& a, int32_t type, int32_t out_type, const Shape& h, const Plan& p,
                         cudaStream_t s) {
  if (type == GBA_F32) return launch_as<float, float, GRAD>(a, h, p, s);
  if (type == GBA_BF16)
    return out_type == GBA_F32 ? launch_as<bf16, float, GRAD>(a, h, p, s) : launch_as<bf16, bf16, GRAD>(a, h, p, s);
  return out_type == GBA_F32 ? launch_as<f16, float, GRAD>(a, h, p, s) : launch_as<f16, f16, GRAD>(a, h, p, s);
}

}  // namespace

size_t scan_workspace(const ScanArgs& a, int32_t type, int32_t out_type, bool grad, int num_sms) {
  return shape_of(a, type, out_type, grad, num_sms).bytes;
}

cudaError_t launch_scan(const ScanArgs& a, int32_t type, int32_t out_type, bool grad, char* ws, int64_t wait_ns,
                        int num_sms, cudaStream_t s) {
  const Shape h = shape_of(a, type, out_type, grad, num_sms);
  Plan p{};
  p.ticket = reinterpret_cast<uint32_t*>(ws);
  p.n_tiles = h.n_tiles;
  p.n_cols = h.n_cols;
  p.pad = h.n_cols * h.cols;
  p.each = (uint32_t)h.each;
  p.chained = h.chained;
  p.wait_ns = wait_ns;
  const size_t groups = (h.n_tiles + GROUP - 1) / GROUP;
  p.tiles = reinterpret_cast<uint64_t*>(ws + 16);
  p.groups = p.tiles + (size_t)h.n_tiles * p.pad;
  p.spans = p.groups + groups * p.pad;
  int32_t* marks = h.marks ? reinterpret_cast<int32_t*>(ws + h.bytes - (size_t)a.n * 4) : nullptr;
  p.marks = marks;
  if (h.marks || h.chained || a.n == 0) {
    const int64_t work = std::max<int64_t>(std::max<int64_t>((int64_t)h.words, a.n), a.n_seq * 32);
    const unsigned grid = (unsigned)std::min<int64_t>((work + THREADS - 1) / THREADS, (int64_t)num_sms * 8);
    const cudaError_t e = launch_following(k_scan_marks, dim3(std::max(1u, grid)), THREADS, 0, s, a, marks,
                                           reinterpret_cast<uint4*>(ws), (int64_t)h.words, h.each);
    if (e != cudaSuccess || a.n == 0) return e;
  }
  return grad ? launch_typed<true>(a, type, out_type, h, p, s) : launch_typed<false>(a, type, out_type, h, p, s);
}

}  // namespace gba

// The gradient of the gated scan (see gba_scan.cu), a scan from the last row to the first:
//   G_t = dy_t + S_(t+1),  S_t = a_t G_t,  dx = G (1 - a) or G,  df = G (h_(t-1) - x or 0) a (1 - a or 1).
#include "gba_scan.cuh"

namespace gba {

namespace {

constexpr int STAGES = 2;

template <typename T, typename O, int TX, int STEPS, bool LOOSE, bool TAIL>
struct Shared {
  Joint<TX, STEPS> j;
  struct {
    Stage<T, TX, STEPS, LOOSE> f;
    Stage<O, TX, STEPS, LOOSE> dy;
    Stage<T, TX, TAIL ? 1 : STEPS, LOOSE> x;  // not needed for a segment's pair
    Stage<O, TX, TAIL ? 1 : STEPS, LOOSE> y;
    Marks<TX, STEPS> marks;
  } in[STAGES];
};

// TAIL: only the pair of each segment but the last, from its last entry on.
template <typename T, typename O, int TX, int STEPS, bool LOOSE, bool TAIL>
__global__ void __launch_bounds__(SCAN_THREADS, GRAD_BLOCKS) k_scan_grad(ScanArgs a, ScanPlan plan) {
  extern __shared__ __align__(16) char smem[];
  auto& sh = *reinterpret_cast<Shared<T, O, TX, STEPS, LOOSE, TAIL>*>(smem);
  using At = Spot<TX, STEPS>;
  follow();
  const At at(plan);
  const bool in = at.c < a.d;
  // the segment's rows, from the last on
  int64_t hi = a.n - (int64_t)at.seg * plan.rows;
  const int64_t lo = hi > plan.rows ? hi - plan.rows : 0;
  Pairs run;
  run.clear();
  if constexpr (TAIL) {
    const int32_t m = mark_of(plan, lo - 1);
    if (m < 0 || (m & LAST)) return;  // nothing goes there
    if (plan.marks) {
      for (int64_t low = lo; low < hi; low += SCAN_THREADS) {
        const int64_t r = low + threadIdx.x;
        const int32_t q = r < hi ? plan.marks[r] : 0;
        if (__syncthreads_or(q < 0 || (q & LAST))) {
          hi = low + SCAN_THREADS < hi ? low + SCAN_THREADS : hi;
          break;
        }
      }
    } else {
      const int64_t behind = (lo + plan.each - 1) / plan.each * plan.each;  // of the sequence that lo is in
      if (behind < hi) hi = behind;
    }
  } else if (plan.chained && at.seg > 0) {
    const int32_t m = mark_of(plan, hi - 1);
    if (m >= 0 && !(m & LAST)) into_segment(sh.j, plan, at, run);
  }
  const int tiles = (int)((hi - lo + At::ROWS - 1) / At::ROWS);
  int64_t row = hi - 1 - at.ty * STEPS, ahead = row;
  uint32_t pos = place_of(plan, row - (STEPS - 1));
  int32_t mark = coming<STEPS, true>(plan, ahead, lo, hi);
  auto fetch = [&](int to) {
    auto& s = sh.in[to];
    if (mark > -STEPS) {  // else none of the rows belongs to a sequence
      s.f.template fetch<true>(a.f, at, ahead, lo, hi, a.d, a.n);
      s.dy.template fetch<true>(a.dy, at, ahead, lo, hi, a.d, a.n);
      if constexpr (!TAIL) {
        if (a.tied) s.x.template fetch<true>(a.x, at, ahead, lo, hi, a.d, a.n);
        s.y.template fetch<true>(a.y, at, ahead - 1, lo > 0 ? lo - 1 : 0, hi, a.d, a.n);
      }
    }
    s.marks.template fetch<true>(plan, at, ahead, lo, hi);
    ahead -= At::ROWS;
    mark = coming<STEPS, true>(plan, ahead, lo, hi);
    copies_begun();
  };
#pragma unroll
  for (int k = 0; k < STAGES; ++k) fetch(k);
  int stage = 0;
  for (int t = 0; t < tiles; ++t, row -= At::ROWS, pos = moved<true>(plan, pos, At::ROWS)) {
    copies_done<STAGES - 1>();
    sync_row<TX>();
    auto& here = sh.in[stage];
    Pairs mine;  // S -> A S + h
    mine.clear();
    Vec A[STEPS], R[STEPS];  // the decays, and what dx and df have of 1 - a
    // Rows where sequences begin or end, or that are none, go one after another, in code of few
    // instructions: unrolled like the others they leave no room in the instruction cache (65,536 x
    // 2,048 in 64 sequences 398 us instead of 364; branches within one unrolled loop, 484).
    const bool mixed = here.marks.template mixed<true>(plan, at, row, lo, hi, pos);
    const bool none = mixed && here.marks.template none<true>(plan, at, row, lo, hi);
    if (none) {
      Vec zero;
      zero.fill(0.f);
      mine.then(zero, zero, true);
    } else if (mixed) {
#pragma unroll 1
      for (int i = 0; i < STEPS && row - i >= lo; ++i) {
        const int32_t m = here.marks.get(plan, at, i, row - i);
        Vec g, rest, dy = here.dy.get(i, at);
        gates(a.decay, here.f.get(i, at), g, rest);
        if (m >= 0 && (m & LAST) && a.state && in) dy = dy + state_row<TX, LOOSE>(a.state, a.state_stride, m, at.c, a.d);
        dy = g * dy;
        if (m < 0) dy.fill(0.f);
        mine.then(g, dy, m < 0 || (m & LAST));
      }
    } else {
      if (a.decay == GBA_DECAY_SIGMOID) {
#pragma unroll
        for (int i = 0; i < STEPS; ++i) sigmoid_gates(here.f.get(i, at), A[i], R[i]);
      } else if (!TAIL && a.tied) {  // a segment's pair has nothing of one minus the decay
#pragma unroll
        for (int i = 0; i < STEPS; ++i) log_gates<true>(here.f.get(i, at), A[i], R[i]);
      } else {
#pragma unroll
        for (int i = 0; i < STEPS; ++i) log_gates<false>(here.f.get(i, at), A[i], R[i]);
      }
#pragma unroll
      for (int i = 0; i < STEPS; ++i) mine.then(A[i], A[i] * here.dy.get(i, at), false);
    }
    sh.j.put(t & 1, at, mine);
    __syncthreads();
    Vec v;
    sh.j.then(t & 1, at, run, v);
    if constexpr (!TAIL) {
      // dx and df of position i, from the gradient v that comes to it and h before it
      auto outputs = [&](int i, const Vec& decay, const Vec& rest, const Vec& h) {
        v = v + here.dy.get(i, at);  // G
        Vec dx = v, df;
        v = v * decay;  // S
        if (a.tied) {
          float x[V], y[V];
          here.x.get(i, at).get(x);
          h.get(y);
#pragma unroll
          for (int j = 0; j < V; ++j) y[j] -= x[j];
          Vec diff;
          diff.set(y);
          dx = dx * rest;
          df = v * diff;
        } else {
          df = v * h;
        }
        if (a.decay == GBA_DECAY_SIGMOID) {
          df = df * rest;
        } else {
          float f[V], g[V];
          here.f.get(i, at).get(f);
          df.get(g);
#pragma unroll
          for (int j = 0; j < V; ++j) g[j] = f[j] > 0.f ? 0.f : g[j];
          df.set(g);
        }
        put_row<T, TX, STEPS, LOOSE>(a.out, at, row - i, a.d, dx);
        put_row<T, TX, STEPS, LOOSE>(a.df, at, row - i, a.d, df);
      };
      if (mixed) {
#pragma unroll 1
        for (int i = 0; i < STEPS && row - i >= lo; ++i) {
          if (!in) break;
          const int32_t m = here.marks.get(plan, at, i, row - i);
          if (m < 0) {
            v.fill(0.f);
            put_row<T, TX, STEPS, LOOSE>(a.out, at, row - i, a.d, v);
            put_row<T, TX, STEPS, LOOSE>(a.df, at, row - i, a.d, v);
            continue;
          }
          Vec g, rest, h = here.y.get(i, at);
          gates(a.decay, here.f.get(i, at), g, rest);
          if ((m & FIRST) && in) h = state_row<TX, LOOSE>(a.h0, a.h0_stride, m, at.c, a.d);
          if ((m & LAST) && in) v = state_row<TX, LOOSE>(a.state, a.state_stride, m, at.c, a.d);
          outputs(i, g, rest, h);
          if (a.last && (m & FIRST) && in) keep_row<TX, LOOSE>(a.last, a.last_stride, m, at.c, a.d, v);
        }
      } else if (in) {
#pragma unroll
        for (int i = 0; i < STEPS; ++i) outputs(i, A[i], R[i], here.y.get(i, at));
      }
    }
    sync_row<TX>();  // the row's lanes have read this stage
    fetch(stage);
    stage = stage == STAGES - 1 ? 0 : stage + 1;
  }
  copies_done<0>();
  if constexpr (TAIL) {
    if (at.ty == 0) run.put(plan.words + (size_t)at.seg * plan.pad + (size_t)at.col * At::COLS + at.tx * V);
  }
}

template <typename T, typename O, int TX, int STEPS, bool LOOSE>
cudaError_t start(const ScanArgs& a, const ScanPlan& p, cudaStream_t s) {
  if (p.chained) {
    const cudaError_t e = start_scan<Shared<T, O, TX, STEPS, LOOSE, true>>(
        k_scan_grad<T, O, TX, STEPS, LOOSE, true>, (p.n_segs - 1) * p.n_cols, a, p, s);
    if (e != cudaSuccess) return e;
  }
  // One or two blocks for each SM ask for so much shared memory that they are spread evenly: 256 blocks,
  // of which three fit an SM, took 522 us, and two an SM 413.
  constexpr size_t ONE = 226 << 10;
  const uint32_t blocks = p.n_segs * p.n_cols, each = (blocks + p.num_sms - 1) / p.num_sms;
  return start_scan<Shared<T, O, TX, STEPS, LOOSE, false>>(k_scan_grad<T, O, TX, STEPS, LOOSE, false>, blocks, a, p, s,
                                                           each == 1 ? ONE : each == 2 ? 112 << 10 : 0, ONE);
}

template <typename T, typename O>
cudaError_t launch_as(const ScanArgs& a, const ScanPlan& p, cudaStream_t s) {
  if (p.tx == 8)
    return p.loose ? start<T, O, 8, SCAN_STEPS, true>(a, p, s) : start<T, O, 8, SCAN_STEPS, false>(a, p, s);
  if constexpr (sizeof(T) == 4 || sizeof(O) == 4)
    if (p.steps == SCAN_WIDE)
      return p.loose ? start<T, O, 32, SCAN_WIDE, true>(a, p, s) : start<T, O, 32, SCAN_WIDE, false>(a, p, s);
  if (p.loose) return start<T, O, 32, SCAN_STEPS, true>(a, p, s);
  return p.steps == SCAN_STEPS ? start<T, O, 32, SCAN_STEPS, false>(a, p, s) : start<T, O, 32, SCAN_FEW, false>(a, p, s);
}

}  // namespace

cudaError_t start_scan_grad(const ScanArgs& a, int32_t type, int32_t out_type, const ScanPlan& p, cudaStream_t s) {
  if (type == GBA_F32) return launch_as<float, float>(a, p, s);
  if (type == GBA_BF16) return out_type == GBA_F32 ? launch_as<bf16, float>(a, p, s) : launch_as<bf16, bf16>(a, p, s);
  return out_type == GBA_F32 ? launch_as<f16, float>(a, p, s) : launch_as<f16, f16>(a, p, s);
}

}  // namespace gba

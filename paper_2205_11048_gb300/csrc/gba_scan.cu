// A gated linear recurrence over sequences, h_t = a_t h_(t-1) + b_t for every channel, and its
// gradient: with S the gradient that leaves a row towards the row before it,
//   G_t = dy_t + S_(t+1),  S_t = a_t G_t,  dx = G (1 - a) or G,  da = G (h_(t-1) - x) or G h_(t-1).
// Both are one scan, of the rows in order or from the last to the first; here a position is a
// row's place in that order, an entry a row before which the scan starts anew (from a state or
// zero), an exit one after which its value is kept.
//
// Bound by HBM bandwidth: the inputs are read once and the outputs written once where no sequence
// has to be split.  The positions are cut into as many segments as fill the GPU with the groups
// of channels; a block walks over its segment tile by tile, with the rows of the next tiles
// under way, and carries what comes out of one tile into the next.  In a tile a thread holds a few
// consecutive positions of four channels; the threads' stretches are joined as pairs (A, h) that
// stand for v -> A v + h, or for v -> h where an entry lies within, one barrier a tile.  Sequences
// that begin where segments do need no more.  Else a kernel before forms the pair of every
// segment, from the last entry in it on, which reads those rows once more; a block joins the
// pairs of the segments before its own.  Every order is fixed by the sizes: equal calls give
// equal bits.
//   bf16 65,536 x 2,048   64 sequences 137 us (5.9 TB/s), 16 164 us: few blocks, each a latency a tile; one
//                         239 us; in blocks that waited for one another's pairs 16 took 606 us
//   bf16 262,144 x 256    one sequence 130 us, of which the pairs' kernel takes two fifths: it reads both
//                         inputs once more, of which L2 keeps half for the kernel after it
//   gradient              bf16 65,536 x 2,048, 64 sequences 373 us, 32 padded ones 352 us; float32 20,003 x 501,
//                         packed, 109 us
// The gradient has 40 to 55 instructions an element and three blocks of four warps an SM, by its shared memory
// (four matrices, two tiles each): 44% of the issue slots, 3.9 TB/s, latency before bandwidth.
#include <algorithm>

#include "gba_scan.cuh"

namespace gba {

namespace {

constexpr int MARK_THREADS = 256;

// ---- marks -----------------------------------------------------------------------------
// Marks every row, checks offsets and lengths, and passes the states of empty sequences on.
__global__ void __launch_bounds__(MARK_THREADS)
    k_scan_marks(ScanArgs a, int32_t* marks, int64_t each) {
  follow();
  const int64_t id = (int64_t)blockIdx.x * MARK_THREADS + threadIdx.x, all = (int64_t)gridDim.x * MARK_THREADS;
  if (marks)
    for (int64_t t = id; t < a.n; t += all) {
      int32_t m;
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
        else  // before the first or behind the last
          m = -(int32_t)(lo < 0 && a.offsets[0] < a.n ? a.offsets[0] - t : a.n - t);
      } else {
        const int64_t seq = t / each, pos = t - seq * each, len = a.lengths[seq];
        m = pos < len ? (int32_t)seq * 4 + (pos == 0 ? FIRST : 0) + (pos + 1 == len || pos + 1 == each ? LAST : 0)
                      : -(int32_t)(each - pos);
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

// Sets the incoming states aside where the outgoing ones take their place: a sequence's last row may be
// written by another block than the one that reads its first.
__global__ void __launch_bounds__(MARK_THREADS) k_scan_states(ScanArgs a, float* to, int64_t stride) {
  follow();
  const int lane = threadIdx.x & 31;
  const int64_t all = (int64_t)gridDim.x * (MARK_THREADS / 32);
  for (int64_t s = (int64_t)blockIdx.x * (MARK_THREADS / 32) + (threadIdx.x >> 5); s < a.n_seq; s += all)
    for (int c = lane; c < a.d; c += 32) to[s * stride + c] = a.state[s * a.state_stride + c];
}

// ---- the scan ------------------------------------------------------------------------------
constexpr int STAGES = 2;  // tiles whose rows are in shared memory or under way

template <typename T, int TX, int STEPS, bool LOOSE>
struct Shared {
  Joint<TX, STEPS> j;
  struct {
    Stage<T, TX, STEPS, LOOSE> x, f;
    Marks<TX, STEPS> marks;
  } in[STAGES];
};

// TAIL: only the pair of each segment but the last, from its last entry on.
template <typename T, typename O, int TX, int STEPS, bool LOOSE, bool TAIL>
__global__ void __launch_bounds__(SCAN_THREADS, SCAN_BLOCKS) k_scan(ScanArgs a, ScanPlan plan) {
  extern __shared__ __align__(16) char smem[];
  auto& sh = *reinterpret_cast<Shared<T, TX, STEPS, LOOSE>*>(smem);
  using At = Spot<TX, STEPS>;
  follow();
  const At at(plan);
  const bool in = at.c < a.d;
  int64_t lo = (int64_t)at.seg * plan.rows;
  const int64_t hi = lo + plan.rows < a.n ? lo + plan.rows : a.n;
  Pairs run;  // of what has been walked over
  run.clear();
  if constexpr (TAIL) {
    const int32_t m = mark_of(plan, hi);  // of the next segment
    if (m < 0 || (m & FIRST)) return;  // nothing goes there
    // rows before the last entry do not matter
    if (plan.marks) {
      for (int64_t top = hi; top > lo; top -= SCAN_THREADS) {
        const int64_t r = top - 1 - threadIdx.x;
        const int32_t q = r >= lo ? plan.marks[r] : 0;
        const int found = __syncthreads_or(q < 0 || (q & FIRST) ? (int)(r - lo) + 1 : 0);
        if (found) {  // at least one in these rows: start with the lowest of them, the others follow
          lo = top - SCAN_THREADS > lo ? top - SCAN_THREADS : lo;
          break;
        }
      }
    } else {
      const int64_t first = hi / plan.each * plan.each;
      if (first > lo) lo = first;
    }
  } else if (plan.chained && at.seg > 0) {
    const int32_t m = mark_of(plan, lo);
    if (m >= 0 && !(m & FIRST)) into_segment(sh.j, plan, at, run);
  }
  const int tiles = (int)((hi - lo + At::ROWS - 1) / At::ROWS);
  int64_t row = lo + at.ty * STEPS, ahead = row;
  uint32_t pos = place_of(plan, row);
  int32_t mark = coming<STEPS, false>(plan, ahead, lo, hi);
  auto fetch = [&](int to) {
    if (mark > -STEPS) {  // else none of the rows belongs to a sequence
      sh.in[to].f.template fetch<false>(a.f, at, ahead, lo, hi, a.d, a.n);
      sh.in[to].x.template fetch<false>(a.x, at, ahead, lo, hi, a.d, a.n);
    }
    sh.in[to].marks.template fetch<false>(plan, at, ahead, lo, hi);
    ahead += At::ROWS;
    mark = coming<STEPS, false>(plan, ahead, lo, hi);
    copies_begun();
  };
#pragma unroll
  for (int k = 0; k < STAGES - 1; ++k) fetch(k);
  int stage = 0;
  for (int t = 0; t < tiles; ++t, row += At::ROWS, pos = moved<false>(plan, pos, At::ROWS)) {
    sync_row<TX>();  // the row's lanes have done with the stage that is filled next
    fetch(stage == 0 ? STAGES - 1 : stage - 1);
    copies_done<STAGES - 1>();
    sync_row<TX>();
    const auto& here = sh.in[stage];
    Pairs mine;
    mine.clear();
    Vec A[STEPS], B[STEPS];  // h -> A h + B
    if (a.decay == GBA_DECAY_SIGMOID) {
#pragma unroll
      for (int i = 0; i < STEPS; ++i) sigmoid_gates(here.f.get(i, at), A[i], B[i]);
    } else if (a.tied) {
#pragma unroll
      for (int i = 0; i < STEPS; ++i) log_gates<true>(here.f.get(i, at), A[i], B[i]);
    } else {
#pragma unroll
      for (int i = 0; i < STEPS; ++i) log_gates<false>(here.f.get(i, at), A[i], B[i]);
    }
    if (a.tied) {
#pragma unroll
      for (int i = 0; i < STEPS; ++i) B[i] = B[i] * here.x.get(i, at);
    } else {
#pragma unroll
      for (int i = 0; i < STEPS; ++i) B[i] = here.x.get(i, at);
    }
    int32_t m[STEPS];
    const bool mixed = here.marks.template mixed<false>(plan, at, row, lo, hi, pos);
    if (mixed) {
      here.marks.template all<false>(plan, at, row, lo, hi, m);
#pragma unroll
      for (int i = 0; i < STEPS; ++i) {
        if (m[i] < 0) {
          B[i].fill(0.f);
          if (!inside(row + i, lo, hi)) continue;  // no row of the segment: it changes nothing
        } else if ((m[i] & FIRST) && a.state && in) {
          B[i] = fma_v(A[i], state_row<TX, LOOSE>(a.state, a.state_stride, m[i], at.c, a.d), B[i]);
        }
        mine.then(A[i], B[i], m[i] < 0 || (m[i] & FIRST));
      }
    } else {
#pragma unroll
      for (int i = 0; i < STEPS; ++i) mine.then(A[i], B[i], false);
    }
    sh.j.put(t & 1, at, mine);
    __syncthreads();
    stage = stage == STAGES - 1 ? 0 : stage + 1;
    Vec h;
    sh.j.then(t & 1, at, run, h);
    if constexpr (!TAIL) {
      if (in) {
        if (mixed) {
#pragma unroll
          for (int i = 0; i < STEPS; ++i) {
            if (!inside(row + i, lo, hi)) break;
            h = m[i] < 0 || (m[i] & FIRST) ? B[i] : fma_v(A[i], h, B[i]);
            if (a.last && m[i] >= 0 && (m[i] & LAST) && in) keep_row<TX, LOOSE>(a.last, a.last_stride, m[i], at.c, a.d, h);
            put_row<O, TX, STEPS, LOOSE>(a.out, at, row + i, a.d, h);
          }
        } else {
#pragma unroll
          for (int i = 0; i < STEPS; ++i) {
            h = fma_v(A[i], h, B[i]);
            put_row<O, TX, STEPS, LOOSE>(a.out, at, row + i, a.d, h);
          }
        }
      }
    }
  }
  copies_done<0>();
  if constexpr (TAIL) {
    if (at.ty == 0) run.put(plan.words + (size_t)at.seg * plan.pad + (size_t)at.col * At::COLS + at.tx * V);
  }
}

// ---- launches ------------------------------------------------------------------------------
constexpr int64_t SHORT = 256;  // rows of a segment of whole sequences, about
// Segments of ragged batches differ in work, so there are up to four for each place on the SMs, of at
// least LONG rows: gradient of 65,536 x 2,048, padded, 394 us with one, 352 with four; of 20,003 x 501
// (float32, packed) 126 with one, 152 with three.
constexpr int64_t LONG = 512;

struct Shape {
  ScanPlan p;
  bool marks;
  int64_t aside;        // floats of a row of the states that are set aside, or 0
  size_t words, states, bytes;  // of the workspace: the pairs, then the marks, from `states` on the states
};

Shape shape_of(const ScanArgs& a, int32_t type, int32_t out_type, bool grad, int num_sms) {
  Shape s{};
  ScanPlan& p = s.p;
  auto fits = [&](const void* q, int64_t stride, size_t bytes) {
    return !q || vector_of(V, q, stride, a.d, bytes) == V;
  };
  const size_t b = type_bytes(type), ob = type_bytes(out_type);
  bool ok = fits(a.x.p, a.x.stride, b) && fits(a.f.p, a.f.stride, b) && fits(a.state, a.state_stride, 4) &&
            fits(a.last, a.last_stride, 4) && fits(a.h0, a.h0_stride, 4) &&
            fits(a.out.p, a.out.stride, grad ? b : ob);
  if (grad) ok = ok && fits(a.y.p, a.y.stride, ob) && fits(a.dy.p, a.dy.stride, ob) && fits(a.df.p, a.df.stride, b);
  p.loose = !ok;
  p.num_sms = num_sms;
  p.tx = a.d <= 16 * V ? 8 : 32;
  const uint32_t cols = (uint32_t)(p.tx * V);
  p.n_cols = (uint32_t)((a.d + cols - 1) / cols);
  p.pad = p.n_cols * cols;
  p.each = (uint32_t)(a.n_seq > 0 ? a.n / a.n_seq : 0);
  s.marks = a.offsets || a.lengths;
  // blocks that run at a time: 16-bit rows of four (the gradient: three) fit an SM, float32 rows of one less.
  // The gradient's float32 rows of ragged or of many sequences go half as many at a time, of which three
  // blocks fit: 256 x 128 x 2,048 239 us against 408, packed 20,003 x 501 109 and 126; but one sequence of
  // 131,072 x 512 390 against 324.
  const bool wide = grad ? b == 4 || ob == 4 : b == 4;
  const bool many = a.n_seq * p.n_cols >= (int64_t)num_sms * (grad ? 8 : 5) / 4;
  const bool half = grad && wide && p.tx == 32 && (s.marks || many);
  const int64_t ty = SCAN_THREADS / p.tx;
  const int64_t slots = (int64_t)num_sms * ((grad ? GRAD_BLOCKS : SCAN_BLOCKS) - (wide && !half));
  const int steps = half ? SCAN_WIDE : SCAN_STEPS;
  const bool few = (a.n + ty * steps - 1) / (ty * steps) * p.n_cols < num_sms;
  p.steps = few && !p.loose && p.tx == 32 ? SCAN_FEW : steps;
  const int64_t tile = ty * p.steps, want = std::max<int64_t>(1, slots / p.n_cols);
  int64_t rows = std::max((a.n + want - 1) / want, tile);
  if (s.marks) {
    rows = std::max(rows / 4, std::min(rows, LONG));
    rows = (rows + tile - 1) / tile * tile;
    p.chained = rows < a.n;
  } else if (a.n > 0) {
    const int64_t each = p.each;
    if (each <= 2 * rows || many) {
      // whole sequences, which need nothing of one another, so the segments may be short
      rows = std::max(tile, std::min(rows, SHORT));
      rows = std::max<int64_t>(1, (rows + each / 2) / each) * each;
    } else {
      const int64_t pieces = std::max<int64_t>(1, want / a.n_seq);
      p.chained = pieces > 1;
      rows = pieces == 1 ? each : ((each + pieces - 1) / pieces + tile - 1) / tile * tile;
    }
  }
  p.rows = rows;
  p.n_segs = (uint32_t)((a.n + rows - 1) / std::max<int64_t>(rows, 1));
  // Whole sequences in fewer blocks than run at a time: forwards groups of half as many channels (16 x 4,096
  // x 2,048 164 us, with whole ones 177; float32 32 x 1,024 x 2,048 139 and 146).  Elsewhere they are slower:
  // 64 x 1,024 x 2,048 156 us against 138, its gradient 406 against 371.
  if (!grad && !s.marks && !p.chained && !p.loose && p.tx == 32 && p.steps == SCAN_STEPS &&
      (int64_t)p.n_segs * p.n_cols <= (int64_t)num_sms * SCAN_BLOCKS) {
    p.tx = 16;
    p.n_cols = (uint32_t)((a.d + 16 * V - 1) / (16 * V));
    p.pad = p.n_cols * 16 * V;
  }
  s.words = p.chained ? (size_t)p.n_segs * p.pad * 8 : 0;
  s.states = (s.words + (s.marks ? (size_t)a.n * 4 : 0) + 15) / 16 * 16;
  // Forwards a block reads a state before the barrier behind which it writes one; backwards it reads it
  // behind that barrier once more, while another warp may write.
  if (a.n > 0 && a.state && a.state == a.last && (grad || p.chained)) s.aside = ((int64_t)a.d + V - 1) / V * V;
  s.bytes = s.states + (size_t)(a.n_seq * s.aside) * 4;
  return s;
}

template <typename T, typename O, int TX, int STEPS, bool LOOSE>
cudaError_t start(const ScanArgs& a, const ScanPlan& p, cudaStream_t s) {
  using S = Shared<T, TX, STEPS, LOOSE>;
  if (p.chained) {
    const cudaError_t e = start_scan<S>(k_scan<T, T, TX, STEPS, LOOSE, true>, (p.n_segs - 1) * p.n_cols, a, p, s);
    if (e != cudaSuccess) return e;
  }
  return start_scan<S>(k_scan<T, O, TX, STEPS, LOOSE, false>, p.n_segs * p.n_cols, a, p, s);
}

template <typename T, typename O>
cudaError_t launch_as(const ScanArgs& a, const ScanPlan& p, cudaStream_t s) {
  if (p.tx == 8)
    return p.loose ? start<T, O, 8, SCAN_STEPS, true>(a, p, s) : start<T, O, 8, SCAN_STEPS, false>(a, p, s);
  if (p.tx == 16)  // of whole sequences
    return start_scan<Shared<T, 16, SCAN_STEPS, false>>(k_scan<T, O, 16, SCAN_STEPS, false, false>, p.n_segs * p.n_cols, a, p, s);
  if (p.loose) return start<T, O, 32, SCAN_STEPS, true>(a, p, s);
  return p.steps == SCAN_STEPS ? start<T, O, 32, SCAN_STEPS, false>(a, p, s) : start<T, O, 32, SCAN_FEW, false>(a, p, s);
}

cudaError_t start_scan_forward(const ScanArgs& a, int32_t type, int32_t out_type, const ScanPlan& p, cudaStream_t s) {
  if (type == GBA_F32) return launch_as<float, float>(a, p, s);
  if (type == GBA_BF16) return out_type == GBA_F32 ? launch_as<bf16, float>(a, p, s) : launch_as<bf16, bf16>(a, p, s);
  return out_type == GBA_F32 ? launch_as<f16, float>(a, p, s) : launch_as<f16, f16>(a, p, s);
}

}  // namespace

size_t scan_workspace(const ScanArgs& a, int32_t type, int32_t out_type, bool grad, int num_sms) {
  return shape_of(a, type, out_type, grad, num_sms).bytes;
}

cudaError_t launch_scan(const ScanArgs& args, int32_t type, int32_t out_type, bool grad, char* ws, int num_sms,
                        cudaStream_t s) {
  ScanArgs a = args;
  Shape h = shape_of(a, type, out_type, grad, num_sms);
  h.p.words = reinterpret_cast<uint64_t*>(ws);
  int32_t* marks = h.marks ? reinterpret_cast<int32_t*>(ws + h.words) : nullptr;
  h.p.marks = marks;
  if (h.marks || a.n == 0) {
    const int64_t work = std::max<int64_t>(a.n, a.n_seq * 32);
    const unsigned grid = (unsigned)std::min<int64_t>((work + MARK_THREADS - 1) / MARK_THREADS, (int64_t)num_sms * 8);
    const cudaError_t e = launch_following(k_scan_marks, dim3(std::max(1u, grid)), MARK_THREADS, 0, s, a, marks,
                                           a.n_seq > 0 ? a.n / a.n_seq : 0);
    if (e != cudaSuccess || a.n == 0) return e;
  }
  if (h.aside) {
    float* const to = reinterpret_cast<float*>(ws + h.states);
    const unsigned grid = (unsigned)std::min<int64_t>((a.n_seq + MARK_THREADS / 32 - 1) / (MARK_THREADS / 32), (int64_t)num_sms * 8);
    const cudaError_t e = launch_following(k_scan_states, dim3(grid), MARK_THREADS, 0, s, a, to, h.aside);
    if (e != cudaSuccess) return e;
    a.state = to;
    a.state_stride = h.aside;
  }
  return grad ? start_scan_grad(a, type, out_type, h.p, s) : start_scan_forward(a, type, out_type, h.p, s);
}

}  // namespace gba

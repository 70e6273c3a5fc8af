// Scaled embedding lookup, and its gradient by sorted tokens.
//
// Lookup: out_i = s * W[row(id_i)], a gather like k_pull_rows with a scale, types and
// strides.  Bound by HBM bandwidth or, where rows repeat, by L2's: the rows that occur are
// read (repeated ones from L2) and n rows written.
//
// Gradient: G[r] = s * sum over the positions i with row(id_i) = r of g_i.  The rows of the
// ids are sorted with their positions as payload (the step's onesweep passes; stable, so
// a row's positions stay ascending and its sum has one order), and then each gradient row
// is read once, where it lies:
//  - items: a run of equal rows is cut at the sorted positions p = 0 mod c whose row stood
//    at p - c too, so runs shorter than c stay whole and no item is longer than 2 c - 1
//    positions;
//  - sums: one lane group per item and column slab adds the item's gradient rows; a run of
//    one item goes straight to the output, the others leave float32 sums of their items
//    (in slots that follow from the cut's position: 2 p / c for the item before the first
//    cut p, one more for the item that starts at p).  Rows of a dense output that do not
//    occur are cleared by the same kernel, so that every row is written once;
//  - merge: a warp per cut run and slab, or one or several blocks where the run has many
//    items, adds the items' sums in their order.
// The rows of an item follow one another through a lane group, so the length of a hot row's
// items bounds the time of small calls, and their sums' traffic that of large ones: c is 16
// for gradients of up to 2^26 elements (a message of 6,656 x 16 floats, kernel of the sums:
// 7.8 us, and 24.7 with 64), 64 above.
#include <cooperative_groups.h>

#include <algorithm>

#include "gba_worker.cuh"

namespace cg = cooperative_groups;

namespace gba {

namespace {

constexpr int THREADS = 256;
constexpr uint32_t FULL = 0xffffffffu;
constexpr int MERGE_THREADS = 512, HUGE_SPLIT = 8;
constexpr int64_t SMALL_N = 8192;  // that k_token_small takes
constexpr uint32_t LONG_PARTS = 16, HUGE_PARTS = 256;
constexpr int MIN_CUT_LG = 4, MAX_CUT_LG = 6;
inline int cut_lg_of(int64_t n, int64_t d) { return n * d <= 1ll << 26 ? MIN_CUT_LG : MAX_CUT_LG; }
constexpr int ITEM_TILE = 2048;  // sorted positions per tile of the item scan
constexpr int MAX_RADIX = 512;   // of a sort pass

__device__ __forceinline__ unsigned long long ld_relaxed_u64(const unsigned long long* p) {
  unsigned long long v;
  asm volatile("ld.relaxed.gpu.global.u64 %0, [%1];" : "=l"(v) : "l"(p) : "memory");
  return v;
}
__device__ __forceinline__ void st_relaxed_u64(unsigned long long* p, unsigned long long v) {
  asm volatile("st.relaxed.gpu.global.u64 [%0], %1;" ::"l"(p), "l"(v) : "memory");
}
__device__ __forceinline__ uint32_t lanemask_lt() {
  uint32_t m;
  asm("mov.u32 %0, %%lanemask_lt;" : "=r"(m));
  return m;
}

// ---- lookup -----------------------------------------------------------------------

// The lanes of the group of 1 << lg that this lane is in.
__device__ __forceinline__ uint32_t group_mask(int lg) {
  const uint32_t first = (threadIdx.x & 31) >> lg << lg;
  return lg == 5 ? FULL : ((1u << (1 << lg)) - 1u) << first;
}

// Writes a lane group's values x, V consecutive ones a lane, to the n elements that exist from
// `to` on (ADD: adds them), neighbouring lanes to neighbouring elements: the lanes' values
// change places through shared memory.  For outputs whose rows do not start on the boundary
// that vectors need.
template <typename T, int V, bool ADD>
__device__ __forceinline__ void write_in_order(float* swap, const float (&x)[V], int lg, int64_t n, T* to) {
  const uint32_t mask = group_mask(lg);
  const int L = 1 << lg, l = threadIdx.x & (L - 1);
  float* mine = swap + (threadIdx.x >> lg << lg) * V;  // the group's
  __syncwarp(mask);
#pragma unroll
  for (int j = 0; j < V; j += 4)
    *reinterpret_cast<float4*>(mine + l * V + j) = make_float4(x[j], x[j + 1], x[j + 2], x[j + 3]);
  __syncwarp(mask);
  const int count = n < L * V ? (int)n : L * V;
  if constexpr (sizeof(T) == 4) {
    mine += l;
    to += l;
    if (count == 32 * V) {
#pragma unroll
      for (int i = 0; i < V; ++i) to[i * 32] = ADD ? to[i * 32] + mine[i * 32] : mine[i * 32];
    } else {
      for (int e = 0; e + l < count; e += L) to[e] = ADD ? to[e] + mine[e] : mine[e];
    }
  } else {  // in pairs from the first 4-byte boundary on
    static_assert(!ADD, "");
    const int odd = (int)((uintptr_t)to >> 1 & 1), pairs = (count - odd) >> 1;
    if (odd && l == 0) to[0] = from_float<T>(mine[0]);
    if (odd + 2 * pairs < count && l == L - 1) to[count - 1] = from_float<T>(mine[count - 1]);
    mine += odd + 2 * l;
    to += odd + 2 * l;
    auto put = [&](int e) {
      const float y[2] = {mine[e], mine[e + 1]};
      Pack<T, 2> o;
      o.set(y);
      o.store(to + e);
    };
    if (pairs >= 16 * V - 1 && lg == 5) {  // all of them, but for the last where the first is odd
#pragma unroll
      for (int i = 0; i < V / 2 - 1; ++i) put(i * 64);
      if ((V / 2 - 1) * 32 + l < pairs) put((V / 2 - 1) * 64);
    } else {
      for (int q = l; q < pairs; q += L) put(2 * (q - l));
    }
  }
}

// Which rows may start anywhere, or not be whole numbers of vectors: none, the input's, or the
// output's as well.
enum Rows { EVEN, LOOSE_IN, LOOSE };

// A lane group of 1 << lg lanes per token and slab of K * V columns a lane; the next token's id
// is read while this one's row arrives (float32 131,072 x 64: 18.5 -> 11 us).  131,072 x 1,024
// float32 to bf16 takes 70 us: 805 MB through L2 (11.5 TB/s), 344 MB of them from and to HBM.
template <typename TI, typename TO, int V, int K, Rows R>
__global__ void __launch_bounds__(THREADS) k_embed(EmbedArgs a, int lg) {
  __shared__ __align__(16) float swap[R == LOOSE ? THREADS * V : 4];
  follow();
  const int L = 1 << lg;
  const int l = threadIdx.x & (L - 1);
  const int64_t groups = (int64_t)gridDim.x * (THREADS >> lg);
  const int64_t g0 = ((int64_t)blockIdx.x * THREADS + threadIdx.x) >> lg;
  const int64_t c0 = ((int64_t)blockIdx.y * K * L + l) * V;
  // A HASH table is where its description says at the time: a captured lookup runs on after the
  // table has moved to more slots.
  const bool hash = a.id_mode == GBA_ID_HASH;
  const TI* w = static_cast<const TI*>(hash ? static_cast<const void*>(a.hinfo->w) : a.w);
  const uint64_t rows = hash ? a.hinfo->mask + 1 : (uint64_t)a.V;
  const char* lo = reinterpret_cast<const char*>(w);
  const char* hi = lo + ((rows - 1) * (uint64_t)a.w_stride + (uint64_t)a.d) * sizeof(TI);
  int64_t next = g0 < a.n ? a.ids[g0] : 0;
  for (int64_t i = g0; i < a.n; i += groups) {
    const int64_t id = next;
    if (i + groups < a.n) next = a.ids[i + groups];
    bool zero = id == a.pad_id && a.pad_id != GBA_NO_PAD;
    bool fresh = false;  // HASH: an id never seen has its initial values
    uint64_t row = 0;
    if (!zero) {
      bool bad = false;
      if (a.id_mode == GBA_ID_DIRECT) {
        bad = id < 0 || id >= a.V;
        row = (uint64_t)id;
      } else if (a.id_mode == GBA_ID_MODULO) {
        row = mod_u64((uint64_t)id, (uint64_t)a.V, a.mod_magic);
      } else {
        bad = (unsigned long long)id == HASH_EMPTY;
        if (!bad) {
          row = hash_find(*a.hinfo, id);
          fresh = row > a.hinfo->mask;
        }
      }
      if (bad) {
        if (l == 0 && blockIdx.y == 0) raise_error(a.err, ERR_ID_RANGE);
        zero = true;
      }
    }
    const TI* src = w + row * (uint64_t)a.w_stride;
    TO* dst = static_cast<TO*>(a.out) + (uint64_t)i * (uint64_t)a.out_stride;
    std::conditional_t<R != EVEN, Loose<TI>, Pack<TI, V>> in[K];
    if (!zero && !fresh) {
#pragma unroll
      for (int k = 0; k < K; ++k) {
        const int64_t c = c0 + (int64_t)k * L * V;
        if (c >= a.d) continue;
        if constexpr (R != EVEN)
          in[k].load(src + c, a.d - c, lo, hi);
        else
          in[k].load(src + c);
      }
    }
#pragma unroll
    for (int k = 0; k < K; ++k) {
      const int64_t c = c0 + (int64_t)k * L * V;
      if (c - l * V >= a.d || (R != LOOSE && c >= a.d)) continue;  // of the group, or of the lane
      float x[V] = {};
      if (!zero && c < a.d) {
        if (fresh) {
#pragma unroll
          for (int j = 0; j < V; ++j)
            x[j] = init_weight(a.hinfo->seed, a.hinfo->tag, (uint64_t)id * (uint64_t)a.d + (uint64_t)(c + j));
        } else {
          in[k].get(x);
        }
#pragma unroll
        for (int j = 0; j < V; ++j) x[j] *= a.scale;
      }
      if constexpr (R == LOOSE) {
        write_in_order<TO, V, false>(swap, x, lg, a.d - (c - l * V), dst + (c - l * V));
      } else {
        Pack<TO, V> o;
        o.set(x);
        o.store(dst + c);
      }
    }
  }
}

template <typename TI, typename TO, int V, Rows R>
cudaError_t embed_as(const EmbedArgs& a, int num_sms, cudaStream_t s) {
  const int64_t pieces = (a.d + V - 1) / V;
  int lg = 0;
  while ((1 << lg) < pieces && lg < 5) ++lg;
  const int64_t each = (pieces + (1 << lg) - 1) >> lg;  // of a lane
  // up to four pieces a lane in flight, unless that leaves SMs without work
  const bool wide = a.n * pieces / 128 >= (int64_t)num_sms * 16;
  const int64_t slabs = wide ? (each + 3) / 4 : each;
  const int64_t blocks = (a.n + (THREADS >> lg) - 1) / (THREADS >> lg);
  const dim3 grid((unsigned)std::min<int64_t>(blocks, (int64_t)num_sms * 32), (unsigned)slabs);
  auto kernel = k_embed<TI, TO, V, 1, R>;
  switch ((each + slabs - 1) / slabs) {
    case 2: kernel = k_embed<TI, TO, V, 2, R>; break;
    case 3: kernel = k_embed<TI, TO, V, 3, R>; break;
    case 4: kernel = k_embed<TI, TO, V, 4, R>; break;
  }
  return launch_following(kernel, grid, THREADS, 0, s, a, lg);
}

// Vectors of 8 elements, or of 4 float32; loose rows by 16 bytes of the input.
template <typename TI, typename TO>
cudaError_t embed_types(const EmbedArgs& a, int num_sms, cudaStream_t s) {
  constexpr int V = 16 / (int)std::min(sizeof(TI), sizeof(TO)), VL = Loose<TI>::V;
  if (vector_of(V, a.w, a.w_stride, a.d, sizeof(TI)) == V && vector_of(V, a.out, a.out_stride, a.d, sizeof(TO)) == V)
    return embed_as<TI, TO, V, EVEN>(a, num_sms, s);
  if (vector_of(VL, a.out, a.out_stride, a.d, sizeof(TO)) == VL) return embed_as<TI, TO, VL, LOOSE_IN>(a, num_sms, s);
  return embed_as<TI, TO, VL, LOOSE>(a, num_sms, s);
}

// ---- gradient: workspace -------------------------------------------------------------

struct Counters {
  uint32_t step;     // the call's error word
  uint32_t tickets[MAX_PASSES];
  uint32_t scan_ticket;
  uint32_t n_items, n_runs;
  uint32_t n_cut[3];  // cut runs of a few items, of LONG_PARTS and more, of HUGE_PARTS and more
  uint32_t P;        // positions that are no padding: the first P of the sorted ones
  uint32_t rest;     // claims of the rows that are cleared
  uint32_t pad[3];
};
static_assert(sizeof(Counters) == 64, "the histograms follow it");

struct Item {
  uint32_t start;  // position << 1 | starts its run
  uint32_t run;    // run << 1 | the run has several items
};

// Where the parts of the workspace are; what must start at zero comes first.
struct GradPlan {
  SortPlan sort;
  size_t counters, hist, sort_status, scan_status, present, huge_done, cleared;  // cleared: bytes from 0 on
  size_t keys[2], vals[2], items, run_row, run_start, cuts, parts, huge, bytes;
  int64_t tiles, n_huge_done;
  int cut_lg;
  bool small;  // keys, sort and items by one cluster, or one block
};

// Floats from one item's sum to the next: vectors of them are aligned, whatever the width.
__host__ __device__ __forceinline__ uint64_t part_stride(int64_t d) { return ((uint64_t)d + 7) / 8 * 8; }

GradPlan plan_of(const EmbedGradArgs& a) {
  GradPlan p{};
  const uint64_t top = (uint64_t)a.V;  // the key that stands for padding
  int bits = 1;
  while (bits < 32 && (top >> bits) != 0) ++bits;
  // (a table whose bits of presence eight blocks would take long to clear is not for it)
  p.small = a.n <= SMALL_N && (!a.dense || a.accumulate || a.V <= 1 << 22);
  p.sort = make_sort_plan(bits, 9);
  p.tiles = (a.n + ITEM_TILE - 1) / ITEM_TILE;
  p.cut_lg = cut_lg_of(a.n, a.d);
  size_t at = 0;
  auto take = [&](size_t bytes) {
    const size_t o = at;
    at += (bytes + 255) & ~(size_t)255;
    return o;
  };
  const size_t n = (size_t)a.n;
  p.counters = take(sizeof(Counters));
  p.hist = take((size_t)MAX_PASSES * MAX_RADIX * 4);
  p.sort_status = take(sort_status_words(a.n, p.sort.radix) * 8);
  p.scan_status = take((size_t)p.tiles * 8);
  p.present = take(a.dense && !a.accumulate ? ((size_t)a.V + 31) / 32 * 4 : 0);
  const size_t huge_units = ((size_t)(a.n >> p.cut_lg) / HUGE_PARTS + 1) * (((size_t)a.d + 127) / 128);
  p.huge_done = take(huge_units * 4);
  p.cleared = at;
  for (int i = 0; i < 2; ++i) {
    p.keys[i] = take(n * 4);
    p.vals[i] = take(n * 4);
  }
  p.items = take(n * sizeof(Item));
  p.run_row = take(n * 4);
  p.run_start = take(n * 4);
  p.cuts = take(3 * ((n >> p.cut_lg) + 1) * 8);
  p.parts = take((2 * (n >> p.cut_lg) + 2) * part_stride(a.d) * 4);
  p.huge = take(huge_units * HUGE_SPLIT * 64 * sizeof(float4));
  p.n_huge_done = (int64_t)huge_units;
  p.bytes = at;
  return p;
}

// ---- gradient: sort --------------------------------------------------------------------

__global__ void __launch_bounds__(THREADS) k_token_clear(uint4* p, int64_t n) {
  follow();
  for (int64_t i = (int64_t)blockIdx.x * THREADS + threadIdx.x; i < n; i += (int64_t)gridDim.x * THREADS)
    p[i] = make_uint4(0u, 0u, 0u, 0u);
}

struct KeyArgs {
  const int64_t* ids;
  uint32_t n;
  int32_t id_mode;
  int64_t pad_id;
  int64_t V;
  uint64_t mod_magic;
  uint32_t* hist;  // [passes][radix]
  uint32_t* keys;
};

// The row of an id, or V for padding, which so sorts last.
__device__ __forceinline__ uint32_t key_of(const KeyArgs& a, int64_t id, bool& bad) {
  if (id == a.pad_id && a.pad_id != GBA_NO_PAD) return (uint32_t)a.V;
  if (a.id_mode == GBA_ID_MODULO) return (uint32_t)mod_u64((uint64_t)id, (uint64_t)a.V, a.mod_magic);
  if (id >= 0 && id < a.V) return (uint32_t)id;
  bad = true;
  return (uint32_t)a.V;
}

// The keys of every id and the digit counts of every pass (262,144 ids: 7 us, latency).
__global__ void __launch_bounds__(THREADS) k_token_keys(KeyArgs a, SortPlan plan, ErrSink err) {
  __shared__ uint32_t h[MAX_PASSES * MAX_RADIX];
  const int words = plan.passes * plan.radix;
  for (int i = threadIdx.x; i < words; i += THREADS) h[i] = 0u;
  follow();
  __syncthreads();
  const uint32_t stride = gridDim.x * THREADS;
  for (uint32_t i = blockIdx.x * THREADS + threadIdx.x; i < a.n; i += stride) {
    bool bad = false;
    const uint32_t key = key_of(a, a.ids[i], bad);
    if (bad) raise_error(err, ERR_ID_RANGE);
    a.keys[i] = key;
    for (int p = 0; p < plan.passes; ++p)
      atomicAdd(h + p * plan.radix + ((key >> plan.shift[p]) & plan.mask[p]), 1u);
  }
  __syncthreads();
  for (int i = threadIdx.x; i < words; i += THREADS)
    if (h[i]) atomicAdd(a.hist + i, h[i]);
}

// ---- gradient: items ---------------------------------------------------------------------

struct ItemArgs {
  const uint32_t* keys;  // sorted rows
  uint32_t n;
  uint32_t pad_key;
  Counters* ctr;
  unsigned long long* status;  // [tiles]
  Item* items;
  uint32_t* run_row;
  uint32_t* run_start;
  uint2* cuts;       // (run, first cut): [3][n >> cut_lg + 1]
  int64_t* ids_out;  // message form
  uint32_t* present; // dense form, overwriting: a bit per row that occurs
  int32_t cut_lg;
  uint32_t* huge_done;
  int64_t n_huge_done;
};

// What stands at sorted position p < n.
struct Marks {
  bool head, start;        // of a run, of an item
  bool several;            // the run has more items than this one
  bool first_cut;          // p is the run's first cut
  bool is_long, is_huge;   // and the run has LONG_PARTS items at least, HUGE_PARTS at least
  bool last;               // before the padding, or the end
};
__device__ __forceinline__ Marks marks_of(const ItemArgs& a, const uint32_t* keys, uint32_t p, uint32_t& key) {
  const uint32_t cut = 1u << a.cut_lg;
  key = keys[p];
  const uint32_t before = p > 0 ? keys[p - 1] : ~0u;
  const uint32_t after = p + 1 < a.n ? keys[p + 1] : a.pad_key;
  const uint32_t q = ((p + cut - 1) >> a.cut_lg << a.cut_lg) + cut;  // a head's first cut, if its run is so long
  const bool at_cut = (p & (cut - 1)) == 0 && p >= cut;
  const uint64_t far = (uint64_t)p + ((uint64_t)(LONG_PARTS - 1) << a.cut_lg);
  const uint32_t at_q = q < a.n ? keys[q] : ~0u;
  const uint32_t back = at_cut ? keys[p - cut] : ~0u;
  const uint32_t back2 = at_cut && p >= 2 * cut ? keys[p - 2 * cut] : ~0u;
  const uint64_t farther = (uint64_t)p + ((uint64_t)(HUGE_PARTS - 1) << a.cut_lg);
  const uint32_t at_far = at_cut && far < a.n ? keys[far] : ~0u;
  const uint32_t at_farther = at_cut && farther < a.n ? keys[farther] : ~0u;
  const bool real = key != a.pad_key;
  Marks m;
  m.head = real && key != before;
  m.start = m.head || (real && back == key);
  m.several = !m.head || at_q == key;
  m.first_cut = !m.head && m.start && back2 != key;
  m.is_long = at_far == key;
  m.is_huge = at_farther == key;
  m.last = real && after == a.pad_key;
  return m;
}

__device__ __forceinline__ void write_item(const ItemArgs& a, uint32_t p, uint32_t key, uint32_t item, uint32_t run,
                                           bool head, bool several, bool first_cut, bool is_long, bool is_huge) {
  if (head) {
    a.run_row[run] = key;
    a.run_start[run] = p;
    if (a.ids_out) a.ids_out[run] = (int64_t)key;
    if (a.present) atomicOr(a.present + (key >> 5), 1u << (key & 31u));
  } else if (first_cut) {
    const uint32_t which = is_huge ? 2u : is_long ? 1u : 0u, room = (a.n >> a.cut_lg) + 1u;
    const uint32_t c = atomicAdd(&a.ctr->n_cut[which], 1u);
    if (c < room) a.cuts[which * room + c] = make_uint2(run, p);
  }
  a.items[item] = Item{p << 1 | (head ? 1u : 0u), run << 1 | (several ? 1u : 0u)};
}

// Look-back word: [61:60] flag, [59:30] items, [29:0] runs.
constexpr unsigned long long SCAN_AGG = 1ull << 60;
constexpr unsigned long long SCAN_INCL = 2ull << 60;
constexpr unsigned long long SCAN_VALUE = (1ull << 60) - 1;

// Heads of runs and items, numbered over the whole array by one pass with decoupled
// look-back (Merrill & Garland 2016), tiles by ticket.  Every wait is bounded.  Latency bounds
// it (20 tiles 10.5 us, 128 tiles 13): a ticket, the loads of a tile all at once, the tiles before.
__global__ void __launch_bounds__(THREADS) k_token_items(ItemArgs a, ErrSink err, int64_t wait_ns) {
  constexpr int WARPS = THREADS / 32, PER_WARP = ITEM_TILE / WARPS, ROUNDS = PER_WARP / 32;
  __shared__ uint32_t s_tile, s_failed;
  __shared__ unsigned long long s_warp[WARPS];
  __shared__ unsigned long long s_prefix;
  follow();
  const int tid = threadIdx.x, lane = tid & 31, warp = tid >> 5;
  if (tid == 0) {
    s_tile = atomicAdd(&a.ctr->scan_ticket, 1u);
    s_failed = *(const volatile uint32_t*)err.step;
  }
  __syncthreads();
  if (s_failed != 0u) return;  // the counters stay zero: no items, no runs
  const uint32_t tile = s_tile;
  const uint32_t base = tile * (uint32_t)ITEM_TILE + (uint32_t)(warp * PER_WARP);

  uint32_t key[ROUNDS], heads[ROUNDS], starts[ROUNDS], several[ROUNDS], firsts[ROUNDS], longs[ROUNDS], huges[ROUNDS];
  unsigned long long sum = 0ull;
#pragma unroll
  for (int j = 0; j < ROUNDS; ++j) {  // every load of the tile before anything is written
    const uint32_t p = base + (uint32_t)(j * 32 + lane);
    Marks m{};
    key[j] = a.pad_key;
    if (p < a.n) {
      m = marks_of(a, a.keys, p, key[j]);
      if (m.last) a.ctr->P = p + 1;
    }
    heads[j] = __ballot_sync(FULL, m.head);
    starts[j] = __ballot_sync(FULL, m.start);
    several[j] = __ballot_sync(FULL, m.several);
    firsts[j] = __ballot_sync(FULL, m.first_cut);
    longs[j] = __ballot_sync(FULL, m.is_long);
    huges[j] = __ballot_sync(FULL, m.is_huge);
    sum += (unsigned long long)__popc(starts[j]) << 30 | (unsigned long long)__popc(heads[j]);
  }
  if (lane == 0) s_warp[warp] = sum;
  __syncthreads();
  unsigned long long before = 0ull, total = 0ull;
#pragma unroll
  for (int w = 0; w < WARPS; ++w) {
    if (w < warp) before += s_warp[w];
    total += s_warp[w];
  }
  if (warp == 0) {
    unsigned long long prefix = 0ull;
    if (lane == 0) st_relaxed_u64(a.status + tile, (tile == 0 ? SCAN_INCL : SCAN_AGG) | total);
    if (tile > 0) {
      int64_t j = (int64_t)tile - 1 - lane;
      const uint64_t t0 = globaltimer_ns();
      for (;;) {
        const unsigned long long v = j >= 0 ? ld_relaxed_u64(a.status + j) : SCAN_INCL;
        const uint32_t incl = __ballot_sync(FULL, (v & SCAN_INCL) != 0ull);
        const uint32_t ready = __ballot_sync(FULL, v >> 60 != 0ull);
        const uint32_t used = incl ? (incl & (0u - incl)) * 2u - 1u : FULL;  // up to the nearest inclusive one
        if ((ready & used) == used) {
          unsigned long long x = used >> lane & 1u ? v & SCAN_VALUE : 0ull;
#pragma unroll
          for (int o = 16; o > 0; o >>= 1) x += __shfl_xor_sync(FULL, x, o);
          prefix += x;
          if (incl) break;
          j -= 32;
          continue;
        }
        const bool give_up = (int64_t)(globaltimer_ns() - t0) > wait_ns;
        if (__any_sync(FULL, give_up)) {
          if (lane == 0) raise_error(err, ERR_TIMEOUT);
          break;
        }
        __nanosleep(LOOKBACK_SLEEP_NS);
      }
      if (lane == 0) st_relaxed_u64(a.status + tile, SCAN_INCL | ((prefix + total) & SCAN_VALUE));
    }
    if (lane == 0) {
      s_prefix = prefix;
      if (tile + 1 == gridDim.x) {
        a.ctr->n_items = (uint32_t)((prefix + total) >> 30) & 0x3FFFFFFFu;
        a.ctr->n_runs = (uint32_t)(prefix + total) & 0x3FFFFFFFu;
      }
    }
  }
  __syncthreads();
  before += s_prefix;
  uint32_t item = (uint32_t)(before >> 30) & 0x3FFFFFFFu, run = (uint32_t)before & 0x3FFFFFFFu;
  const uint32_t lt = lanemask_lt();
#pragma unroll
  for (int j = 0; j < ROUNDS; ++j) {
    const uint32_t p = base + (uint32_t)(j * 32 + lane);
    const uint32_t me = 1u << lane;
    const uint32_t at = item + __popc(starts[j] & lt);
    const uint32_t r = run + __popc(heads[j] & (lt | me)) - 1u;  // the run p belongs to
    if ((starts[j] & me) && at < a.n && r < a.n)  // the bounds hold unless a wait gave up
      write_item(a, p, key[j], at, r, (heads[j] & me) != 0u, (several[j] & me) != 0u, (firsts[j] & me) != 0u,
                 (longs[j] & me) != 0u, (huges[j] & me) != 0u);
    item += __popc(starts[j]);
    run += __popc(heads[j]);
  }
}

// ---- gradient: keys, sort and items of a small call, by one cluster or block -------------------
// The same passes over digits as the larger sort, with the keys in the shared memory of
// eight blocks: a warp ranks its keys among equal digits, the blocks tell each other their
// counts and send the keys to their places.  One launch instead of five or six whose work is a
// few microseconds: whole calls of 1,000, 4,000 and 8,000 tokens x 64 floats take 14.5, 17.2 and
// 22.0 us by a cluster and 20.5, 25.9 and 27.4 the other way; with four keys a thread, which are
// not built, 16,000 took 29.9 against 29.5.  So it is for up to 8,192.  Up to 1,024 tokens one block does it without the cluster's barriers (30, 500 and 1,000
// tokens 7.0, 10.7 and 12.4 us, by a cluster 11.1, 14.6 and 15.5; 6,656 keys would take it 30 us:
// match.any gives an SM about one key every two cycles).
constexpr int CL_BLOCKS = 8, CL_THREADS = 512, CL_WARPS = CL_THREADS / 32;
constexpr int CL_RADIX = 512;  // a digit for each thread
static_assert(CL_RADIX == CL_THREADS && 2 * CL_BLOCKS * CL_THREADS == SMALL_N, "");

template <int I, int BLOCKS>  // keys a thread, blocks
__global__ void __cluster_dims__(BLOCKS, 1, 1) __launch_bounds__(CL_THREADS)
    k_token_small(KeyArgs ka, SortPlan plan, ItemArgs a, uint32_t* sorted, uint32_t* order, ErrSink err) {
  constexpr int PER = CL_THREADS * I;  // a block's
  __shared__ uint32_t s_keys[PER];
  __shared__ uint16_t s_vals[PER];
  __shared__ uint16_t s_cnt[CL_WARPS][CL_RADIX];  // per warp: counts, then offsets among equal digits
  __shared__ uint32_t s_all[BLOCKS][CL_RADIX];  // every block's counts of the pass
  __shared__ uint32_t s_place[CL_RADIX];           // where this block's keys of a digit go
  __shared__ uint32_t s_scan[CL_RADIX / 32];
  __shared__ unsigned long long s_warp[CL_WARPS];
  __shared__ unsigned long long s_sums[BLOCKS];
  __shared__ uint32_t s_bad[BLOCKS];
  follow();
  const int me = BLOCKS == 1 ? 0 : (int)cg::this_cluster().block_rank();
  auto sync = [] {
    if constexpr (BLOCKS == 1)
      __syncthreads();
    else
      cg::this_cluster().sync();
  };
  auto of_block = [](auto* p, uint32_t b) {  // p of block b
    if constexpr (BLOCKS == 1)
      return p;
    else
      return cg::this_cluster().map_shared_rank(p, b);
  };
  const int tid = threadIdx.x, lane = tid & 31, warp = tid >> 5;
  const uint32_t at = (uint32_t)(warp * 32 * I + lane), base = (uint32_t)(me * PER), lt = lanemask_lt();
  uint32_t key[I], val[I];
  bool bad = false;
#pragma unroll
  for (int j = 0; j < I; ++j) {
    const uint32_t p = base + at + j * 32;
    key[j] = p < ka.n ? key_of(ka, ka.ids[p], bad) : ~0u;  // the rest ranks behind every key
    val[j] = p;
  }
  if (me == 0 && tid == 0) *a.ctr = Counters{};
  if (a.present)
    for (int64_t i = base / I + tid; i < (ka.V + 31) / 32; i += BLOCKS * CL_THREADS) a.present[i] = 0u;
  for (int64_t i = base / I + tid; i < a.n_huge_done; i += BLOCKS * CL_THREADS) a.huge_done[i] = 0u;
  const int any_bad = __syncthreads_or(bad);
  sync();  // every block has started: its shared memory may be written
  if (tid < BLOCKS) of_block(s_bad, tid)[me] = any_bad ? 1u : 0u;

  for (int pass = 0; pass < plan.passes; ++pass) {
    const int shift = plan.shift[pass];
    const uint32_t mask = plan.mask[pass];
    for (int i = tid; i < CL_WARPS * CL_RADIX / 2; i += CL_THREADS) reinterpret_cast<uint32_t*>(s_cnt)[i] = 0u;
    __syncthreads();
    uint32_t rank[I];
#pragma unroll
    for (int j = 0; j < I; ++j) {
      const uint32_t d = (key[j] >> shift) & mask;
      const uint32_t peers = __match_any_sync(FULL, d);
      const uint32_t before = s_cnt[warp][d];
      rank[j] = before + __popc(peers & lt);
      __syncwarp();
      if ((peers & lt) == 0u) s_cnt[warp][d] = (uint16_t)(before + __popc(peers));
      __syncwarp();
    }
    __syncthreads();
    uint32_t own = 0u;
#pragma unroll
    for (int w = 0; w < CL_WARPS; ++w) {
      const uint32_t c = s_cnt[w][tid];
      s_cnt[w][tid] = (uint16_t)own;
      own += c;
    }
#pragma unroll
    for (int b = 0; b < BLOCKS; ++b) of_block(&s_all[me][tid], b)[0] = own;
    sync();  // and every block has read the keys of the pass before
    if (pass == 0) {  // the same answer in every block
      uint32_t failed = 0u;
      for (int b = 0; b < BLOCKS; ++b) failed |= s_bad[b];
      if (failed) {
        if (me == 0 && tid == 0) raise_error(err, ERR_ID_RANGE);
        return;
      }
    }
    uint32_t total = 0u, before_me = 0u;
#pragma unroll
    for (int b = 0; b < BLOCKS; ++b) {
      const uint32_t c = s_all[b][tid];
      if (b < me) before_me += c;
      total += c;
    }
    uint32_t incl = total;
#pragma unroll
    for (int o = 1; o < 32; o <<= 1) {
      const uint32_t y = __shfl_up_sync(FULL, incl, o);
      if (lane >= o) incl += y;
    }
    if (lane == 31) s_scan[warp] = incl;
    __syncthreads();
    uint32_t place = incl - total + before_me;
#pragma unroll
    for (int w = 0; w < CL_WARPS; ++w)
      if (w < warp) place += s_scan[w];
    s_place[tid] = place;
    __syncthreads();
#pragma unroll
    for (int j = 0; j < I; ++j) {
      const uint32_t d = (key[j] >> shift) & mask;
      const uint32_t pos = s_place[d] + s_cnt[warp][d] + rank[j];  // a permutation of 0 .. 8 PER - 1
      const uint32_t block = pos / PER, slot = pos % PER;
      of_block(s_keys, block)[slot] = key[j];
      of_block(s_vals, block)[slot] = (uint16_t)val[j];
    }
    sync();
#pragma unroll
    for (int j = 0; j < I; ++j) {
      key[j] = s_keys[at + j * 32];
      val[j] = s_vals[at + j * 32];
    }
  }
#pragma unroll
  for (int j = 0; j < I; ++j) {
    const uint32_t p = base + at + j * 32;
    if (p < a.n) {
      sorted[p] = key[j];
      order[p] = val[j];
    }
  }
  sync();  // the marks look at other blocks' keys
  Marks m[I];
  unsigned long long sum = 0ull;
#pragma unroll
  for (int j = 0; j < I; ++j) {
    const uint32_t p = base + at + j * 32;
    m[j] = Marks{};
    if (p < a.n) m[j] = marks_of(a, sorted, p, key[j]);
    if (m[j].last) a.ctr->P = p + 1;
    sum += (unsigned long long)__popc(__ballot_sync(FULL, m[j].start)) << 30 |
           (unsigned long long)__popc(__ballot_sync(FULL, m[j].head));
  }
  if (lane == 0) s_warp[warp] = sum;
  __syncthreads();
  unsigned long long before = 0ull, mine = 0ull;
#pragma unroll
  for (int w = 0; w < CL_WARPS; ++w) {
    if (w < warp) before += s_warp[w];
    mine += s_warp[w];
  }
  if (tid < BLOCKS) of_block(s_sums, tid)[me] = mine;
  sync();
  unsigned long long all = 0ull;
#pragma unroll
  for (int b = 0; b < BLOCKS; ++b) {
    if (b < me) before += s_sums[b];
    all += s_sums[b];
  }
  if (me == 0 && tid == 0) {
    a.ctr->n_items = (uint32_t)(all >> 30);
    a.ctr->n_runs = (uint32_t)all & 0x3FFFFFFFu;
  }
  uint32_t item = (uint32_t)(before >> 30), run = (uint32_t)before & 0x3FFFFFFFu;
#pragma unroll
  for (int j = 0; j < I; ++j) {
    const uint32_t starts = __ballot_sync(FULL, m[j].start), heads = __ballot_sync(FULL, m[j].head);
    if (m[j].start)
      write_item(a, base + at + j * 32, key[j], item + __popc(starts & lt),
                 run + __popc(heads & (lt | 1u << lane)) - 1u, m[j].head, m[j].several, m[j].first_cut, m[j].is_long,
                 m[j].is_huge);
    item += __popc(starts);
    run += __popc(heads);
  }
}

// ---- gradient: sums ------------------------------------------------------------------------

struct SumArgs {
  const void* grad;
  int64_t stride;
  int32_t d;
  int32_t accumulate;
  float scale;
  uint32_t n;
  int32_t cut_lg;
  const uint32_t* order;
  Counters* ctr;
  const Item* items;
  const uint32_t* run_row;
  const uint32_t* run_start;
  const uint2* cuts;
  float* parts;
  float4* huge;         // sums of the blocks that share a run
  uint32_t* huge_done;  // how many of them are there
  int64_t* ids_out;  // message form: rows_out, n rows of d
  int64_t* n_out;
  float* out;
  int64_t out_stride;
  const uint32_t* present;  // dense form, overwriting
  int64_t V;
};

// Where run's sum goes, from column c on.
__device__ __forceinline__ float* sum_at(const SumArgs& a, uint32_t run, int64_t c) {
  return a.out + (uint64_t)(a.ids_out ? run : a.run_row[run]) * (uint64_t)a.out_stride + c;
}

template <int V>
__device__ __forceinline__ void write_sum(const SumArgs& a, float* dst, const float (&x)[V]) {
  float y[V] = {};
  Pack<float, V> o;
  if (a.accumulate) {
    o.load(dst);
    o.get(y);
  }
#pragma unroll
  for (int j = 0; j < V; ++j) y[j] = a.accumulate ? y[j] + x[j] * a.scale : x[j] * a.scale;
  o.set(y);
  o.store(dst);
}

template <Rows R>
constexpr int SUM_BLOCKS = R == EVEN ? 4 : 3;  // of k_token_sums, that an SM holds

// A lane group of 1 << lg lanes per item and slab of V columns a lane, the slabs of an item
// side by side.  A group takes every so-many-th item and adds its gradient rows in ascending
// order of their positions, U at a time; where the next U rows lie, of this item or the next
// one, is read while these arrive, since most rows of a table occur once or twice and their
// loads would wait for two others each time.  Warps that are done clear the message form's
// slots that no row needs, or the rows of the dense form that do not occur.  Of the latter
// they claim `claim` at a time: which warp clears a row changes no value, and it evens out
// what hot rows leave uneven (262,144 x 2048 bf16 into 131,072 rows, 2.08 GB: 427 us with equal
// shares, 376 to 404 with claims, 5.2 to 5.5 TB/s; what is left is rows read in no order
// beside rows written).
template <typename T, Rows R>
__global__ void __launch_bounds__(THREADS, SUM_BLOCKS<R>)
    k_token_sums(SumArgs a, int lg, int slabs, int claim, ErrSink err) {
  constexpr int U = 4, V = 16 / (int)sizeof(T);
  __shared__ __align__(16) float swap[R == LOOSE ? THREADS * V : 4];
  follow();
  const bool failed = *(const volatile uint32_t*)err.step != 0u;
  const uint32_t n_items = failed ? 0u : a.ctr->n_items, n_runs = failed ? 0u : a.ctr->n_runs, P = a.ctr->P;
  const int L = 1 << lg;
  const int l = threadIdx.x & (L - 1);
  const uint32_t group = (blockIdx.x * THREADS + threadIdx.x) >> lg;
  const uint32_t streams = ((gridDim.x * THREADS) >> lg) / slabs;
  const uint32_t stream = group / slabs, slab = group - stream * slabs;
  if (a.n_out && blockIdx.x == 0 && threadIdx.x == 0) *a.n_out = n_runs;
  const int64_t c = ((int64_t)slab * L + l) * V;
  const bool in = c < a.d;
  const T* grad = static_cast<const T*>(a.grad) + c;
  const char* lo = static_cast<const char*>(a.grad);
  const char* hi = lo + ((uint64_t)(a.n - 1) * (uint64_t)a.stride + (uint64_t)a.d) * sizeof(T);

  // the item being added, its positions [p, e), and the places of the next U of them
  uint32_t unit = stream < streams ? stream : n_items, p = 0, e = 0, next_e = 0;
  Item it{}, next{};
  auto item_at = [&](uint64_t u, Item& to, uint32_t& end) {
    end = 0;
    if (u >= n_items) return;
    to = a.items[u];
    end = u + 1 < n_items ? a.items[u + 1].start >> 1 : P;
  };
  item_at(unit, it, e);
  p = it.start >> 1;
  item_at((uint64_t)unit + streams, next, next_e);
  uint32_t at[U];
#pragma unroll
  for (int i = 0; i < U; ++i)
    if (p + i < e) at[i] = a.order[p + i];
  float x[V] = {};
  while (unit < n_items) {
    std::conditional_t<R != EVEN, Loose<T>, Pack<T, V>> g[U];
#pragma unroll
    for (int i = 0; i < U; ++i) {
      if (!in || p + i >= e) continue;
      const T* from = grad + (uint64_t)at[i] * (uint64_t)a.stride;
      if constexpr (R != EVEN)
        g[i].load(from, a.d - c, lo, hi);
      else
        g[i].load(from);
    }
    const uint32_t here = e - p;
    const bool more = here > (uint32_t)U;
    const uint32_t p1 = more ? p + U : next.start >> 1, e1 = more ? e : next_e;
#pragma unroll
    for (int i = 0; i < U; ++i)
      if (p1 + i < e1) at[i] = a.order[p1 + i];
    Item after = next;
    uint32_t after_e = next_e;
    if (!more) item_at((uint64_t)unit + 2ull * streams, after, after_e);
#pragma unroll
    for (int i = 0; i < U; ++i)
      if (in && (uint32_t)i < here) {
        float y[V];
        g[i].get(y);
#pragma unroll
        for (int j = 0; j < V; ++j) x[j] += y[j];
      }
    if (!more) {
      if (it.run & 1u) {
        // the item before the first cut, or the one that starts at a cut
        const uint32_t up = ((it.start >> 1) + (1u << a.cut_lg) - 1u) >> a.cut_lg;
        const uint32_t slot = it.start & 1u ? 2u * (up + 1u) : 2u * up + 1u;
        Pack<float, V> o;
        o.set(x);
        if (in) o.store(a.parts + (uint64_t)slot * part_stride(a.d) + c);
      } else if constexpr (R == LOOSE) {
        const int64_t group_column = c - l * V;
#pragma unroll
        for (int j = 0; j < V; ++j) x[j] *= a.scale;
        if (a.accumulate)
          write_in_order<float, V, true>(swap, x, lg, a.d - group_column, sum_at(a, it.run >> 1, group_column));
        else
          write_in_order<float, V, false>(swap, x, lg, a.d - group_column, sum_at(a, it.run >> 1, group_column));
      } else if (in) {
        write_sum<V>(a, sum_at(a, it.run >> 1, c), x);
      }
#pragma unroll
      for (int j = 0; j < V; ++j) x[j] = 0.f;
      it = next;
      next = after;
      next_e = after_e;
      unit = (uint64_t)unit + streams < n_items ? unit + streams : n_items;
    }
    p = p1;
    e = e1;
  }
  const uint64_t rest = a.ids_out ? a.n - n_runs : a.present ? (uint64_t)a.V : 0u;
  if (rest == 0) return;
  __syncwarp();
  const int lane = threadIdx.x & 31;
  constexpr int VZ = R == LOOSE ? 1 : V;
  const Pack<float, VZ> zero{};
  auto clear = [&](uint64_t row) {
    float* dst = a.out + row * (uint64_t)a.out_stride;
    for (int64_t q = (int64_t)l * VZ; q < a.d; q += L * VZ) zero.store(dst + q);
  };
  if (a.ids_out) {
    const int64_t id = n_runs > 0 ? (int64_t)a.run_row[n_runs - 1] : -1;
    for (uint64_t row = (uint64_t)n_runs + group; row < a.n; row += (gridDim.x * THREADS) >> lg) {
      if (l == 0) a.ids_out[row] = id;
      clear(row);
    }
    return;
  }
  for (;;) {
    uint32_t mine = 0;
    if (lane == 0) mine = atomicAdd(&a.ctr->rest, 1u);
    const uint64_t first = (uint64_t)__shfl_sync(FULL, mine, 0) * (uint64_t)claim;
    if (first >= rest) break;
    const uint64_t last = first + claim < rest ? first + claim : rest;
    for (uint64_t row = first; row < last; row = (row | 31u) + 1u) {  // those of one word of presence
      const uint32_t there = failed ? 0u : a.present[row >> 5] >> (row & 31u);
      const uint32_t rows = (uint32_t)min((uint64_t)(32u - (uint32_t)(row & 31u)), last - row);
      for (uint32_t i = lane >> lg; i < rows; i += 32u >> lg)
        if (!(there >> i & 1u)) clear(row + i);
    }
  }
}

// Adds the sums lo .. hi - 1 of a cut run's items to x, at columns c .. c + 3, in order.
// Compensated, so that a row of a million tokens is as exact as one of a hundred.
__device__ __forceinline__ void add_parts(const SumArgs& a, uint32_t first_cut, uint32_t lo, uint32_t hi, int64_t c,
                                          CSum (&x)[4]) {
  constexpr int U = 8;
  if (c >= a.d) return;
  for (uint32_t k = lo; k < hi; k += U) {
    Pack<float, 4> g[U];
#pragma unroll
    for (int i = 0; i < U; ++i) {
      const uint64_t slot = 2ull * (first_cut >> a.cut_lg) + (k + i == 0 ? 0u : 2u * (k + i) - 1u);
      if (k + i < hi) g[i].load(a.parts + slot * part_stride(a.d) + c);
    }
#pragma unroll
    for (int i = 0; i < U; ++i) {
      if (k + i >= hi) continue;
      float y[4];
      g[i].get(y);
#pragma unroll
      for (int j = 0; j < 4; ++j) csum_add(x[j], y[j]);
    }
  }
}

// hi is the plain sum.  Once that is an infinity its correction is a NaN (inf - inf), and the sum
// is what a run of one item gives: the infinity, or the NaN that hi has become since.
__device__ __forceinline__ float sum_value(const CSum& x) { return isfinite(x.hi) ? csum_value(x) : x.hi; }

// aligned: rows of the output start on 16 bytes and are whole numbers of them.
__device__ __forceinline__ void write_parts(const SumArgs& a, uint32_t run, int64_t c, const CSum (&x)[4],
                                            bool aligned) {
  if (c >= a.d) return;
  float* dst = sum_at(a, run, c);
  float y[4];
#pragma unroll
  for (int j = 0; j < 4; ++j) y[j] = sum_value(x[j]);
  if (aligned) {
    write_sum<4>(a, dst, y);
    return;
  }
#pragma unroll
  for (int j = 0; j < 4; ++j)
    if (c + j < a.d) dst[j] = a.accumulate ? dst[j] + y[j] * a.scale : y[j] * a.scale;
}

// Cut runs, in slabs of 128 columns: those of very many items by HUGE_SPLIT blocks each, whose
// warps add a share of the items' sums each and then the shares in order, and the last of
// which to finish adds the blocks' sums in order (58,000 tokens of one row in 3,600 items: 43 us
// by one block); those of many by a block each; then the others by a warp each.
__global__ void __launch_bounds__(MERGE_THREADS) k_token_merge(SumArgs a, int slabs, int aligned, ErrSink err) {
  constexpr int WARPS = MERGE_THREADS / 32;
  __shared__ float s_hi[WARPS][128], s_lo[WARPS][128];
  follow();
  if (*(const volatile uint32_t*)err.step != 0u) return;
  const uint32_t n_runs = a.ctr->n_runs, P = a.ctr->P, room = (a.n >> a.cut_lg) + 1u;
  const uint32_t n_short = a.ctr->n_cut[0], n_long = a.ctr->n_cut[1], n_huge = a.ctr->n_cut[2];
  const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
  // the items of a run: the one before the first cut, and one from each cut on
  auto parts_of = [&](const uint2& cut) {
    const uint32_t end = cut.x + 1 < n_runs ? a.run_start[cut.x + 1] : P;
    return 1u + ((end - cut.y + (1u << a.cut_lg) - 1u) >> a.cut_lg);
  };
  // this warp's share, the w-th of so many, of the sums of cut's run
  auto share = [&](const uint2& cut, int64_t c, int w, int warps, CSum (&x)[4]) {
    const uint32_t parts = parts_of(cut), each = (parts + warps - 1) / warps;
    const uint32_t lo = min(parts, w * each), hi = min(parts, lo + each);
    add_parts(a, cut.y, lo, hi, c, x);
#pragma unroll
    for (int j = 0; j < 4; ++j) {
      s_hi[warp][lane * 4 + j] = x[j].hi;
      s_lo[warp][lane * 4 + j] = x[j].lo;
    }
  };
  auto merge = [&](const float* hi, const float* lo, CSum (&x)[4]) {
#pragma unroll
    for (int j = 0; j < 4; ++j) csum_merge(x[j], hi[lane * 4 + j], lo[lane * 4 + j]);
  };
  for (uint64_t i = blockIdx.x; i < (uint64_t)n_huge * slabs * HUGE_SPLIT; i += gridDim.x) {
    const uint64_t unit = i / HUGE_SPLIT, part = i % HUGE_SPLIT;
    const uint2 cut = a.cuts[2 * room + unit / slabs];
    const int64_t c = (int64_t)(unit % slabs) * 128 + lane * 4;
    CSum x[4] = {};
    share(cut, c, (int)part * WARPS + warp, HUGE_SPLIT * WARPS, x);
    __syncthreads();
    if (warp == 0) {
      for (int w = 1; w < WARPS; ++w) merge(s_hi[w], s_lo[w], x);
      float4* out = a.huge + (unit * HUGE_SPLIT + part) * 64 + lane;  // of 32 lanes: hi, then lo
      out[0] = make_float4(x[0].hi, x[1].hi, x[2].hi, x[3].hi);
      out[32] = make_float4(x[0].lo, x[1].lo, x[2].lo, x[3].lo);
      __threadfence();
      __syncwarp();
      uint32_t before = 0;
      if (lane == 0) before = atomicAdd(a.huge_done + unit, 1u);
      if (__shfl_sync(FULL, before, 0) + 1u == (uint32_t)HUGE_SPLIT) {
        __threadfence();
#pragma unroll
        for (int j = 0; j < 4; ++j) x[j] = CSum{0.f, 0.f};
        for (int q = 0; q < HUGE_SPLIT; ++q) {
          const float* in = reinterpret_cast<const float*>(a.huge + (unit * HUGE_SPLIT + q) * 64 + lane);
#pragma unroll
          for (int j = 0; j < 4; ++j)
            csum_merge(x[j], *(const volatile float*)(in + j), *(const volatile float*)(in + 128 + j));
        }
        write_parts(a, cut.x, c, x, aligned);
      }
    }
    __syncthreads();
  }
  for (uint64_t i = blockIdx.x; i < (uint64_t)n_long * slabs; i += gridDim.x) {
    const uint2 cut = a.cuts[room + i / slabs];
    const int64_t c = (int64_t)(i % slabs) * 128 + lane * 4;
    CSum x[4] = {};
    share(cut, c, warp, WARPS, x);
    __syncthreads();
    if (warp == 0) {
      for (int w = 1; w < WARPS; ++w) merge(s_hi[w], s_lo[w], x);
      write_parts(a, cut.x, c, x, aligned);
    }
    __syncthreads();
  }
  for (uint64_t i = (uint64_t)blockIdx.x * WARPS + warp; i < (uint64_t)n_short * slabs;
       i += (uint64_t)gridDim.x * WARPS) {
    const uint2 cut = a.cuts[i / slabs];
    const int64_t c = (int64_t)(i % slabs) * 128 + lane * 4;
    CSum x[4] = {};
    add_parts(a, cut.y, 0u, parts_of(cut), c, x);
    write_parts(a, cut.x, c, x, aligned);
  }
}

template <typename T, Rows R>
cudaError_t sums_as(const SumArgs& a, ErrSink err, int num_sms, cudaStream_t s) {
  constexpr int V = 16 / (int)sizeof(T);
  const int64_t pieces = (a.d + V - 1) / V;
  int lg = 0;
  while ((1 << lg) < pieces && lg < 5) ++lg;
  const int64_t slabs = (pieces + (1 << lg) - 1) >> lg;
  const int64_t units = ((int64_t)a.n + (a.n >> a.cut_lg) + (a.present ? a.V : 0)) * slabs;
  const int64_t blocks = (units + (THREADS >> lg) - 1) / (THREADS >> lg);
  const int64_t least = (slabs + (THREADS >> lg) - 1) / (THREADS >> lg);  // that hold one item
  const int64_t grid = std::min(blocks, std::max<int64_t>(least, (int64_t)num_sms * SUM_BLOCKS<R>));
  // claims of up to 16 KB, of which every warp finds several
  int claim = 32 >> lg;
  while ((int64_t)claim * 2 * a.d * 4 <= 16384 && (int64_t)claim * 2 * 4 * grid * (THREADS / 32) <= a.V) claim *= 2;
  const cudaError_t e = launch_following(k_token_sums<T, R>, dim3((unsigned)grid), THREADS, 0, s, a, lg,
                                         (int)slabs, claim, err);
  if (e != cudaSuccess || a.n <= 1u << a.cut_lg) return e;  // no run can be cut
  const int64_t mslabs = (a.d + 127) / 128;
  const int64_t mblocks = ((a.n >> a.cut_lg) * mslabs + MERGE_THREADS / 32 - 1) / (MERGE_THREADS / 32);
  const int aligned = vector_of(4, a.out, a.out_stride, a.d, 4) == 4;
  return launch_following(k_token_merge, dim3((unsigned)std::min<int64_t>(mblocks, num_sms)),
                          MERGE_THREADS, 0, s, a, (int)mslabs, aligned, err);
}

template <typename T>
cudaError_t sums_type(const SumArgs& a, ErrSink err, int num_sms, cudaStream_t s) {
  constexpr int V = 16 / (int)sizeof(T);
  if (vector_of(V, a.out, a.out_stride, a.d, 4) != V) return sums_as<T, LOOSE>(a, err, num_sms, s);
  return vector_of(V, a.grad, a.stride, a.d, sizeof(T)) == V ? sums_as<T, EVEN>(a, err, num_sms, s)
                                                            : sums_as<T, LOOSE_IN>(a, err, num_sms, s);
}

}  // namespace

cudaError_t launch_embed(const EmbedArgs& a, int32_t type, int32_t out_type, int num_sms,
                         cudaStream_t s) {
  if (type == GBA_F32) {
    if (out_type == GBA_F32) return embed_types<float, float>(a, num_sms, s);
    if (out_type == GBA_BF16) return embed_types<float, bf16>(a, num_sms, s);
    return embed_types<float, f16>(a, num_sms, s);
  }
  if (type == GBA_BF16)
    return out_type == GBA_F32 ? embed_types<bf16, float>(a, num_sms, s)
                               : embed_types<bf16, bf16>(a, num_sms, s);
  return out_type == GBA_F32 ? embed_types<f16, float>(a, num_sms, s)
                             : embed_types<f16, f16>(a, num_sms, s);
}

size_t embed_grad_workspace(const EmbedGradArgs& a, size_t* step_word) {
  const GradPlan p = plan_of(a);
  *step_word = p.counters + offsetof(Counters, step);
  return p.bytes;
}

cudaError_t launch_embed_grad(const EmbedGradArgs& a, char* ws, int64_t wait_ns, int num_sms,
                              cudaStream_t s) {
  if (a.n == 0) {  // the dense form: nothing is added
    if (a.accumulate) return cudaSuccess;
    return a.dense_stride == a.d
               ? cudaMemsetAsync(a.dense, 0, (size_t)a.V * a.d * 4, s)
               : cudaMemset2DAsync(a.dense, (size_t)a.dense_stride * 4, 0, (size_t)a.d * 4, (size_t)a.V, s);
  }
  const GradPlan p = plan_of(a);
  auto at = [&](size_t o) { return reinterpret_cast<uint32_t*>(ws + o); };
  Counters* ctr = reinterpret_cast<Counters*>(ws + p.counters);
  const KeyArgs ka{a.ids, (uint32_t)a.n, a.id_mode, a.pad_id, a.V, a.mod_magic, at(p.hist), at(p.keys[0])};
  ItemArgs ia{nullptr, (uint32_t)a.n, (uint32_t)a.V, ctr, reinterpret_cast<unsigned long long*>(ws + p.scan_status),
              reinterpret_cast<Item*>(ws + p.items), at(p.run_row), at(p.run_start),
              reinterpret_cast<uint2*>(ws + p.cuts), a.ids_out,
              a.dense && !a.accumulate ? at(p.present) : nullptr, p.cut_lg, at(p.huge_done), p.n_huge_done};
  const uint32_t* order = nullptr;
  cudaError_t e;
  if (p.small) {
    order = at(p.vals[0]);
    ia.keys = at(p.keys[0]);
    const bool one = a.n <= 2 * CL_THREADS;
    auto kernel = a.n <= CL_THREADS               ? k_token_small<1, 1>
                  : one                           ? k_token_small<2, 1>
                  : a.n <= CL_BLOCKS * CL_THREADS ? k_token_small<1, CL_BLOCKS>
                                                  : k_token_small<2, CL_BLOCKS>;
    e = launch_following(kernel, dim3(one ? 1 : CL_BLOCKS), CL_THREADS, 0, s, ka, p.sort, ia, at(p.keys[0]), at(p.vals[0]),
                         a.err);
    if (e != cudaSuccess) return e;
  } else {
    const int64_t words = (int64_t)p.cleared / 16;
    e = launch_following(k_token_clear,
                         dim3((unsigned)std::min<int64_t>((words + THREADS - 1) / THREADS, num_sms * 4)), THREADS, 0,
                         s, reinterpret_cast<uint4*>(ws), words);
    if (e != cudaSuccess) return e;
    e = launch_following(k_token_keys, dim3((unsigned)std::min<int64_t>((a.n + 1023) / 1024, num_sms * 6)), THREADS,
                         0, s, ka, p.sort, a.err);
    if (e != cudaSuccess) return e;
    int in = 0;
    for (int i = 0; i < p.sort.passes; ++i, in ^= 1) {
      SortPass sp{};
      sp.N = (uint32_t)a.n;
      sp.hist = at(p.hist) + i * p.sort.radix;
      sp.ticket = &ctr->tickets[i];
      sp.keys_in = at(p.keys[in]);
      sp.vals_in = at(p.vals[in]);
      sp.keys_out = at(p.keys[in ^ 1]);
      sp.vals_out = at(p.vals[in ^ 1]);
      sp.status = reinterpret_cast<unsigned long long*>(ws + p.sort_status);
      sp.epoch = (uint32_t)i + 1u;
      launch_onesweep(p.sort, i, sp, a.err, wait_ns, s);
    }
    e = cudaGetLastError();
    if (e != cudaSuccess) return e;
    order = at(p.vals[in]);
    ia.keys = at(p.keys[in]);
    e = launch_following(k_token_items, dim3((unsigned)p.tiles), THREADS, 0, s, ia, a.err, wait_ns);
    if (e != cudaSuccess) return e;
  }
  SumArgs sa{};
  sa.grad = a.grad;
  sa.stride = a.stride;
  sa.d = a.d;
  sa.accumulate = a.accumulate;
  sa.scale = a.scale;
  sa.n = (uint32_t)a.n;
  sa.cut_lg = p.cut_lg;
  sa.order = order;
  sa.ctr = ctr;
  sa.items = ia.items;
  sa.run_row = ia.run_row;
  sa.run_start = ia.run_start;
  sa.cuts = ia.cuts;
  sa.parts = reinterpret_cast<float*>(ws + p.parts);
  sa.huge = reinterpret_cast<float4*>(ws + p.huge);
  sa.huge_done = at(p.huge_done);
  sa.ids_out = a.ids_out;
  sa.n_out = a.n_out;
  sa.out = a.dense ? a.dense : a.rows_out;
  sa.out_stride = a.dense ? a.dense_stride : a.d;
  sa.present = ia.present;
  sa.V = a.V;
  if (a.type == GBA_F32) return sums_type<float>(sa, a.err, num_sms, s);
  if (a.type == GBA_BF16) return sums_type<bf16>(sa, a.err, num_sms, s);
  return sums_type<f16>(sa, a.err, num_sms, s);
}

}  // namespace gba

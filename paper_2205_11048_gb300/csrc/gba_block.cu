// The C ABI of a block's operators with the checks of their arguments (include/gba.h).  The
// kernels are in gba_resnorm.cu, gba_scan.cu and gba_adamw.cu.
#include <cuda_runtime.h>

#include <cfloat>
#include <cmath>
#include <initializer_list>

#include "gba.h"
#include "gba_worker_handle.cuh"

using namespace gba;

namespace {

constexpr int64_t MAX_ROWS = (1ll << 30) - 1;
constexpr int64_t MAX_SEQUENCES = (1ll << 29) - 1;

Rows in_rows(const gba_matrix* m) { return m ? Rows{m->data, m->stride} : Rows{nullptr, 0}; }
OutRows out_rows(const gba_matrix* m) { return m ? OutRows{m->data, m->stride} : OutRows{nullptr, 0}; }

// Memory that a call reads or writes: rows of `row` bytes, `stride` bytes apart, of a matrix (0: bytes that follow
// one another), `bytes` from the first to the end of the last.
struct Range {
  const void* p;
  uint64_t bytes, row = 0, stride = 0;
};
Range range(const gba_matrix* m) {
  if (!m) return Range{nullptr, 0};
  const uint64_t b = type_bytes(m->type);
  return Range{m->data, span(m), m->cols * b, m->stride * b};
}

// Do the rows of two matrices lie beside one another's, as those of columns of a wider matrix do?
bool beside(const Range& a, const Range& b) {
  if (a.row == 0 || a.stride != b.stride || b.row == 0) return false;
  // where b's rows start from a's on, modulo the stride
  const uint64_t ahead = (uintptr_t)b.p >= (uintptr_t)a.p ? ((uintptr_t)b.p - (uintptr_t)a.p) % a.stride
                                                          : a.stride - 1 - ((uintptr_t)a.p - (uintptr_t)b.p - 1) % a.stride;
  return ahead >= a.row && ahead + b.row <= a.stride;
}

// Does out overlap one of the others?
bool meets(const Range& out, std::initializer_list<Range> others) {
  for (const Range& o : others)
    if (out.p && o.p && overlap(out.p, out.bytes, o.p, o.bytes) && !beside(out, o)) return true;
  return false;
}

// A matrix that must be there (or may be NULL), of the shape of x and one of two types.
const char* bad_like(const gba_matrix* m, const gba_matrix* x, int32_t type, int32_t other) {
  const char* bad = bad_matrix(m);
  if (bad) return bad;
  if (m->rows != x->rows || m->cols != x->cols) return "matrices of different shape";
  return m->type != type && m->type != other ? "a matrix of another type than it may have" : nullptr;
}

const char* bad_block(const gba_block* b, const gba_matrix* gate) {
  if (!b) return "the block is NULL";
  for (int32_t k : {b->post_norm, b->pre_norm})
    if (k != GBA_NORM_NONE && k != GBA_NORM_RMS && k != GBA_NORM_LAYER) return "unknown norm";
  if (b->gate < GBA_GATE_NONE || b->gate > GBA_GATE_SILU) return "unknown gate";
  if ((b->gate == GBA_GATE_NONE) != (gate == nullptr)) return "a gate without its kind, or a kind without its gate";
  for (const void* p : {b->post_weight, b->post_bias, b->pre_weight, b->pre_bias})
    if (const char* bad = bad_param(p, b->param_type)) return bad;
  if (b->pre_norm == GBA_NORM_NONE && (b->pre_weight || b->pre_bias)) return "parameters of a norm that is not taken";
  if (!(b->eps >= 0.f && std::isfinite(b->eps))) return "eps is negative or not finite";
  if (!std::isfinite(b->residual_scale) || !std::isfinite(b->block_scale)) return "a scale is not finite";
  return nullptr;
}

void set_block(ResNormArgs& a, const gba_block* b, const gba_matrix* x, const gba_matrix* gate) {
  a.x = in_rows(x);
  a.g = in_rows(gate);
  a.post_weight = b->post_weight;
  a.post_bias = b->post_bias;
  a.pre_weight = b->pre_weight;
  a.pre_bias = b->pre_bias;
  a.n = x->rows;
  a.d = x->cols;
  a.post = b->post_norm;
  a.pre = b->pre_norm;
  a.gate = b->gate;
  a.param_type = b->param_type;
  a.eps = b->eps;
  a.rscale = b->residual_scale;
  a.bscale = b->block_scale;
}

Range param_range(const void* p, int32_t type, int32_t d) { return {p, p ? (uint64_t)d * type_bytes(type) : 0}; }

const char* bad_scan(const gba_scan* s, const gba_matrix* x) {
  if (!s) return "the scan is NULL";
  if (s->decay != GBA_DECAY_SIGMOID && s->decay != GBA_DECAY_LOG) return "unknown decay";
  if (s->tied != 0 && s->tied != 1) return "tied is neither 0 nor 1";
  if (s->n_seq < 0 || s->n_seq > MAX_SEQUENCES) return "n_seq outside [0, 2^29)";
  if (x->rows > MAX_ROWS) return "2^30 rows or more";
  if (s->n_seq == 0 && x->rows > 0) return "rows without sequences";
  if (s->lengths && s->offsets) return "lengths and offsets";
  if ((uintptr_t)s->lengths % 8 != 0 || (uintptr_t)s->offsets % 8 != 0) return "lengths or offsets not 8-byte aligned";
  if (!s->offsets && s->n_seq > 0 && x->rows % s->n_seq != 0) return "rows is no multiple of n_seq";
  return nullptr;
}

// A matrix of states, or NULL.
const char* bad_state(const gba_matrix* m, const gba_scan* s, const gba_matrix* x) {
  if (!m) return nullptr;
  const char* bad = bad_matrix(m);
  if (bad) return bad;
  return m->type != GBA_F32 || m->rows != s->n_seq || m->cols != x->cols ? "states are n_seq x cols of float32"
                                                                          : nullptr;
}

bool same(const gba_matrix* a, const gba_matrix* b) { return a && b && a->data == b->data && a->stride == b->stride; }

void set_scan(ScanArgs& a, const gba_worker* w, const gba_scan* s, const gba_matrix* x, const gba_matrix* f) {
  a.x = in_rows(x);
  a.f = in_rows(f);
  a.lengths = s->lengths;
  a.offsets = s->offsets;
  a.n_seq = s->n_seq;
  a.n = x->rows;
  a.d = x->cols;
  a.decay = s->decay;
  a.tied = s->tied;
  a.err = w->sink;
}

gba_status run_scan(gba_worker* w, const ScanArgs& a, int32_t type, int32_t out_type, bool grad) {
  if (a.n == 0 && (a.n_seq == 0 || !(a.last || a.offsets || a.lengths))) return GBA_OK;
  const gba_status st = reserve(w, scan_workspace(a, type, out_type, grad, w->num_sms));
  if (st != GBA_OK) return st;
  const cudaError_t e = launch_scan(a, type, out_type, grad, w->ws, w->num_sms, w->stream);
  return e == cudaSuccess ? GBA_OK : cuda_fail(w, e, "launch the scan");
}

const char* bad_adamw_parts(const gba_adamw_part* parts, int32_t n_parts) {
  if (n_parts < 0 || n_parts > (1 << 20)) return "n_parts outside [0, 2^20]";
  if (n_parts > 0 && !parts) return "parts is NULL";
  for (int32_t i = 0; i < n_parts; ++i) {
    const gba_adamw_part& p = parts[i];
    if (p.n < 0 || p.n > (1ll << 40)) return "a part's n is out of range";
    if (p.bits != 32 && p.bits != 8) return "states have 32 or 8 bits";
    if (p.n == 0) continue;
    if (!p.m || !p.v) return "a part's m or v is NULL";
    if (p.bits == 32) {
      if ((uintptr_t)p.m % 4 != 0 || (uintptr_t)p.v % 4 != 0) return "a part's m or v is not 4-byte aligned";
      if (p.m_scale || p.v_scale) return "scales of states in 32 bits";
    } else if (!p.m_scale || !p.v_scale || (uintptr_t)p.m_scale % 4 != 0 || (uintptr_t)p.v_scale % 4 != 0) {
      return "a part's scales are NULL or not 4-byte aligned";
    }
  }
  return nullptr;
}

// The arrays of one part do not overlap; those of different parts are not looked at.
const char* bad_adamw_arrays(const gba_adamw_part& p) {
  if (p.n == 0) return nullptr;
  if (p.type < GBA_F32 || p.type > GBA_F16 || p.grad_type < GBA_F32 || p.grad_type > GBA_F16) return "unknown type";
  if (p.copy && (p.copy_type < GBA_F32 || p.copy_type > GBA_F16)) return "unknown type";
  if (!p.weight || !p.grad) return "a part's weight or grad is NULL";
  if ((uintptr_t)p.weight % type_bytes(p.type) != 0 || (uintptr_t)p.grad % type_bytes(p.grad_type) != 0 ||
      (p.copy && (uintptr_t)p.copy % type_bytes(p.copy_type) != 0))
    return "a part's weight, grad or copy is not aligned to its type";
  if (!(p.weight_decay >= 0.f && std::isfinite(p.weight_decay))) return "a weight decay is negative or not finite";
  const uint64_t n = (uint64_t)p.n, state = n * (p.bits / 8), scales = (n + 255) / 256 * 4;
  const Range at[] = {{p.weight, n * type_bytes(p.type)},
                      {p.grad, n * type_bytes(p.grad_type)},
                      {p.m, state},
                      {p.v, state},
                      {p.m_scale, p.m_scale ? scales : 0},
                      {p.v_scale, p.v_scale ? scales : 0},
                      {p.copy, p.copy ? n * type_bytes(p.copy_type) : 0}};
  for (const Range& a : at)
    for (const Range* b = at; b != &a; ++b)
      if (overlap(a.p, a.bytes, b->p, b->bytes)) return "arrays of a part overlap";
  return nullptr;
}

}  // namespace

extern "C" {

gba_status gba_residual_norm(gba_worker* w, const gba_block* b, const gba_matrix* x, const gba_matrix* residual,
                             const gba_matrix* gate, const gba_matrix* z, const gba_matrix* y, float* stats) {
  if (!w) return GBA_E_ARG;
  const char* bad = bad_matrix(x);
  if (!bad) bad = bad_block(b, gate);
  if (!bad && residual) bad = bad_like(residual, x, x->type, GBA_F32);
  if (!bad && gate) bad = bad_like(gate, x, x->type, x->type);
  if (!bad && z) bad = residual ? bad_like(z, x, residual->type, residual->type) : bad_like(z, x, x->type, GBA_F32);
  if (!bad && y) bad = bad_like(y, x, x->type, x->type);
  if (!bad && (b->pre_norm == GBA_NORM_NONE) != (y == nullptr)) bad = "y without its norm, or a norm without y";
  if (!bad && !z && !y) bad = "neither z nor y";
  if (!bad && (uintptr_t)stats % 16 != 0) bad = "stats is not 16-byte aligned";
  if (!bad) {
    const Range st{stats, stats ? (uint64_t)x->rows * 16 : 0};
    const bool in_place = same(z, residual);
    if (meets(range(z), {range(x), range(gate), in_place ? Range{} : range(residual), range(y), st}) ||
        meets(range(y), {range(x), range(gate), range(residual), st}) ||
        meets(st, {range(x), range(gate), range(residual)}))
      bad = "an output overlaps an input or another output";
    for (const void* p : {b->post_weight, b->post_bias, b->pre_weight, b->pre_bias})
      if (!bad && (meets(range(z), {param_range(p, b->param_type, x->cols)}) ||
                   meets(range(y), {param_range(p, b->param_type, x->cols)}) ||
                   meets(st, {param_range(p, b->param_type, x->cols)})))
        bad = "an output overlaps a parameter";
  }
  if (bad) return fail(w, GBA_E_ARG, bad);
  if (x->rows == 0) return GBA_OK;
  const OnDevice on(w->device);
  ResNormArgs a{};
  set_block(a, b, x, gate);
  a.r = in_rows(residual);
  a.z = out_rows(z);
  a.y = out_rows(y);
  a.stats = reinterpret_cast<float4*>(stats);
  const int32_t wide = residual ? residual->type : z ? z->type : x->type;
  const cudaError_t e = launch_residual_norm(a, x->type, wide, w->num_sms, w->stream);
  return e == cudaSuccess ? GBA_OK : cuda_fail(w, e, "launch the block's norms");
}

gba_status gba_residual_norm_grad(gba_worker* w, const gba_block* b, const gba_matrix* dy, const gba_matrix* dz,
                                  const gba_matrix* x, const gba_matrix* z, const gba_matrix* gate,
                                  const float* stats, const gba_matrix* dx, const gba_matrix* dresidual,
                                  const gba_matrix* dgate, const gba_block_grads* grads) {
  if (!w) return GBA_E_ARG;
  const char* bad = bad_matrix(x);
  if (!bad) bad = bad_block(b, gate);
  if (!bad && gate) bad = bad_like(gate, x, x->type, x->type);
  if (!bad && ((gate == nullptr) != (dgate == nullptr))) bad = "dgate without its gate, or a gate without dgate";
  if (!bad && dgate) bad = bad_like(dgate, x, x->type, x->type);
  if (!bad) bad = bad_like(dx, x, x->type, x->type);
  const bool pre = !bad && b->pre_norm != GBA_NORM_NONE;
  if (!bad && (pre != (dy != nullptr) || pre != (z != nullptr))) bad = "dy and z go with the norm before the next block";
  if (!bad && !dy && !dz) bad = "neither dy nor dz";
  if (!bad && dy) bad = bad_like(dy, x, x->type, x->type);
  int32_t wide = GBA_F32;
  if (!bad) {
    const gba_matrix* const of = z ? z : dz;  // one of them is there
    bad = bad_like(of, x, x->type, GBA_F32);
    if (!bad) wide = of->type;
  }
  if (!bad && dz) bad = bad_like(dz, x, wide, wide);
  if (!bad && dresidual) bad = bad_like(dresidual, x, wide, wide);
  if (!bad && x->rows > 0 && !stats) bad = "stats is NULL";
  if (!bad && (uintptr_t)stats % 16 != 0) bad = "stats is not 16-byte aligned";
  const gba_block_grads none{};
  const gba_block_grads& g = grads ? *grads : none;
  float* const sums[4] = {g.post_weight, g.post_bias, g.pre_weight, g.pre_bias};
  for (const float* p : sums)
    if (!bad) bad = bad_floats(p);
  if (!bad && !pre && (sums[2] || sums[3])) bad = "gradients of a norm that is not taken";
  if (!bad) {
    const Range st{stats, stats ? (uint64_t)x->rows * 16 : 0};
    const bool in_place = same(dresidual, dz);
    const Range ins[] = {range(dy), range(x), range(z), range(gate), st,
                         param_range(b->post_weight, b->param_type, x->cols), param_range(b->post_bias, b->param_type, x->cols),
                         param_range(b->pre_weight, b->param_type, x->cols), range(dz)};
    Range outs[7] = {range(dx), range(dgate), range(dresidual)};
    for (int i = 0; i < 4; ++i) outs[3 + i] = Range{sums[i], sums[i] ? (uint64_t)x->cols * 4 : 0};
    for (int i = 0; i < 7; ++i) {
      for (int j = 0; j < i; ++j)
        if (meets(outs[i], {outs[j]})) bad = "an output overlaps another";
      for (const Range& in : ins)
        if (!(i == 2 && in_place && &in == &ins[8]) && meets(outs[i], {in})) bad = "an output overlaps an input";
    }
  }
  if (bad) return fail(w, GBA_E_ARG, bad);
  const OnDevice on(w->device);
  if (x->rows == 0) {
    for (float* p : sums) {
      const cudaError_t e = p ? cudaMemsetAsync(p, 0, (size_t)x->cols * 4, w->stream) : cudaSuccess;
      if (e != cudaSuccess) return cuda_fail(w, e, "clear the parameters' gradients");
    }
    return GBA_OK;
  }
  ResNormArgs a{};
  set_block(a, b, x, gate);
  a.dy = in_rows(dy);
  a.dz = in_rows(dz);
  a.zin = in_rows(z);
  a.dx = out_rows(dx);
  a.dr = out_rows(dresidual);
  a.dg = out_rows(dgate);
  a.stats = reinterpret_cast<float4*>(const_cast<float*>(stats));
  for (int i = 0; i < 4; ++i) a.sums[i] = sums[i];
  const gba_status st = reserve(w, residual_norm_grad_workspace(a, x->type, wide, w->num_sms));
  if (st != GBA_OK) return st;
  a.parts = reinterpret_cast<float*>(w->ws);
  const cudaError_t e = launch_residual_norm_grad(a, x->type, wide, w->num_sms, w->stream);
  return e == cudaSuccess ? GBA_OK : cuda_fail(w, e, "launch the gradient of the block's norms");
}

gba_status gba_gated_scan(gba_worker* w, const gba_scan* s, const gba_matrix* x, const gba_matrix* f,
                          const gba_matrix* state, const gba_matrix* y, const gba_matrix* state_out) {
  if (!w) return GBA_E_ARG;
  const char* bad = bad_matrix(x);
  if (!bad) bad = bad_scan(s, x);
  if (!bad) bad = bad_like(f, x, x->type, x->type);
  if (!bad) bad = bad_like(y, x, x->type, GBA_F32);
  if (!bad) bad = bad_state(state, s, x);
  if (!bad) bad = bad_state(state_out, s, x);
  if (!bad) {
    const Range lengths{s->lengths, s->lengths ? (uint64_t)s->n_seq * 8 : 0};
    const Range offsets{s->offsets, s->offsets ? (uint64_t)(s->n_seq + 1) * 8 : 0};
    if (meets(range(y), {range(x), range(f), range(state), range(state_out), lengths, offsets}) ||
        meets(range(state_out), {range(x), range(f), same(state, state_out) ? Range{} : range(state), lengths, offsets}))
      bad = "an output overlaps an input or another output";
  }
  if (bad) return fail(w, GBA_E_ARG, bad);
  const OnDevice on(w->device);
  ScanArgs a{};
  set_scan(a, w, s, x, f);
  a.out = out_rows(y);
  if (state) a.state = static_cast<const float*>(state->data), a.state_stride = state->stride;
  if (state_out) a.last = static_cast<float*>(state_out->data), a.last_stride = state_out->stride;
  return run_scan(w, a, x->type, y->type, false);
}

gba_status gba_gated_scan_grad(gba_worker* w, const gba_scan* s, const gba_matrix* dy, const gba_matrix* dstate_out,
                               const gba_matrix* x, const gba_matrix* f, const gba_matrix* state,
                               const gba_matrix* y, const gba_matrix* dx, const gba_matrix* df,
                               const gba_matrix* dstate) {
  if (!w) return GBA_E_ARG;
  const char* bad = bad_matrix(x);
  if (!bad) bad = bad_scan(s, x);
  if (!bad) bad = bad_like(f, x, x->type, x->type);
  if (!bad) bad = bad_like(y, x, x->type, GBA_F32);
  if (!bad) bad = bad_like(dy, x, y->type, y->type);
  if (!bad) bad = bad_like(dx, x, x->type, x->type);
  if (!bad) bad = bad_like(df, x, x->type, x->type);
  for (const gba_matrix* m : {dstate_out, state, dstate})
    if (!bad) bad = bad_state(m, s, x);
  if (!bad) {
    const Range lengths{s->lengths, s->lengths ? (uint64_t)s->n_seq * 8 : 0};
    const Range offsets{s->offsets, s->offsets ? (uint64_t)(s->n_seq + 1) * 8 : 0};
    const Range ds = same(dstate, dstate_out) ? Range{} : range(dstate_out);
    for (const gba_matrix* m : {dx, df, dstate})
      if (meets(range(m), {range(dy), range(x), range(f), range(state), range(y), lengths, offsets,
                           m == dstate ? ds : range(dstate_out)}))
        bad = "an output overlaps an input";
    if (meets(range(dx), {range(df), range(dstate)}) || meets(range(df), {range(dstate)}))
      bad = "an output overlaps another";
  }
  if (bad) return fail(w, GBA_E_ARG, bad);
  const OnDevice on(w->device);
  ScanArgs a{};
  set_scan(a, w, s, x, f);
  a.y = in_rows(y);
  a.dy = in_rows(dy);
  a.out = out_rows(dx);
  a.df = out_rows(df);
  if (dstate_out) a.state = static_cast<const float*>(dstate_out->data), a.state_stride = dstate_out->stride;
  if (state) a.h0 = static_cast<const float*>(state->data), a.h0_stride = state->stride;
  if (dstate) a.last = static_cast<float*>(dstate->data), a.last_stride = dstate->stride;
  return run_scan(w, a, x->type, y->type, true);
}

gba_status gba_adamw(gba_worker* w, const gba_adamw_part* parts, int32_t n_parts, const gba_adamw_desc* d,
                     int64_t* step) {
  if (!w) return GBA_E_ARG;
  const char* bad = bad_adamw_parts(parts, n_parts);
  for (int32_t i = 0; !bad && i < n_parts; ++i) bad = bad_adamw_arrays(parts[i]);
  if (!bad && !d) bad = "the description is NULL";
  if (!bad && !(d->lr >= 0.0 && std::isfinite((float)d->lr))) bad = "lr is negative or not finite";
  if (!bad && !(d->beta1 >= 0.0 && d->beta1 < 1.0 && d->beta2 >= 0.0 && d->beta2 < 1.0)) bad = "a beta outside [0, 1)";
  if (!bad && !((float)d->eps >= FLT_MIN && std::isfinite((float)d->eps))) bad = "eps is below 2^-126 or not finite";
  if (!bad && d->norm && !(d->max_norm >= 0.f)) bad = "max_norm is negative or NaN";
  if (!bad && d->rounding != GBA_ROUND_NEAREST && d->rounding != GBA_ROUND_CHANCE) bad = "unknown rounding";
  if (!bad) bad = bad_floats(d->norm);
  if (!bad) bad = bad_floats(d->lr_now);
  if (!bad && (!step || (uintptr_t)step % 8 != 0)) bad = "step is NULL or not 8-byte aligned";
  for (int32_t i = 0; !bad && i < n_parts; ++i) {
    const gba_adamw_part& p = parts[i];
    if (p.n == 0) continue;
    const uint64_t n = (uint64_t)p.n, state = n * (p.bits / 8), scales = p.bits == 8 ? (n + 255) / 256 * 4 : 0;
    const Range outs[] = {{p.weight, n * type_bytes(p.type)}, {p.m, state},        {p.v, state},
                          {p.m_scale, scales},                {p.v_scale, scales}, {p.copy, p.copy ? n * type_bytes(p.copy_type) : 0}};
    for (const Range& o : outs)
      if (meets(o, {Range{d->norm, 4}, Range{d->lr_now, 4}, Range{step, 8}})) bad = "a part overlaps norm, lr_now or step";
  }
  if (bad) return fail(w, GBA_E_ARG, bad);
  const OnDevice on(w->device);
  AdamWArgs a{};
  a.lr = (float)d->lr;
  a.beta1 = (float)d->beta1;
  a.beta2 = (float)d->beta2;
  a.rest1 = (float)(1.0 - d->beta1);
  a.rest2 = (float)(1.0 - d->beta2);
  a.eps = (float)d->eps;
  a.log1 = std::log(d->beta1);
  a.log2 = std::log(d->beta2);
  a.lr_now = d->lr_now;
  a.norm = d->norm;
  a.max_norm = d->max_norm;
  a.step = step;
  a.rounding = d->rounding;
  a.ticket = w->words + 1;
  const cudaError_t e = launch_adamw(parts, n_parts, a, w->num_sms, w->stream);
  return e == cudaSuccess ? GBA_OK : cuda_fail(w, e, "launch AdamW");
}

gba_status gba_adamw_values(gba_worker* w, const gba_adamw_part* parts, int32_t n_parts, float* const* m_out,
                            float* const* v_out) {
  if (!w) return GBA_E_ARG;
  const char* bad = bad_adamw_parts(parts, n_parts);
  if (!bad && n_parts > 0 && (!m_out || !v_out)) bad = "m_out or v_out is NULL";
  for (int32_t i = 0; !bad && i < n_parts; ++i) {
    const gba_adamw_part& p = parts[i];
    if (p.n == 0) continue;
    if (!m_out[i] || !v_out[i]) bad = "an output is NULL";
    if (!bad) bad = bad_floats(m_out[i]);
    if (!bad) bad = bad_floats(v_out[i]);
    const uint64_t n = (uint64_t)p.n, state = n * (p.bits / 8), scales = p.bits == 8 ? (n + 255) / 256 * 4 : 0;
    const Range m{m_out[i], n * 4}, v{v_out[i], n * 4};
    for (const Range& o : {m, v})
      if (!bad && meets(o, {Range{p.m, state}, Range{p.v, state}, Range{p.m_scale, scales}, Range{p.v_scale, scales}}))
        bad = "an output overlaps a state";
    if (!bad && meets(m, {v})) bad = "an output overlaps another";
  }
  if (bad) return fail(w, GBA_E_ARG, bad);
  const OnDevice on(w->device);
  const cudaError_t e = launch_adamw_values(parts, n_parts, m_out, v_out, w->num_sms, w->stream);
  return e == cudaSuccess ? GBA_OK : cuda_fail(w, e, "launch the reading of states");
}

}  // extern "C"

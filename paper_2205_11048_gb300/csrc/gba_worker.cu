// The worker handle, and the C ABI of lookups, norm and clipping and layer norm with the
// checks of their arguments (include/gba.h).  The kernels are in gba_embed.cu, gba_norm.cu
// and gba_layernorm.cu.
#include <cuda_runtime.h>

#include <cmath>
#include <new>

#include "gba.h"
#include "gba_worker_handle.cuh"

using namespace gba;

namespace {

constexpr int64_t MAX_TOKENS = (1ll << 30) - 1;
constexpr int64_t MAX_TABLE_ROWS = 0xFFFFFFFDll;  // keys are 32-bit; the next stands for padding, the last for none

const char* bad_ids(const int64_t* ids, int64_t n) {
  if (n < 0 || n > MAX_TOKENS) return "n outside [0, 2^30)";
  if (n > 0 && !ids) return "ids is NULL";
  if ((uintptr_t)ids % 8 != 0) return "ids not 8-byte aligned";
  return nullptr;
}

const char* bad_mode(int32_t id_mode, int64_t rows) {
  if (id_mode != GBA_ID_DIRECT && id_mode != GBA_ID_MODULO) return "id_mode is neither DIRECT nor MODULO";
  if (rows < 1 || rows > MAX_TABLE_ROWS) return "rows of the table outside [1, 2^32 - 3]";
  return nullptr;
}

gba_status run_embed(gba_worker* w, EmbedArgs& a, int32_t type, const int64_t* ids, int64_t n, float scale,
                     int64_t pad_id, const gba_matrix* out) {
  const char* bad = bad_matrix(out);
  if (!bad) bad = bad_ids(ids, n);
  if (!bad && (out->rows != n || out->cols != a.d)) bad = "out is not n x the table's width";
  if (!bad && overlap(ids, (uint64_t)n * 8, out->data, span(out))) bad = "out overlaps the ids";
  if (!bad && type != GBA_F32 && out->type != GBA_F32 && out->type != type)
    bad = "weights of 16 bits give their own type or float32";
  if (bad) return fail(w, GBA_E_ARG, bad);
  if (n == 0) return GBA_OK;
  a.ids = ids;
  a.n = n;
  a.pad_id = pad_id;
  a.scale = scale;
  a.out = out->data;
  a.out_stride = out->stride;
  a.err = w->sink;
  const cudaError_t e = launch_embed(a, type, out->type, w->num_sms, w->stream);
  return e == cudaSuccess ? GBA_OK : cuda_fail(w, e, "launch the lookup");
}

gba_status run_embed_grad(gba_worker* w, EmbedGradArgs& a) {
  size_t step_word = 0;
  const gba_status st = reserve(w, embed_grad_workspace(a, &step_word));
  if (st != GBA_OK) return st;
  a.err = w->sink;
  a.err.step = reinterpret_cast<uint32_t*>(w->ws + step_word);
  const cudaError_t e = launch_embed_grad(a, w->ws, WAIT_NS, w->num_sms, w->stream);
  return e == cudaSuccess ? GBA_OK : cuda_fail(w, e, "launch the lookup's gradient");
}

// norm: where clipping writes it (it reads the gradients again after that), or null
const char* bad_parts(const gba_grad_part* parts, int32_t n_parts, bool clip, const float* norm) {
  if (n_parts < 0 || n_parts > (1 << 20)) return "n_parts outside [0, 2^20]";
  if (n_parts > 0 && !parts) return "parts is NULL";
  for (int32_t i = 0; i < n_parts; ++i) {
    const gba_grad_part& p = parts[i];
    if (p.n < 0 || p.n > (1ll << 40)) return "a part's n is out of range";
    if (p.type < GBA_F32 || p.type > GBA_F16) return "unknown type";
    if (p.n == 0) continue;
    if (!p.grad) return "a part's grad is NULL";
    if ((uintptr_t)p.grad % type_bytes(p.type) != 0) return "a part's grad is not aligned to its type";
    if (!clip) continue;
    if (p.out_type < GBA_F32 || p.out_type > GBA_F16) return "unknown type";
    if (!p.out) return "a part's out is NULL";
    if ((uintptr_t)p.out % type_bytes(p.out_type) != 0) return "a part's out is not aligned to its type";
    if (norm && (overlap(norm, 4, p.grad, (uint64_t)p.n * type_bytes(p.type)) ||
                 overlap(norm, 4, p.out, (uint64_t)p.n * type_bytes(p.out_type))))
      return "norm overlaps a part";
    if (p.out == p.grad) {
      if (p.out_type != p.type) return "a part clipped in place keeps its type";
    } else if (overlap(p.grad, (uint64_t)p.n * type_bytes(p.type), p.out,
                       (uint64_t)p.n * type_bytes(p.out_type))) {
      return "a part's out overlaps its grad";
    }
  }
  return nullptr;
}

gba_status run_norm(gba_worker* w, const gba_grad_part* parts, int32_t n_parts, bool clip, float max_norm,
                    float* norm) {
  const gba_status st = reserve(w, norm_workspace(n_parts, w->num_sms));
  if (st != GBA_OK) return st;
  const cudaError_t e = launch_norm(parts, n_parts, clip, max_norm, norm, w->ws, w->words + 1,
                                    w->num_sms, w->stream);
  return e == cudaSuccess ? GBA_OK : cuda_fail(w, e, "launch the norm");
}

}  // namespace

extern "C" {

gba_status gba_worker_create(void* cuda_stream, gba_worker** out) {
  if (!out) return GBA_E_ARG;
  *out = nullptr;
  gba_worker* w = new (std::nothrow) gba_worker();
  if (!w) return GBA_E_OOM;
  auto give_up = [&](gba_status s) {
    cudaGetLastError();
    if (w->event) cudaEventDestroy(w->event);
    if (w->h_flag) cudaFreeHost(w->h_flag);
    cudaFree(w->words);
    delete w;
    return s;
  };
  if (cudaGetDevice(&w->device) != cudaSuccess) return give_up(GBA_E_CUDA);
  int sms = 0;
  if (cudaDeviceGetAttribute(&sms, cudaDevAttrMultiProcessorCount, w->device) == cudaSuccess && sms > 0)
    w->num_sms = sms;
  w->stream = (cudaStream_t)cuda_stream;
  if (cudaEventCreateWithFlags(&w->event, cudaEventDisableTiming) != cudaSuccess) return give_up(GBA_E_CUDA);
  if (cudaMalloc((void**)&w->words, 16) != cudaSuccess) return give_up(GBA_E_OOM);
  if (cudaHostAlloc((void**)&w->h_flag, 4, cudaHostAllocMapped) != cudaSuccess) return give_up(GBA_E_OOM);
  *w->h_flag = 0u;
  uint32_t* flag = nullptr;
  if (cudaHostGetDevicePointer((void**)&flag, w->h_flag, 0) != cudaSuccess ||
      cudaMemsetAsync(w->words, 0, 16, w->stream) != cudaSuccess)
    return give_up(GBA_E_CUDA);
  w->sink = ErrSink{w->words, w->words, flag};
  *out = w;
  return GBA_OK;
}

gba_status gba_worker_sync(gba_worker* w) {
  if (!w) return GBA_E_ARG;
  const OnDevice on(w->device);
  cudaError_t e = cudaStreamSynchronize(w->stream);
  if (e != cudaSuccess) return cuda_fail(w, e, "wait for the worker's stream");
  if (*(volatile uint32_t*)w->h_flag == 0u) return GBA_OK;
  uint32_t word = 0;
  e = cudaMemcpyAsync(&word, w->words, 4, cudaMemcpyDeviceToHost, w->stream);
  if (e == cudaSuccess) e = cudaMemsetAsync(w->words, 0, 4, w->stream);
  if (e == cudaSuccess) e = cudaStreamSynchronize(w->stream);
  if (e != cudaSuccess) return cuda_fail(w, e, "read the worker's error word");
  *(volatile uint32_t*)w->h_flag = 0u;
  if (word & ERR_ID_RANGE) return fail(w, GBA_E_ID_RANGE, "an id outside [0, rows), or a reserved one");
  if (word & ERR_SEQUENCES) return fail(w, GBA_E_ARG, "offsets or lengths of sequences out of order or range");
  if (word & ERR_TIMEOUT) return fail(w, GBA_E_DEVICE_TIMEOUT, "a bounded device wait gave up");
  return fail(w, GBA_E_CUDA, "device consistency check failed");
}

const char* gba_worker_last_error(gba_worker* w) { return w ? w->last_error : ""; }

void gba_worker_destroy(gba_worker* w) {
  if (!w) return;
  const OnDevice on(w->device);
  cudaStreamSynchronize(w->stream);
  for (int i = 0; i < w->n_old; ++i) cudaFree(w->old_ws[i]);
  cudaFree(w->ws);
  cudaFree(w->words);
  if (w->h_flag) cudaFreeHost(w->h_flag);
  if (w->event) cudaEventDestroy(w->event);
  delete w;
}

gba_status gba_embed(gba_worker* w, const gba_matrix* weights, int32_t id_mode, const int64_t* ids,
                     int64_t n, float scale, int64_t pad_id, const gba_matrix* out) {
  if (!w) return GBA_E_ARG;
  const char* bad = bad_matrix(weights);
  if (!bad) bad = bad_mode(id_mode, weights->rows);
  if (!bad) bad = bad_matrix(out);
  if (!bad && overlap(weights->data, span(weights), out->data, span(out))) bad = "out overlaps the weights";
  if (bad) return fail(w, GBA_E_ARG, bad);
  const OnDevice on(w->device);
  EmbedArgs a{};
  a.w = weights->data;
  a.w_stride = weights->stride;
  a.V = weights->rows;
  a.d = weights->cols;
  a.id_mode = id_mode;
  a.mod_magic = ~0ull / (uint64_t)weights->rows;
  return run_embed(w, a, weights->type, ids, n, scale, pad_id, out);
}

gba_status gba_embed_table(gba_worker* w, gba_handle* h, int32_t t, const int64_t* ids, int64_t n,
                           float scale, int64_t pad_id, const gba_matrix* out) {
  if (!w) return GBA_E_ARG;
  const OnDevice on(w->device);
  TableView v{};
  const gba_status st = table_view(h, t, &v);  // makes the server's device current
  if (st != GBA_OK || v.device != w->device) cudaSetDevice(w->device);
  if (st != GBA_OK) return fail(w, st, "no such table of a working handle");
  if (v.device != w->device) return fail(w, GBA_E_ARG, "the worker and the server are on different devices");
  EmbedArgs a{};
  a.w = v.w;
  a.w_stride = v.dim;
  a.V = v.rows;
  a.d = v.dim;
  a.id_mode = v.id_mode;
  a.mod_magic = v.mod_magic;
  a.hinfo = v.hinfo;
  const bool apart = v.stream != w->stream;
  if (apart) {
    cudaError_t e = cudaEventRecord(w->event, v.stream);
    if (e == cudaSuccess) e = cudaStreamWaitEvent(w->stream, w->event, 0);
    if (e != cudaSuccess) return cuda_fail(w, e, "order the lookup after the server's steps");
  }
  const gba_status r = run_embed(w, a, GBA_F32, ids, n, scale, pad_id, out);
  if (r == GBA_OK && apart) {
    cudaError_t e = cudaEventRecord(w->event, w->stream);
    if (e == cudaSuccess) e = cudaStreamWaitEvent(v.stream, w->event, 0);
    if (e != cudaSuccess) return cuda_fail(w, e, "order the server's steps after the lookup");
  }
  return r;
}

gba_status gba_embed_grad(gba_worker* w, const int64_t* ids, int64_t n, const gba_matrix* grad,
                          int64_t rows, int32_t id_mode, float scale, int64_t pad_id, int64_t* ids_out,
                          float* rows_out, int64_t* n_out) {
  if (!w) return GBA_E_ARG;
  const char* bad = bad_ids(ids, n);
  if (!bad) bad = bad_matrix(grad);
  if (!bad && grad->rows != n) bad = "grad has not n rows";
  if (!bad) bad = bad_mode(id_mode, rows);
  if (!bad && (!n_out || (uintptr_t)n_out % 8 != 0)) bad = "n_out is NULL or not 8-byte aligned";
  if (!bad && n > 0 && (!ids_out || !rows_out)) bad = "ids_out or rows_out is NULL";
  if (!bad && ((uintptr_t)ids_out % 8 != 0 || (uintptr_t)rows_out % 16 != 0))
    bad = "ids_out not 8-byte or rows_out not 16-byte aligned";
  if (!bad) {
    const struct {
      const void* p;
      uint64_t bytes;
    } at[] = {{ids, (uint64_t)n * 8}, {grad->data, span(grad)},  // the inputs, then the outputs
              {ids_out, (uint64_t)n * 8}, {rows_out, (uint64_t)n * grad->cols * 4}, {n_out, 8}};
    for (int i = 2; i < 5; ++i)
      for (int j = 0; j < i; ++j)
        if (overlap(at[i].p, at[i].bytes, at[j].p, at[j].bytes)) bad = "an output overlaps an input or another output";
  }
  if (bad) return fail(w, GBA_E_ARG, bad);
  const OnDevice on(w->device);
  if (n == 0) {
    const cudaError_t e = cudaMemsetAsync(n_out, 0, 8, w->stream);
    return e == cudaSuccess ? GBA_OK : cuda_fail(w, e, "clear n_out");
  }
  EmbedGradArgs a{};
  a.ids = ids;
  a.n = n;
  a.pad_id = pad_id;
  a.grad = grad->data;
  a.stride = grad->stride;
  a.type = grad->type;
  a.d = grad->cols;
  a.V = rows;
  a.mod_magic = ~0ull / (uint64_t)rows;
  a.id_mode = id_mode;
  a.scale = scale;
  a.ids_out = ids_out;
  a.rows_out = rows_out;
  a.n_out = n_out;
  return run_embed_grad(w, a);
}

gba_status gba_embed_grad_dense(gba_worker* w, const int64_t* ids, int64_t n, const gba_matrix* grad,
                                int32_t id_mode, float scale, int64_t pad_id, const gba_matrix* out,
                                int32_t accumulate) {
  if (!w) return GBA_E_ARG;
  const char* bad = bad_ids(ids, n);
  if (!bad) bad = bad_matrix(grad);
  if (!bad) bad = bad_matrix(out);
  if (!bad && grad->rows != n) bad = "grad has not n rows";
  if (!bad && (out->type != GBA_F32 || out->cols != grad->cols)) bad = "out is not float32 of grad's width";
  if (!bad) bad = bad_mode(id_mode, out->rows);
  if (!bad && accumulate != 0 && accumulate != 1) bad = "accumulate is neither 0 nor 1";
  if (!bad && (overlap(grad->data, span(grad), out->data, span(out)) ||
               overlap(ids, (uint64_t)n * 8, out->data, span(out))))
    bad = "an output overlaps an input";
  if (bad) return fail(w, GBA_E_ARG, bad);
  const OnDevice on(w->device);
  EmbedGradArgs a{};
  a.ids = ids;
  a.n = n;
  a.pad_id = pad_id;
  a.grad = grad->data;
  a.stride = grad->stride;
  a.type = grad->type;
  a.d = grad->cols;
  a.V = out->rows;
  a.mod_magic = ~0ull / (uint64_t)out->rows;
  a.id_mode = id_mode;
  a.scale = scale;
  a.dense = static_cast<float*>(out->data);
  a.dense_stride = out->stride;
  a.accumulate = accumulate;
  return run_embed_grad(w, a);
}

gba_status gba_grad_norm(gba_worker* w, const gba_grad_part* parts, int32_t n_parts, float* norm) {
  if (!w) return GBA_E_ARG;
  const char* bad = bad_parts(parts, n_parts, false, nullptr);
  if (!bad && !norm) bad = "norm is NULL";
  if (!bad) bad = bad_floats(norm);
  if (bad) return fail(w, GBA_E_ARG, bad);
  const OnDevice on(w->device);
  return run_norm(w, parts, n_parts, false, 0.f, norm);
}

gba_status gba_clip_grads(gba_worker* w, const gba_grad_part* parts, int32_t n_parts, float max_norm,
                          float* norm) {
  if (!w) return GBA_E_ARG;
  const char* bad = bad_parts(parts, n_parts, true, norm);
  if (!bad && !(max_norm >= 0.f)) bad = "max_norm is negative or NaN";
  if (!bad) bad = bad_floats(norm);
  if (bad) return fail(w, GBA_E_ARG, bad);
  const OnDevice on(w->device);
  return run_norm(w, parts, n_parts, true, max_norm, norm);
}

gba_status gba_layer_norm(gba_worker* w, const gba_matrix* x, const void* gamma, const void* beta,
                          int32_t param_type, float eps, const gba_matrix* y, float* mean, float* rstd) {
  if (!w) return GBA_E_ARG;
  const char* bad = bad_matrix(x);
  if (!bad) bad = bad_matrix(y);
  if (!bad) bad = not_alike(x, y);
  if (!bad) bad = not_apart(y, x);
  if (!bad) bad = bad_param(gamma, param_type);
  if (!bad) bad = bad_param(beta, param_type);
  if (!bad) bad = bad_floats(mean);
  if (!bad) bad = bad_floats(rstd);
  if (!bad && !(eps >= 0.f && std::isfinite(eps))) bad = "eps is negative or not finite";
  if (bad) return fail(w, GBA_E_ARG, bad);
  if (x->rows == 0) return GBA_OK;
  const OnDevice on(w->device);
  LayerNormArgs a{};
  a.x = x->data;
  a.x_stride = x->stride;
  a.gamma = gamma;
  a.beta = beta;
  a.y = y->data;
  a.y_stride = y->stride;
  a.mean = mean;
  a.rstd = rstd;
  a.n = x->rows;
  a.d = x->cols;
  a.param_type = param_type;
  a.eps = eps;
  const cudaError_t e = launch_layer_norm(a, x->type, RingWait{w->sink, WAIT_NS}, w->num_sms, w->stream);
  return e == cudaSuccess ? GBA_OK : cuda_fail(w, e, "launch the layer norm");
}

gba_status gba_layer_norm_grad(gba_worker* w, const gba_matrix* dy, const gba_matrix* x, const void* gamma,
                               int32_t param_type, const float* mean, const float* rstd,
                               const gba_matrix* dx, float* dgamma, float* dbeta) {
  if (!w) return GBA_E_ARG;
  const char* bad = bad_matrix(dy);
  if (!bad) bad = bad_matrix(x);
  if (!bad) bad = bad_matrix(dx);
  if (!bad) bad = not_alike(x, dy);
  if (!bad) bad = not_alike(x, dx);
  if (!bad && dx->rows > 0 && overlap(dx->data, span(dx), x->data, span(x))) bad = "dx overlaps x";
  if (!bad) bad = not_apart(dx, dy);
  if (!bad) bad = bad_param(gamma, param_type);
  if (!bad && x->rows > 0 && (!mean || !rstd)) bad = "mean or rstd is NULL";
  for (const float* p : {mean, rstd, (const float*)dgamma, (const float*)dbeta})
    if (!bad) bad = bad_floats(p);
  if (bad) return fail(w, GBA_E_ARG, bad);
  const OnDevice on(w->device);
  if (x->rows == 0) {
    for (float* p : {dgamma, dbeta}) {
      const cudaError_t e = p ? cudaMemsetAsync(p, 0, (size_t)x->cols * 4, w->stream) : cudaSuccess;
      if (e != cudaSuccess) return cuda_fail(w, e, "clear the weight's gradient");
    }
    return GBA_OK;
  }
  LayerNormArgs a{};
  a.x = x->data;
  a.x_stride = x->stride;
  a.gamma = gamma;
  a.y = dx->data;
  a.y_stride = dx->stride;
  a.dy = dy->data;
  a.dy_stride = dy->stride;
  a.mean = const_cast<float*>(mean);
  a.rstd = const_cast<float*>(rstd);
  a.dgamma = dgamma;
  a.dbeta = dbeta;
  a.n = x->rows;
  a.d = x->cols;
  a.param_type = param_type;
  const gba_status st = reserve(w, layer_norm_grad_workspace(a, x->type, w->num_sms));
  if (st != GBA_OK) return st;
  a.parts = reinterpret_cast<float*>(w->ws);
  const cudaError_t e = launch_layer_norm_grad(a, x->type, RingWait{w->sink, WAIT_NS}, w->num_sms,
                                               w->stream);
  return e == cudaSuccess ? GBA_OK : cuda_fail(w, e, "launch the layer norm's gradient");
}

}  // extern "C"

// Host side of the calls on the pass that g comes from: 4-bit products and their gradients, norms, distillation.  Arguments are
// checked here before anything is enqueued.
#include "pvt_distill.cuh"
#include "pvt_mx.cuh"
#include "pvt_norm.cuh"

using namespace pvt;

namespace {

int fail(cudaError_t e) {
  record_cuda_error(e);
  return PVT_ECUDA;
}
bool aligned(const void* p, size_t a) { return reinterpret_cast<uintptr_t>(p) % a == 0; }
bool known_type(int32_t t) { return t == PVT_F32 || t == PVT_F16 || t == PVT_BF16; }
size_t size_of(int32_t t) { return t == PVT_F32 ? 4 : 2; }
// rows x cols of a type, `ld` elements apart
bool matrix_ok(const void* p, int32_t type, int64_t ld, int64_t cols) {
  return p && known_type(type) && aligned(p, size_of(type)) && ld >= cols && ld < (int64_t)1 << 40;
}
// Spans of 256 columns are counted in 32 bits, a strip's rows that do not exist among them.
bool shape_ok(int32_t rows, int32_t cols) {
  return rows > 0 && cols > 0 &&
         (((uint64_t)rows + 127) / 128 * 128) * (((uint64_t)cols + mx::kSpan - 1) / mx::kSpan) < (uint64_t)1 << 31;
}
// log2(e) / temperature is a binary32 number
bool temperature_ok(float t) { return t > 0.0f && t <= 3.0e38f && 1.0f / t <= 2.0e38f; }
bool format_ok(int32_t f) { return f == PVT_MX_E8M0_32 || f == PVT_MX_E4M3_16; }

int check_mx(const pvt_mx* m) {
  if (!m || !shape_ok(m->rows, m->cols) || !format_ok(m->format)) return PVT_EINVAL;
  if (!m->codes || !m->scales || !aligned(m->codes, 16) || !aligned(m->scales, 16)) return PVT_EINVAL;
  if (m->ld % 16 != 0 || m->ld < ((int64_t)m->cols + 1) / 2 || m->ld >= (int64_t)1 << 40) return PVT_EINVAL;
  if (!aligned(m->tensor_scale, 4) || (m->format == PVT_MX_E8M0_32 && m->tensor_scale)) return PVT_EINVAL;
  return PVT_OK;
}
// the 16-bit gradient of a product's result, as the copy engine takes it
bool gradient_ok(const void* dy, int64_t lddy, int32_t tokens, int32_t n) {
  return dy && tokens > 0 && n > 0 && aligned(dy, 16) && lddy % 8 == 0 && lddy >= n && lddy < (int64_t)1 << 38;
}

int check_distill(const pvt_distill* d) {
  if (!d || d->rows < 1 || d->rows > 0x7fffffff || d->vocab < 1 || d->vocab > PVT_DISTILL_MAX_VOCAB) return PVT_EINVAL;
  if (d->k < 1 || d->k > PVT_DISTILL_MAX_K) return PVT_EINVAL;
  if (!matrix_ok(d->logits, d->dtype, d->ld, d->vocab)) return PVT_EINVAL;
  if (!temperature_ok(d->temperature)) return PVT_EINVAL;
  if (!d->top_idx || !d->top_logit || !aligned(d->top_idx, 4) || !aligned(d->top_logit, 4)) return PVT_EINVAL;
  return aligned(d->teacher_lse, 4) && aligned(d->weight, 4) ? PVT_OK : PVT_EINVAL;
}

// in place every element is written where it was read
bool in_place_ok(const pvt_distill* d, const void* grad, int32_t grad_dtype, int64_t ldg) {
  return grad != d->logits || (grad_dtype == d->dtype && (ldg == d->ld || d->rows == 1));
}

bool norm_shape_ok(const pvt_norm* n) { return n && n->rows >= 1 && n->rows <= 0x7fffffff && n->cols >= 1 && n->cols <= PVT_NORM_MAX_COLS; }
int check_norm(const pvt_norm* n) {
  if (!norm_shape_ok(n) || (n->kind != PVT_NORM_LAYER && n->kind != PVT_NORM_RMS)) return PVT_EINVAL;
  if (!matrix_ok(n->x, n->dtype, n->ldx, n->cols)) return PVT_EINVAL;
  if (n->residual && !matrix_ok(n->residual, n->dtype, n->ldr, n->cols)) return PVT_EINVAL;
  if (!known_type(n->weight_dtype) || !aligned(n->weight, size_of(n->weight_dtype)) || !aligned(n->bias, size_of(n->weight_dtype)))
    return PVT_EINVAL;
  return n->eps > 0.0f && n->eps <= 3.402823466e38f ? PVT_OK : PVT_EINVAL;
}
// a result in the place of an operand: every element is written where it was read
bool same_place_ok(const void* out, int32_t type, int64_t ld, const void* in, int32_t in_type, int64_t in_ld, int64_t rows) {
  return out != in || !in || (type == in_type && (ld == in_ld || rows == 1));
}

int check_gated(const pvt_mx* x, const pvt_mx* w_gate, const pvt_mx* w_up, int32_t activation) {
  for (const pvt_mx* m : {x, w_gate, w_up})
    if (const int rc = check_mx(m)) return rc;
  if (activation != PVT_ACT_SILU && activation != PVT_ACT_GELU && activation != PVT_ACT_GELU_TANH) return PVT_EINVAL;
  return x->format == w_gate->format && x->format == w_up->format && x->cols == w_gate->cols && x->cols == w_up->cols &&
                 w_gate->rows == w_up->rows
             ? PVT_OK
             : PVT_EINVAL;
}

}  // namespace

extern "C" {

size_t pvt_mx_scale_bytes(int32_t rows, int32_t cols, int32_t format) {
  return shape_ok(rows, cols) && format_ok(format) ? mx::scale_bytes(rows, cols, format) : 0;
}

int pvt_mx_quantize(const pvt_mx* m, const void* x, int32_t x_dtype, int64_t ldx, void* cuda_stream) {
  const int rc = check_mx(m);
  if (rc != PVT_OK) return rc;
  if (!matrix_ok(x, x_dtype, ldx, m->cols)) return PVT_EINVAL;
  const cudaError_t e = launch_mx_quantize(*m, x, x_dtype, ldx, device_sm_count(), static_cast<cudaStream_t>(cuda_stream));
  return e == cudaSuccess ? PVT_OK : fail(e);
}

int pvt_mx_dequant(const pvt_mx* m, void* values, int32_t out_dtype, int64_t ldv, void* cuda_stream) {
  const int rc = check_mx(m);
  if (rc != PVT_OK) return rc;
  if (!matrix_ok(values, out_dtype, ldv, m->cols)) return PVT_EINVAL;
  const cudaError_t e = launch_mx_dequant(*m, values, out_dtype, ldv, device_sm_count(), static_cast<cudaStream_t>(cuda_stream));
  return e == cudaSuccess ? PVT_OK : fail(e);
}

int pvt_mx_product(const pvt_mx* x, const pvt_mx* w, void* y, int32_t y_dtype, int64_t ldy, uint32_t* status, void* cuda_stream) {
  int rc = check_mx(x);
  if (rc == PVT_OK) rc = check_mx(w);
  if (rc != PVT_OK) return rc;
  if (x->format != w->format || x->cols != w->cols || !aligned(status, 4)) return PVT_EINVAL;
  if (!matrix_ok(y, y_dtype, ldy, w->rows)) return PVT_EINVAL;
  const cudaError_t e =
      launch_mx_product(*x, *w, y, y_dtype, ldy, status, device_sm_count(), static_cast<cudaStream_t>(cuda_stream));
  return e == cudaSuccess ? PVT_OK : fail(e);
}

int pvt_mx_grad_input(const void* dy, int64_t lddy, int32_t tokens, const pvt_mx* w, void* dx, int32_t dx_dtype, int64_t lddx,
                      uint32_t* status, void* cuda_stream) {
  const int rc = check_mx(w);
  if (rc != PVT_OK) return rc;
  if (!gradient_ok(dy, lddy, tokens, w->rows) || !aligned(status, 4)) return PVT_EINVAL;
  if (!matrix_ok(dx, dx_dtype, lddx, w->cols)) return PVT_EINVAL;
  const cudaError_t e = launch_mx_grad_input(dy, lddy, tokens, *w, dx, dx_dtype, lddx, status, device_sm_count(),
                                             static_cast<cudaStream_t>(cuda_stream));
  return e == cudaSuccess ? PVT_OK : fail(e);
}

int pvt_mx_grad_weight(const void* dy, int64_t lddy, int32_t n, const pvt_mx* x, float* dw, int64_t lddw, int32_t accumulate,
                       uint32_t* status, void* cuda_stream) {
  const int rc = check_mx(x);
  if (rc != PVT_OK) return rc;
  if (!gradient_ok(dy, lddy, x->rows, n) || !aligned(status, 4)) return PVT_EINVAL;
  if (!matrix_ok(dw, PVT_F32, lddw, x->cols)) return PVT_EINVAL;
  const cudaError_t e = launch_mx_grad_weight(dy, lddy, n, *x, dw, lddw, accumulate != 0, status, device_sm_count(),
                                              static_cast<cudaStream_t>(cuda_stream));
  return e == cudaSuccess ? PVT_OK : fail(e);
}

int pvt_mx_gated(const pvt_mx* x, const pvt_mx* w_gate, const pvt_mx* w_up, int32_t activation, void* h, int32_t h_dtype, int64_t ldh,
                 const pvt_mx* hq, uint32_t* status, void* cuda_stream) {
  int rc = check_gated(x, w_gate, w_up, activation);
  if (rc != PVT_OK) return rc;
  if ((!h && !hq) || !aligned(status, 4)) return PVT_EINVAL;
  if (h && !matrix_ok(h, h_dtype, ldh, w_gate->rows)) return PVT_EINVAL;
  if (hq && (rc = check_mx(hq)) != PVT_OK) return rc;
  if (hq && (hq->format != x->format || hq->rows != x->rows || hq->cols != w_gate->rows)) return PVT_EINVAL;
  const cudaError_t e = launch_mx_gated(*x, *w_gate, *w_up, activation, h, h ? h_dtype : PVT_F32, ldh, hq, status, device_sm_count(),
                                        static_cast<cudaStream_t>(cuda_stream));
  return e == cudaSuccess ? PVT_OK : fail(e);
}

int pvt_mx_gated_grad(const pvt_mx* x, const pvt_mx* w_gate, const pvt_mx* w_up, int32_t activation, const void* dh, int32_t dh_dtype,
                      int64_t lddh, void* dgate, void* dup, int64_t ldd, uint32_t* status, void* cuda_stream) {
  const int rc = check_gated(x, w_gate, w_up, activation);
  if (rc != PVT_OK) return rc;
  if (!matrix_ok(dh, dh_dtype, lddh, w_gate->rows) || !aligned(status, 4)) return PVT_EINVAL;
  if (!gradient_ok(dgate, ldd, x->rows, w_gate->rows) || !gradient_ok(dup, ldd, x->rows, w_gate->rows) || dgate == dup) return PVT_EINVAL;
  if (!same_place_ok(dgate, PVT_BF16, ldd, dh, dh_dtype, lddh, x->rows) || !same_place_ok(dup, PVT_BF16, ldd, dh, dh_dtype, lddh, x->rows))
    return PVT_EINVAL;
  const cudaError_t e = launch_mx_gated_grad(*x, *w_gate, *w_up, activation, dh, dh_dtype, lddh, dgate, dup, ldd, status,
                                             device_sm_count(), static_cast<cudaStream_t>(cuda_stream));
  return e == cudaSuccess ? PVT_OK : fail(e);
}

int pvt_mx_gated_grad_input(const void* dgate, const void* dup, int64_t ldd, int32_t tokens, const pvt_mx* w_gate, const pvt_mx* w_up,
                            void* dx, int32_t dx_dtype, int64_t lddx, uint32_t* status, void* cuda_stream) {
  int rc = check_mx(w_gate);
  if (rc == PVT_OK) rc = check_mx(w_up);
  if (rc != PVT_OK) return rc;
  if (w_gate->format != w_up->format || w_gate->rows != w_up->rows || w_gate->cols != w_up->cols) return PVT_EINVAL;
  if (w_gate->tensor_scale != w_up->tensor_scale) return PVT_EINVAL;  // one sum, one factor
  if (!gradient_ok(dgate, ldd, tokens, w_gate->rows) || !gradient_ok(dup, ldd, tokens, w_gate->rows) || !aligned(status, 4)) return PVT_EINVAL;
  if (!matrix_ok(dx, dx_dtype, lddx, w_gate->cols)) return PVT_EINVAL;
  const cudaError_t e = launch_mx_gated_grad_input(dgate, dup, ldd, tokens, *w_gate, *w_up, dx, dx_dtype, lddx, status, device_sm_count(),
                                                   static_cast<cudaStream_t>(cuda_stream));
  return e == cudaSuccess ? PVT_OK : fail(e);
}

int pvt_distill_top(const void* logits, int32_t dtype, int64_t ld, int64_t rows, int32_t vocab, int32_t k, float temperature,
                    int32_t* top_idx, float* top_logit, float* lse, void* cuda_stream) {
  if (rows < 1 || rows > 0x7fffffff || vocab < 1 || vocab > PVT_DISTILL_MAX_VOCAB) return PVT_EINVAL;
  if (k < 1 || k > PVT_DISTILL_MAX_K || k > vocab) return PVT_EINVAL;
  if (!matrix_ok(logits, dtype, ld, vocab)) return PVT_EINVAL;
  if (!temperature_ok(temperature)) return PVT_EINVAL;
  if (!top_idx || !top_logit || !aligned(top_idx, 4) || !aligned(top_logit, 4) || !aligned(lse, 4)) return PVT_EINVAL;
  const cudaError_t e = launch_distill_top(logits, dtype, ld, rows, vocab, k, temperature, top_idx, top_logit, lse,
                                           device_sm_count(), static_cast<cudaStream_t>(cuda_stream));
  return e == cudaSuccess ? PVT_OK : fail(e);
}

int pvt_distill_loss(const pvt_distill* d, float* loss, float* stats, const float* upstream, void* grad, int32_t grad_dtype,
                     int64_t ldg, uint32_t* status, void* cuda_stream) {
  const int rc = check_distill(d);
  if (rc != PVT_OK) return rc;
  if (!loss || !aligned(loss, 4) || !aligned(stats, 4) || !aligned(upstream, 4) || !aligned(status, 4)) return PVT_EINVAL;
  if (grad && !matrix_ok(grad, grad_dtype, ldg, d->vocab)) return PVT_EINVAL;
  if (!in_place_ok(d, grad, grad_dtype, ldg)) return PVT_EINVAL;
  const cudaError_t e = launch_distill_loss(*d, loss, stats, upstream, grad, grad_dtype, ldg, status, device_sm_count(),
                                            static_cast<cudaStream_t>(cuda_stream));
  return e == cudaSuccess ? PVT_OK : fail(e);
}

int pvt_distill_grad(const pvt_distill* d, const float* stats, const float* upstream, void* grad, int32_t grad_dtype, int64_t ldg,
                     uint32_t* status, void* cuda_stream) {
  const int rc = check_distill(d);
  if (rc != PVT_OK) return rc;
  if (!stats || !aligned(stats, 4) || !aligned(upstream, 4) || !aligned(status, 4)) return PVT_EINVAL;
  if (!matrix_ok(grad, grad_dtype, ldg, d->vocab)) return PVT_EINVAL;
  if (!in_place_ok(d, grad, grad_dtype, ldg)) return PVT_EINVAL;
  const cudaError_t e = launch_distill_grad(*d, stats, upstream, grad, grad_dtype, ldg, status, device_sm_count(),
                                            static_cast<cudaStream_t>(cuda_stream));
  return e == cudaSuccess ? PVT_OK : fail(e);
}

int pvt_norm_apply(const pvt_norm* n, void* total, int64_t ldt, void* y, int32_t y_dtype, int64_t ldy, const pvt_mx* yq, float* stats,
                   void* cuda_stream) {
  int rc = check_norm(n);
  if (rc != PVT_OK) return rc;
  if (!total && !y && !yq && !stats) return PVT_EINVAL;
  if (total && !matrix_ok(total, n->dtype, ldt, n->cols)) return PVT_EINVAL;
  if (y && !matrix_ok(y, y_dtype, ldy, n->cols)) return PVT_EINVAL;
  if (y && y == total) return PVT_EINVAL;
  if (yq && (rc = check_mx(yq)) != PVT_OK) return rc;
  if (yq && (yq->rows != n->rows || yq->cols != n->cols)) return PVT_EINVAL;
  if (!aligned(stats, 8)) return PVT_EINVAL;
  const struct {
    const void* p;
    int64_t ld;
  } operands[] = {{n->x, n->ldx}, {n->residual, n->ldr}};  // (which may be one another, of different distances)
  for (const auto& in : operands) {
    if (total && !same_place_ok(total, n->dtype, ldt, in.p, n->dtype, in.ld, n->rows)) return PVT_EINVAL;
    if (y && !same_place_ok(y, y_dtype, ldy, in.p, n->dtype, in.ld, n->rows)) return PVT_EINVAL;
  }
  const cudaError_t e = norm::launch_apply(*n, total, ldt, y, y ? y_dtype : PVT_F32, ldy, yq, stats, device_sm_count(),
                                           static_cast<cudaStream_t>(cuda_stream));
  return e == cudaSuccess ? PVT_OK : fail(e);
}

size_t pvt_norm_workspace_bytes(const pvt_norm* n) {
  return norm_shape_ok(n) ? norm::grad_workspace_bytes(n->rows, n->cols, device_sm_count()) : 0;
}

int pvt_norm_grad(const pvt_norm* n, const float* stats, int32_t dtype, const void* dy, int64_t lddy, const void* dresidual, int64_t lddr,
                  void* dx, int64_t lddx, void* dweight, void* dbias, int32_t dw_dtype, int32_t accumulate, void* ws, size_t ws_bytes,
                  void* cuda_stream) {
  const int rc = check_norm(n);
  if (rc != PVT_OK) return rc;
  if (n->residual || !stats || !aligned(stats, 8)) return PVT_EINVAL;
  if (!matrix_ok(dy, dtype, lddy, n->cols) || !matrix_ok(dx, dtype, lddx, n->cols)) return PVT_EINVAL;
  if (dresidual && !matrix_ok(dresidual, dtype, lddr, n->cols)) return PVT_EINVAL;
  if (!same_place_ok(dx, dtype, lddx, dy, dtype, lddy, n->rows) || !same_place_ok(dx, dtype, lddx, dresidual, dtype, lddr, n->rows) ||
      !same_place_ok(dx, dtype, lddx, n->x, n->dtype, n->ldx, n->rows))
    return PVT_EINVAL;
  if (dweight || dbias) {
    if (dw_dtype != PVT_F32 && dw_dtype != PVT_F64) return PVT_EINVAL;
    const size_t size = dw_dtype == PVT_F64 ? 8 : 4;
    if (!aligned(dweight, size) || !aligned(dbias, size) || dweight == dbias) return PVT_EINVAL;
    if (!ws || !aligned(ws, 256)) return PVT_EINVAL;
    if (ws_bytes < pvt_norm_workspace_bytes(n)) return PVT_EWORKSPACE;
  }
  const cudaError_t e =
      norm::launch_grad(*n, stats, dtype, dy, lddy, dresidual, lddr, dx, lddx, dweight, dbias, dw_dtype, accumulate != 0, ws,
                        device_sm_count(), static_cast<cudaStream_t>(cuda_stream));
  return e == cudaSuccess ? PVT_OK : fail(e);
}

}  // extern "C"

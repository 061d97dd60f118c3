// Host side of the calls on the pass that g comes from: 4-bit products and their gradients, distillation.  Arguments are
// checked here before anything is enqueued.
#include "pvt_distill.cuh"
#include "pvt_mx.cuh"

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

}  // extern "C"

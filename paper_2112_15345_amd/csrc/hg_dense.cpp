// C entry points of the dense operators (include/hg.h): argument checks on the
// host, then the launchers.  Nothing here allocates device memory or waits.
#include <cmath>
#include <cstdarg>
#include <cstdio>

#include "hg_dense.hpp"

using namespace hg;

namespace {

hg_status refuse(hg_status st, const char *fmt, ...) {
  char buf[512];
  va_list ap;
  va_start(ap, fmt);
  vsnprintf(buf, sizeof(buf), fmt, ap);
  va_end(ap);
  return set_error(st, buf);
}

constexpr int64_t kMost = int64_t(1) << 31;

bool is_float(int32_t dt) { return dt == HG_DT_F32 || dt == HG_DT_F16 || dt == HG_DT_BF16; }

#define HG_REQUIRE(cond, ...) \
  do {                        \
    if (!(cond)) return refuse(HG_EINVAL, __VA_ARGS__); \
  } while (0)

hg_status launched(hipError_t e, const char *what) {
  if (e == hipSuccess) return HG_OK;
  (void)hipGetLastError();
  return refuse(HG_EDEVICE, "%s: %s", what, hipGetErrorString(e));
}

// An input matrix: given, with a stride of 0 or more.
bool in_ok(const void *p, int64_t stride) { return p && stride >= 0; }
// An output matrix: given, with rows that do not overlap.
bool out_ok(const void *p, int64_t stride, int64_t cols) { return p && stride >= cols; }

// What another call left pending on this thread is not this call's error.
void clear_pending() { (void)hipGetLastError(); }

}  // namespace

extern "C" {

hg_status hg_rms_norm(const hg_norm_args *a, hipStream_t stream) {
  HG_REQUIRE(a, "hg_rms_norm: NULL arguments");
  HG_REQUIRE(a->rows >= 0 && a->dim >= 1, "hg_rms_norm: rows < 0 or dim < 1");
  HG_REQUIRE(is_float(a->dtype), "hg_rms_norm: type %d", a->dtype);
  HG_REQUIRE(a->out_dtype == a->dtype || a->out_dtype == HG_DT_E4M3, "hg_rms_norm: output type %d",
             a->out_dtype);
  HG_REQUIRE(a->weight_dtype == HG_DT_NONE || a->weight_dtype == HG_DT_F32 ||
                 a->weight_dtype == a->dtype,
             "hg_rms_norm: weight type %d", a->weight_dtype);
  HG_REQUIRE(a->eps >= 0.0f && std::isfinite(a->eps), "hg_rms_norm: eps is negative or not finite");
  if (a->rows >= kMost || a->dim >= kMost)
    return refuse(HG_EUNSUPPORTED, "hg_rms_norm: 2^31 rows or columns, or more");
  if (a->rows == 0) return HG_OK;
  HG_REQUIRE(in_ok(a->x, a->x_stride), "hg_rms_norm: x is NULL or its stride negative");
  HG_REQUIRE(!a->ids || a->x_rows >= 0, "hg_rms_norm: x_rows < 0");
  HG_REQUIRE(!a->residual || a->residual_stride >= 0, "hg_rms_norm: residual stride");
  HG_REQUIRE(a->weight_dtype == HG_DT_NONE || a->weight, "hg_rms_norm: weight is NULL");
  HG_REQUIRE(out_ok(a->y, a->y_stride, a->dim), "hg_rms_norm: y is NULL or its stride below dim");
  HG_REQUIRE(!a->sum || a->sum_stride >= a->dim, "hg_rms_norm: sum's stride below dim");
  HG_REQUIRE(a->out_dtype != HG_DT_E4M3 || a->scale, "hg_rms_norm: 8 bits need scale");
  clear_pending();
  return launched(launch_rms_norm(*a, stream), "hg_rms_norm");
}

int64_t hg_rms_norm_grad_workspace(int64_t rows, int64_t dim) {
  if (rows <= 0 || dim <= 0 || rows >= kMost || dim >= kMost) return 0;
  return rms_norm_grad_parts(rows) * dim * int64_t(sizeof(float));
}

hg_status hg_rms_norm_grad(const hg_norm_grad_args *a, hipStream_t stream) {
  HG_REQUIRE(a, "hg_rms_norm_grad: NULL arguments");
  HG_REQUIRE(a->rows >= 0 && a->dim >= 1, "hg_rms_norm_grad: rows < 0 or dim < 1");
  HG_REQUIRE(is_float(a->dtype), "hg_rms_norm_grad: type %d", a->dtype);
  HG_REQUIRE(a->weight_dtype == HG_DT_NONE || a->weight_dtype == HG_DT_F32 ||
                 a->weight_dtype == a->dtype,
             "hg_rms_norm_grad: weight type %d", a->weight_dtype);
  HG_REQUIRE(a->eps >= 0.0f && std::isfinite(a->eps),
             "hg_rms_norm_grad: eps is negative or not finite");
  if (a->rows >= kMost || a->dim >= kMost)
    return refuse(HG_EUNSUPPORTED, "hg_rms_norm_grad: 2^31 rows or columns, or more");
  if (!a->dx && !a->dweight) return HG_OK;
  if (a->rows > 0) {
    HG_REQUIRE(in_ok(a->x, a->x_stride), "hg_rms_norm_grad: x is NULL or its stride negative");
    HG_REQUIRE(!a->ids || a->x_rows >= 0, "hg_rms_norm_grad: x_rows < 0");
    HG_REQUIRE(in_ok(a->dy, a->dy_stride), "hg_rms_norm_grad: dy is NULL or its stride negative");
    HG_REQUIRE(!a->dsum || a->dsum_stride >= 0, "hg_rms_norm_grad: dsum stride");
    HG_REQUIRE(a->weight_dtype == HG_DT_NONE || a->weight, "hg_rms_norm_grad: weight is NULL");
    HG_REQUIRE(!a->dx || a->dx_stride >= a->dim, "hg_rms_norm_grad: dx stride below dim");
    HG_REQUIRE(!a->dweight || (a->workspace && a->workspace_bytes >=
                                                   hg_rms_norm_grad_workspace(a->rows, a->dim)),
               "hg_rms_norm_grad: workspace too small");
  }
  clear_pending();
  return launched(launch_rms_norm_grad(*a, stream), "hg_rms_norm_grad");
}

int64_t hg_linear_workspace(int64_t m, int64_t k, int64_t n, int32_t dtype) {
  if (m <= 0 || n <= 0 || k <= 0 || m >= kMost || n >= kMost || k >= kMost) return 0;
  return linear_workspace(m, k, n, dtype);
}

hg_status hg_linear(const hg_linear_args *a, hipStream_t stream) {
  HG_REQUIRE(a, "hg_linear: NULL arguments");
  HG_REQUIRE(a->m >= 0 && a->k >= 0 && a->n >= 0, "hg_linear: a negative size");
  HG_REQUIRE(is_float(a->dtype) || a->dtype == HG_DT_E4M3, "hg_linear: type %d", a->dtype);
  HG_REQUIRE(a->dtype == HG_DT_E4M3 ? is_float(a->out_dtype) : a->out_dtype == a->dtype,
             "hg_linear: output type %d with type %d", a->out_dtype, a->dtype);
  HG_REQUIRE(!a->bias || is_float(a->bias_dtype), "hg_linear: bias type %d", a->bias_dtype);
  HG_REQUIRE(a->act >= HG_ACT_NONE && a->act <= HG_ACT_SILU, "hg_linear: activation %d", a->act);
  if (a->m >= kMost || a->k >= kMost || a->n >= kMost)
    return refuse(HG_EUNSUPPORTED, "hg_linear: a size of 2^31 or more");
  if (a->m == 0 || a->n == 0) return HG_OK;
  HG_REQUIRE(a->k == 0 || (in_ok(a->x, a->x_stride) && in_ok(a->w, a->w_stride)),
             "hg_linear: x or w is NULL or its stride negative");
  HG_REQUIRE(a->dtype != HG_DT_E4M3 || (a->x_scale && a->w_scale), "hg_linear: 8 bits need scales");
  HG_REQUIRE(!a->residual || a->residual_stride >= 0, "hg_linear: residual stride");
  HG_REQUIRE(out_ok(a->y, a->y_stride, a->n), "hg_linear: y is NULL or its stride below n");
  HG_REQUIRE(!a->pre || a->pre_stride >= a->n, "hg_linear: pre's stride below n");
  const int64_t need = hg_linear_workspace(a->m, a->k, a->n, a->dtype);
  HG_REQUIRE(need == 0 || (a->workspace && a->workspace_bytes >= need),
             "hg_linear: workspace too small");
  clear_pending();
  return launched(launch_linear(*a, stream), "hg_linear");
}

int64_t hg_linear_grad_workspace(int64_t m, int64_t k, int64_t n, int32_t dtype, int32_t act) {
  if (m <= 0 || n <= 0 || k < 0 || m >= kMost || n >= kMost || k >= kMost) return 0;
  return linear_grad_workspace(m, k, n, dtype, act);
}

hg_status hg_linear_grad(const hg_linear_grad_args *a, hipStream_t stream) {
  HG_REQUIRE(a, "hg_linear_grad: NULL arguments");
  HG_REQUIRE(a->m >= 0 && a->k >= 0 && a->n >= 0, "hg_linear_grad: a negative size");
  HG_REQUIRE(is_float(a->dtype), "hg_linear_grad: type %d", a->dtype);
  HG_REQUIRE(!a->dw || a->dw_dtype == a->dtype || a->dw_dtype == HG_DT_F32,
             "hg_linear_grad: type %d of dw", a->dw_dtype);
  HG_REQUIRE(a->act >= HG_ACT_NONE && a->act <= HG_ACT_SILU, "hg_linear_grad: activation %d",
             a->act);
  if (a->m >= kMost || a->k >= kMost || a->n >= kMost)
    return refuse(HG_EUNSUPPORTED, "hg_linear_grad: a size of 2^31 or more");
  HG_REQUIRE(!a->dx || a->dx_stride >= a->k, "hg_linear_grad: dx's stride below k");
  HG_REQUIRE(!a->dw || a->dw_stride >= a->k, "hg_linear_grad: dw's stride below k");
  if (a->m > 0 && a->n > 0) {
    HG_REQUIRE(in_ok(a->dy, a->dy_stride), "hg_linear_grad: dy is NULL or its stride negative");
    HG_REQUIRE(a->act == HG_ACT_NONE || in_ok(a->pre, a->pre_stride),
               "hg_linear_grad: an activation needs pre");
    HG_REQUIRE(a->k == 0 || !a->dx || in_ok(a->w, a->w_stride),
               "hg_linear_grad: w is NULL or its stride negative");
    HG_REQUIRE(a->k == 0 || !a->dw || in_ok(a->x, a->x_stride),
               "hg_linear_grad: x is NULL or its stride negative");
    const int64_t need = hg_linear_grad_workspace(a->m, a->k, a->n, a->dtype, a->act);
    HG_REQUIRE(need == 0 || (a->workspace && a->workspace_bytes >= need),
               "hg_linear_grad: workspace too small");
  }
  clear_pending();
  return launched(launch_linear_grad(*a, stream), "hg_linear_grad");
}

hg_status hg_distill(const hg_distill_args *a, hipStream_t stream) {
  HG_REQUIRE(a, "hg_distill: NULL arguments");
  HG_REQUIRE(a->rows >= 0 && a->classes >= 1 && a->top >= 0,
             "hg_distill: rows < 0, classes < 1 or top < 0");
  HG_REQUIRE(is_float(a->dtype), "hg_distill: type %d", a->dtype);
  HG_REQUIRE(a->top == 0 || is_float(a->teacher_dtype), "hg_distill: teacher type %d",
             a->teacher_dtype);
  HG_REQUIRE(a->temperature > 0.0f && std::isfinite(a->temperature),
             "hg_distill: the temperature is not positive and finite");
  // (1 / temperature is not a float32 below)
  if (a->temperature < 0x1p-126f)
    return refuse(HG_EUNSUPPORTED, "hg_distill: a temperature below 2^-126");
  if (a->rows >= kMost || a->classes >= kMost)
    return refuse(HG_EUNSUPPORTED, "hg_distill: 2^31 rows or classes, or more");
  if (a->top > HG_MAX_TOP)
    return refuse(HG_EUNSUPPORTED, "hg_distill: more than %d listed classes", HG_MAX_TOP);
  if (a->rows == 0 || (!a->loss && !a->grad)) return HG_OK;
  HG_REQUIRE(in_ok(a->logits, a->logits_stride), "hg_distill: logits are NULL or their stride negative");
  HG_REQUIRE(a->top == 0 || (in_ok(a->ids, a->ids_stride) && in_ok(a->teacher, a->teacher_stride)),
             "hg_distill: ids or teacher is NULL or its stride negative");
  HG_REQUIRE(!a->grad || a->grad_stride >= a->classes, "hg_distill: grad's stride below classes");
  clear_pending();
  return launched(launch_distill(*a, stream), "hg_distill");
}

}  // extern "C"

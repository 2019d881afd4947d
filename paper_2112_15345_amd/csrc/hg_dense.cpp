// C entry points of the dense operators (include/hg.h): argument checks on the
// host, then the launchers.  Nothing here allocates device memory or waits.
#include <algorithm>
#include <cmath>
#include <cstdarg>
#include <cstdio>
#include <numeric>

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
// Products of integers of up to 2^14 each, whose sum is below 2^31.
constexpr int64_t kMostIntegers = (int64_t(1) << 17) - 1;

bool is_float(int32_t dt) { return dt == HG_DT_F32 || dt == HG_DT_F16 || dt == HG_DT_BF16; }

bool is_8_bits(int32_t dt) { return dt == HG_DT_E4M3 || dt == HG_DT_I8; }
// The type of a weight or bias over columns of `dtype`.
bool columns_ok(int32_t dt, int32_t dtype) {
  return dt == HG_DT_NONE || dt == HG_DT_F32 || dt == dtype;
}

bool group_ok(int32_t group) { return group == 0 || group == HG_KEPT_GROUP; }
Kept kept(const void *q, int64_t stride, const float *scale, int32_t group, int64_t cols) {
  Kept k;
  k.p = q;
  k.stride = stride;
  k.scale = scale;
  k.groups = group ? ceil_div<int64_t>(cols, group) : 1;
  return k;
}

// A matrix in memory: rows of `width` bytes, `step` bytes apart (0: one row, or one for all).
struct Span {
  uintptr_t at;
  int64_t rows, step, width;
};
Span span(const void *p, int64_t rows, int64_t stride, int64_t cols, int32_t dtype) {
  const int64_t size = size_of(dtype);
  // (a stride that no array has stays one)
  const int64_t step = rows > 1 ? std::min(stride, int64_t(1) << 58) * size : 0;
  return Span{reinterpret_cast<uintptr_t>(p), rows, step, cols * size};
}
// Whether two of them share memory: their extents meet, and so do the rows' places modulo the largest
// step that both steps are multiples of.  (Rows that would miss each other by their number alone count
// as sharing.)
bool share(const Span &a, const Span &b) {
  const auto end = [](const Span &s) {
    return __int128(s.at) + __int128(s.rows - 1) * s.step + s.width;
  };
  if (a.at >= end(b) || b.at >= end(a)) return false;
  const int64_t step = std::gcd(a.step, b.step);
  if (step == 0) return true;
  const int64_t off = int64_t(((__int128(b.at) - __int128(a.at)) % step + step) % step);
  return off < a.width || off + b.width > step;
}

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

hg_status hg_layer_norm(const hg_layer_norm_args *a, hipStream_t stream) {
  HG_REQUIRE(a, "hg_layer_norm: NULL arguments");
  HG_REQUIRE(a->rows >= 0 && a->dim >= 1, "hg_layer_norm: rows < 0 or dim < 1");
  HG_REQUIRE(is_float(a->dtype), "hg_layer_norm: type %d", a->dtype);
  HG_REQUIRE(a->out_dtype == a->dtype || is_8_bits(a->out_dtype), "hg_layer_norm: output type %d",
             a->out_dtype);
  HG_REQUIRE(columns_ok(a->weight_dtype, a->dtype), "hg_layer_norm: weight type %d",
             a->weight_dtype);
  HG_REQUIRE(columns_ok(a->bias_dtype, a->dtype), "hg_layer_norm: bias type %d", a->bias_dtype);
  HG_REQUIRE(a->eps >= 0.0f && std::isfinite(a->eps),
             "hg_layer_norm: eps is negative or not finite");
  if (a->rows >= kMost || a->dim >= kMost)
    return refuse(HG_EUNSUPPORTED, "hg_layer_norm: 2^31 rows or columns, or more");
  if (a->rows == 0) return HG_OK;
  HG_REQUIRE(in_ok(a->x, a->x_stride), "hg_layer_norm: x is NULL or its stride negative");
  HG_REQUIRE(!a->ids || a->x_rows >= 0, "hg_layer_norm: x_rows < 0");
  HG_REQUIRE(!a->residual || a->residual_stride >= 0, "hg_layer_norm: residual stride");
  HG_REQUIRE(a->weight_dtype == HG_DT_NONE || a->weight, "hg_layer_norm: weight is NULL");
  HG_REQUIRE(a->bias_dtype == HG_DT_NONE || a->bias, "hg_layer_norm: bias is NULL");
  HG_REQUIRE(out_ok(a->y, a->y_stride, a->dim), "hg_layer_norm: y is NULL or its stride below dim");
  HG_REQUIRE(!a->sum || a->sum_stride >= a->dim, "hg_layer_norm: sum's stride below dim");
  HG_REQUIRE(!is_8_bits(a->out_dtype) || a->scale, "hg_layer_norm: 8 bits need scale");
  clear_pending();
  return launched(launch_layer_norm(*a, stream), "hg_layer_norm");
}

int64_t hg_layer_norm_grad_workspace(int64_t rows, int64_t dim) {
  return 2 * hg_rms_norm_grad_workspace(rows, dim);
}

hg_status hg_layer_norm_grad(const hg_layer_norm_grad_args *a, hipStream_t stream) {
  HG_REQUIRE(a, "hg_layer_norm_grad: NULL arguments");
  HG_REQUIRE(a->rows >= 0 && a->dim >= 1, "hg_layer_norm_grad: rows < 0 or dim < 1");
  HG_REQUIRE(is_float(a->dtype), "hg_layer_norm_grad: type %d", a->dtype);
  HG_REQUIRE(columns_ok(a->weight_dtype, a->dtype), "hg_layer_norm_grad: weight type %d",
             a->weight_dtype);
  HG_REQUIRE(a->eps >= 0.0f && std::isfinite(a->eps),
             "hg_layer_norm_grad: eps is negative or not finite");
  if (a->rows >= kMost || a->dim >= kMost)
    return refuse(HG_EUNSUPPORTED, "hg_layer_norm_grad: 2^31 rows or columns, or more");
  if (!a->dx && !a->dweight && !a->dbias) return HG_OK;
  if (a->rows > 0) {
    HG_REQUIRE(in_ok(a->x, a->x_stride), "hg_layer_norm_grad: x is NULL or its stride negative");
    HG_REQUIRE(!a->ids || a->x_rows >= 0, "hg_layer_norm_grad: x_rows < 0");
    HG_REQUIRE(in_ok(a->dy, a->dy_stride), "hg_layer_norm_grad: dy is NULL or its stride negative");
    HG_REQUIRE(!a->dsum || a->dsum_stride >= 0, "hg_layer_norm_grad: dsum stride");
    HG_REQUIRE(a->weight_dtype == HG_DT_NONE || a->weight, "hg_layer_norm_grad: weight is NULL");
    HG_REQUIRE(!a->dx || a->dx_stride >= a->dim, "hg_layer_norm_grad: dx stride below dim");
    HG_REQUIRE((!a->dweight && !a->dbias) ||
                   (a->workspace &&
                    a->workspace_bytes >= hg_layer_norm_grad_workspace(a->rows, a->dim)),
               "hg_layer_norm_grad: workspace too small");
  }
  clear_pending();
  return launched(launch_layer_norm_grad(*a, stream), "hg_layer_norm_grad");
}

hg_status hg_embed(const hg_embed_args *a, hipStream_t stream) {
  HG_REQUIRE(a, "hg_embed: NULL arguments");
  HG_REQUIRE(a->n >= 0 && a->nodes >= 0 && a->dim >= 1, "hg_embed: n or nodes < 0, or dim < 1");
  HG_REQUIRE(is_float(a->table_dtype), "hg_embed: table type %d", a->table_dtype);
  HG_REQUIRE(is_float(a->out_dtype), "hg_embed: output type %d", a->out_dtype);
  HG_REQUIRE(std::isfinite(a->scale), "hg_embed: the scale is not finite");
  if (a->n >= kMost || a->nodes >= kMost || a->dim >= kMost)
    return refuse(HG_EUNSUPPORTED, "hg_embed: 2^31 ids, rows or columns, or more");
  if (a->n == 0) return HG_OK;
  HG_REQUIRE(a->nodes == 0 || in_ok(a->table, a->table_stride),
             "hg_embed: the table is NULL or its stride negative");
  HG_REQUIRE(a->ids, "hg_embed: ids are NULL");
  HG_REQUIRE(out_ok(a->y, a->y_stride, a->dim), "hg_embed: y is NULL or its stride below dim");
  clear_pending();
  return launched(launch_embed(*a, stream), "hg_embed");
}

int64_t hg_embed_grad_workspace(int64_t n, int64_t nodes, int64_t dim) {
  if (n <= 0 || nodes <= 0 || dim <= 0 || n >= kMost || nodes >= kMost || dim >= kMost) return 0;
  return embed_grad_workspace(n, nodes, dim);
}

hg_status hg_embed_grad(const hg_embed_grad_args *a, hipStream_t stream) {
  HG_REQUIRE(a, "hg_embed_grad: NULL arguments");
  HG_REQUIRE(a->n >= 0 && a->nodes >= 0 && a->dim >= 1,
             "hg_embed_grad: n or nodes < 0, or dim < 1");
  HG_REQUIRE(is_float(a->dtype), "hg_embed_grad: type %d", a->dtype);
  HG_REQUIRE(a->add == 0 || a->add == 1, "hg_embed_grad: add is neither 0 nor 1");
  HG_REQUIRE(a->out_dtype == HG_DT_F32 || (!a->add && a->out_dtype == a->dtype),
             "hg_embed_grad: output type %d", a->out_dtype);
  HG_REQUIRE(std::isfinite(a->scale), "hg_embed_grad: the scale is not finite");
  if (a->n >= kMost || a->nodes >= kMost || a->dim >= kMost)
    return refuse(HG_EUNSUPPORTED, "hg_embed_grad: 2^31 ids, rows or columns, or more");
  if (a->nodes == 0 || (a->n == 0 && a->add)) return HG_OK;
  HG_REQUIRE(out_ok(a->dtable, a->dtable_stride, a->dim),
             "hg_embed_grad: dtable is NULL or its stride below dim");
  if (a->n > 0) {
    HG_REQUIRE(in_ok(a->dy, a->dy_stride), "hg_embed_grad: dy is NULL or its stride negative");
    HG_REQUIRE(a->ids, "hg_embed_grad: ids are NULL");
    HG_REQUIRE(a->workspace && a->workspace_bytes >=
                                   hg_embed_grad_workspace(a->n, a->nodes, a->dim),
               "hg_embed_grad: workspace too small");
    HG_REQUIRE(!share(span(a->dy, a->n, a->dy_stride, a->dim, a->dtype),
                      span(a->dtable, a->nodes, a->dtable_stride, a->dim, a->out_dtype)),
               "hg_embed_grad: dy and dtable share memory");
  }
  clear_pending();
  return launched(launch_embed_grad(*a, stream), "hg_embed_grad");
}

hg_status hg_quantize(const hg_quantize_args *a, hipStream_t stream) {
  HG_REQUIRE(a, "hg_quantize: NULL arguments");
  HG_REQUIRE(a->rows >= 0 && a->dim >= 1, "hg_quantize: rows < 0 or dim < 1");
  HG_REQUIRE(is_float(a->dtype), "hg_quantize: type %d", a->dtype);
  HG_REQUIRE(group_ok(a->group), "hg_quantize: group %d", a->group);
  if (a->rows >= kMost || a->dim >= kMost)
    return refuse(HG_EUNSUPPORTED, "hg_quantize: 2^31 rows or columns, or more");
  if (a->rows == 0) return HG_OK;
  HG_REQUIRE(in_ok(a->x, a->x_stride), "hg_quantize: x is NULL or its stride negative");
  HG_REQUIRE(out_ok(a->q, a->q_stride, a->dim), "hg_quantize: q is NULL or its stride below dim");
  HG_REQUIRE(a->scale, "hg_quantize: scale is NULL");
  clear_pending();
  return launched(launch_quantize(*a, stream), "hg_quantize");
}

hg_status hg_dequantize(const hg_dequantize_args *a, hipStream_t stream) {
  HG_REQUIRE(a, "hg_dequantize: NULL arguments");
  HG_REQUIRE(a->rows >= 0 && a->dim >= 1, "hg_dequantize: rows < 0 or dim < 1");
  HG_REQUIRE(is_float(a->dtype), "hg_dequantize: type %d", a->dtype);
  HG_REQUIRE(group_ok(a->group), "hg_dequantize: group %d", a->group);
  if (a->rows >= kMost || a->dim >= kMost)
    return refuse(HG_EUNSUPPORTED, "hg_dequantize: 2^31 rows or columns, or more");
  if (a->rows == 0) return HG_OK;
  HG_REQUIRE(in_ok(a->q, a->q_stride), "hg_dequantize: q is NULL or its stride negative");
  HG_REQUIRE(a->scale, "hg_dequantize: scale is NULL");
  HG_REQUIRE(out_ok(a->x, a->x_stride, a->dim),
             "hg_dequantize: x is NULL or its stride below dim");
  clear_pending();
  return launched(launch_dequantize(kept(a->q, a->q_stride, a->scale, a->group, a->dim), a->rows,
                                    a->dim, a->dim, a->dtype, a->x, a->x_stride, false, stream),
                  "hg_dequantize");
}

int64_t hg_linear_workspace(int64_t m, int64_t k, int64_t n, int32_t dtype) {
  if (m <= 0 || n <= 0 || k <= 0 || m >= kMost || n >= kMost || k >= kMost) return 0;
  return linear_workspace(m, k, n, dtype);
}

hg_status hg_linear(const hg_linear_args *a, hipStream_t stream) {
  HG_REQUIRE(a, "hg_linear: NULL arguments");
  HG_REQUIRE(a->m >= 0 && a->k >= 0 && a->n >= 0, "hg_linear: a negative size");
  HG_REQUIRE(is_float(a->dtype) || is_8_bits(a->dtype), "hg_linear: type %d", a->dtype);
  HG_REQUIRE(is_8_bits(a->dtype) ? is_float(a->out_dtype) : a->out_dtype == a->dtype,
             "hg_linear: output type %d with type %d", a->out_dtype, a->dtype);
  HG_REQUIRE(!a->bias || is_float(a->bias_dtype), "hg_linear: bias type %d", a->bias_dtype);
  HG_REQUIRE(a->act >= HG_ACT_NONE && a->act <= HG_ACT_SILU, "hg_linear: activation %d", a->act);
  if (a->m >= kMost || a->k >= kMost || a->n >= kMost)
    return refuse(HG_EUNSUPPORTED, "hg_linear: a size of 2^31 or more");
  if (a->dtype == HG_DT_I8 && a->k > kMostIntegers)
    return refuse(HG_EUNSUPPORTED, "hg_linear: more than %d products of integers in a sum",
                  int(kMostIntegers));
  if (a->m == 0 || a->n == 0) return HG_OK;
  HG_REQUIRE(a->k == 0 || (in_ok(a->x, a->x_stride) && in_ok(a->w, a->w_stride)),
             "hg_linear: x or w is NULL or its stride negative");
  HG_REQUIRE(!is_8_bits(a->dtype) || (a->x_scale && a->w_scale), "hg_linear: 8 bits need scales");
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
  return linear_grad_workspace(m, k, n, dtype, act, false);
}

static hg_status linear_grad(const hg_linear_grad_args *a, const Kept &x, const Kept &pre,
                             int64_t need, hipStream_t stream) {
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
    HG_REQUIRE(need == 0 || (a->workspace && a->workspace_bytes >= need),
               "hg_linear_grad: workspace too small");
  }
  clear_pending();
  return launched(launch_linear_grad(*a, x, pre, stream), "hg_linear_grad");
}

hg_status hg_linear_grad(const hg_linear_grad_args *a, hipStream_t stream) {
  HG_REQUIRE(a, "hg_linear_grad: NULL arguments");
  return linear_grad(a, Kept(), Kept(),
                     hg_linear_grad_workspace(a->m, a->k, a->n, a->dtype, a->act), stream);
}

int64_t hg_linear_grad_kept_workspace(int64_t m, int64_t k, int64_t n, int32_t dtype, int32_t act) {
  if (m <= 0 || n <= 0 || k < 0 || m >= kMost || n >= kMost || k >= kMost) return 0;
  return linear_grad_workspace(m, k, n, dtype, act, true);
}

hg_status hg_linear_grad_kept(const hg_linear_grad_kept_args *args, hipStream_t stream) {
  HG_REQUIRE(args, "hg_linear_grad_kept: NULL arguments");
  HG_REQUIRE(group_ok(args->group), "hg_linear_grad_kept: group %d", args->group);
  const hg_linear_grad_args &a = args->grad;
  Kept x, pre;
  if (args->x_scale) x = kept(a.x, a.x_stride, args->x_scale, args->group, a.k);
  if (args->pre_scale) pre = kept(a.pre, a.pre_stride, args->pre_scale, args->group, a.n);
  // (x is widened for dw alone)
  const auto workspace = args->x_scale && a.dw ? hg_linear_grad_kept_workspace : hg_linear_grad_workspace;
  return linear_grad(&a, x, pre, workspace(a.m, a.k, a.n, a.dtype, a.act), stream);
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

// Entry points over label logits that take the caller's matrices (include/asgd.h, "Label
// logits"): argument checks and launches.
#include <math.h>
#include <stdio.h>

#include "../../include/asgd.h"
#include "asgd_kernels.h"
#include "ops_check.h"

namespace asgd {

asgd_status set_error_named(asgd_status s, const char* name, const char* msg) {
  char buf[200];
  snprintf(buf, sizeof buf, "%s%s", name, msg);
  return set_error(s, buf);
}

asgd_status hip_failed(hipError_t e, const char* what) {
  char buf[200];
  snprintf(buf, sizeof buf, "%s: %s", what, hipGetErrorString(e));
  return set_error(ASGD_EHIP, buf);
}

asgd_status check_list(const asgd_csr* a, const char* name, int rows, int cols, bool values) {
  if (!a) return ASGD_OK;
  if (a->n_rows != rows) return set_error_named(ASGD_EINVAL, name, ".n_rows differs from the logits' rows");
  if (a->n_cols != cols) return set_error_named(ASGD_EINVAL, name, ".n_cols differs from the logits' columns");
  if (a->nnz < 0) return set_error_named(ASGD_EINVAL, name, ".nnz must be >= 0");
  if (a->nnz >= (1 << 30)) return set_error_named(ASGD_ERANGE, name, ".nnz must be < 2^30");
  if (!a->indptr) return set_error_named(ASGD_EINVAL, name, ".indptr is NULL");
  if (a->nnz > 0 && !a->indices) return set_error_named(ASGD_EINVAL, name, ".indices is NULL");
  if (values && a->nnz > 0 && !a->values) return set_error_named(ASGD_EINVAL, name, ".values is NULL");
  if (((uintptr_t)a->indptr | (uintptr_t)a->indices | (values ? (uintptr_t)a->values : 0)) % 4)
    return set_error_named(ASGD_EINVAL, name, ": indptr, indices and values must be 4-byte aligned");
  return ASGD_OK;
}

IdLists list_dev(const asgd_csr* a, int row0) {
  if (!a || a->nnz == 0) return IdLists{};
  return IdLists{a->indptr, a->indptr + row0, a->indices, a->values, a->nnz};
}

namespace {

constexpr int kMaxRows = 1 << 20;
constexpr int kMaxLabels = 1 << 22;  // as for a model's n_labels

int elem_bytes(int dtype) { return dtype == ASGD_F32 ? 4 : 2; }

// One past the last byte of a matrix.
uintptr_t end_of(const asgd_matrix* a) {
  return (uintptr_t)a->data + ((int64_t)(a->n_rows - 1) * a->ld + a->n_cols) * elem_bytes(a->dtype);
}

}  // namespace

#define TRY(expr)             \
  do {                        \
    asgd_status s_ = (expr);  \
    if (s_) return s_;        \
  } while (0)

asgd_status check_matrix(const asgd_matrix* a, const char* name, bool label_rows) {
  if (!a) return set_error_named(ASGD_EINVAL, name, " is NULL");
  if (a->n_rows < 1 || a->n_cols < 1) return set_error_named(ASGD_EINVAL, name, ": n_rows and n_cols must be >= 1");
  if (label_rows ? a->n_rows >= kMaxLabels : a->n_rows > kMaxRows)
    return set_error_named(ASGD_ERANGE, name, label_rows ? ": n_rows must be < 2^22" : ": more than 2^20 rows");
  if (a->n_cols >= kMaxLabels) return set_error_named(ASGD_ERANGE, name, ": n_cols must be < 2^22");
  if (a->dtype != ASGD_F32 && a->dtype != ASGD_BF16 && a->dtype != ASGD_F16)
    return set_error_named(ASGD_EINVAL, name, ": unknown element type");
  if (a->ld < a->n_cols) return set_error_named(ASGD_EINVAL, name, ".ld is below n_cols");
  if (a->ld > ((int64_t)1 << 40)) return set_error_named(ASGD_ERANGE, name, ".ld is above 2^40");
  if (!a->data) return set_error_named(ASGD_EINVAL, name, ".data is NULL");
  if ((uintptr_t)a->data % elem_bytes(a->dtype))
    return set_error_named(ASGD_EINVAL, name, ".data is not aligned to its elements");
  return ASGD_OK;
}

asgd_status check_fp4(const asgd_fp4* q, const char* name) {
  if (!q) return set_error_named(ASGD_EINVAL, name, " is NULL");
  if (q->n_rows < 1 || q->n_cols < 1) return set_error_named(ASGD_EINVAL, name, ": n_rows and n_cols must be >= 1");
  if (q->n_cols % 32) return set_error_named(ASGD_EINVAL, name, ".n_cols must be a multiple of 32");
  if (q->n_rows >= kMaxLabels || (int64_t)q->n_rows * q->n_cols >= ((int64_t)1 << 31))
    return set_error_named(ASGD_ERANGE, name, ": n_rows must be < 2^22 and n_rows * n_cols < 2^31");
  if (!q->codes || !q->scales) return set_error_named(ASGD_EINVAL, name, ": codes and scales must be non-NULL");
  if ((uintptr_t)q->codes % 16 || (uintptr_t)q->scales % 4)
    return set_error_named(ASGD_EINVAL, name, ": codes must be 16-byte and scales 4-byte aligned");
  return ASGD_OK;
}

asgd_status check_rules(const asgd_logit_rules* r, int rows, int cols) {
  if (!r) return ASGD_OK;
  if (r->allowed && r->allowed_ld != 0 && r->allowed_ld < (cols + 31) / 32)
    return set_error(ASGD_EINVAL, "rules.allowed_ld is below ceil(n_cols / 32)");
  if (r->allowed && r->allowed_ld > ((int64_t)1 << 40)) return set_error(ASGD_ERANGE, "rules.allowed_ld is above 2^40");
  if (((uintptr_t)r->allowed | (uintptr_t)r->bias) % 4)
    return set_error(ASGD_EINVAL, "rules: bias and allowed must be 4-byte aligned");
  if (!(r->repetition >= 0.0) || !isfinite(r->repetition))
    return set_error(ASGD_EINVAL, "rules.repetition must be positive and finite (or 0 for none)");
  if (!isfinite(r->frequency) || !isfinite(r->presence))
    return set_error(ASGD_EINVAL, "rules.frequency and rules.presence must be finite");
  TRY(check_list(r->seen, "rules.seen", rows, cols, false));
  return check_list(r->row_bias, "rules.row_bias", rows, cols, true);
}

asgd_status check_temperature(float t) {
  if (!(t > 0.0f) || !isfinite(t)) return set_error(ASGD_EINVAL, "temperature must be positive and finite");
  if (t < 1e-6f || t > 1e6f) return set_error(ASGD_ERANGE, "temperature must be in [1e-6, 1e6]");
  return ASGD_OK;
}

RankRules rules_dev(const asgd_logit_rules* r, int row0) {
  RankRules d{};
  d.repetition = 1.0;
  if (!r) return d;
  d.bias = r->bias;
  d.allowed = r->allowed ? r->allowed + (int64_t)row0 * r->allowed_ld : nullptr;
  d.allowed_ld = r->allowed_ld;
  d.seen = list_dev(r->seen, row0);
  d.row_bias = list_dev(r->row_bias, row0);
  if (r->repetition > 0.0) d.repetition = r->repetition;
  d.frequency = r->frequency;
  d.presence = r->presence;
  return d;
}

asgd_status check_rules_memory(const asgd_logit_rules* r) {
  if (!r) return ASGD_OK;
  if (r->bias) TRY(check_device(r->bias, "rules.bias"));
  if (r->allowed) TRY(check_device(r->allowed, "rules.allowed"));
  if (r->seen && r->seen->nnz > 0) {
    TRY(check_device(r->seen->indptr, "rules.seen.indptr"));
    TRY(check_device(r->seen->indices, "rules.seen.indices"));
  }
  if (r->row_bias && r->row_bias->nnz > 0) {
    TRY(check_device(r->row_bias->indptr, "rules.row_bias.indptr"));
    TRY(check_device(r->row_bias->indices, "rules.row_bias.indices"));
    TRY(check_device(r->row_bias->values, "rules.row_bias.values"));
  }
  return ASGD_OK;
}

asgd_status check_device(const void* p, const char* name) {
  int dev = 0;
  hipError_t e = hipGetDevice(&dev);
  if (e != hipSuccess) return hip_failed(e, "hipGetDevice");
  return check_device_is(dev, p, name);
}

asgd_status check_device_is(int dev, const void* p, const char* name) {
  hipPointerAttribute_t a{};
  hipError_t e = hipPointerGetAttributes(&a, p);
  if (e != hipSuccess) (void)hipGetLastError();  // (an unknown address leaves an error behind)
  if (e != hipSuccess || (a.type != hipMemoryTypeDevice && a.type != hipMemoryTypeManaged))
    return set_error_named(ASGD_EINVAL, name, " is not device memory");
  if (a.device != dev) return set_error_named(ASGD_EINVAL, name, " is not on the current device");
  return ASGD_OK;
}

asgd_status check_stream(void* hip_stream) {
  if (!hip_stream) return ASGD_OK;
  int dev = 0;
  hipDevice_t of = 0;
  hipError_t e = hipGetDevice(&dev);
  if (e == hipSuccess) e = hipStreamGetDevice((hipStream_t)hip_stream, &of);
  if (e != hipSuccess) return hip_failed(e, "hipStreamGetDevice");
  if (of != dev) return set_error(ASGD_EINVAL, "hip_stream is not on the current device");
  return ASGD_OK;
}

asgd_status check_workspace(const void* ws, size_t have, size_t need) {
  if (need == 0) return ASGD_OK;
  if (have < need) return set_error(ASGD_ERANGE, "the workspace is smaller than the matching _workspace call says");
  if (!ws) return set_error(ASGD_EINVAL, "ws is NULL");
  if ((uintptr_t)ws % 256) return set_error(ASGD_EINVAL, "ws must be 256-byte aligned");
  return check_device(ws, "ws");
}

}  // namespace asgd

using namespace asgd;

#define LAUNCH(expr)                                      \
  do {                                                    \
    hipError_t e_ = (expr);                               \
    if (e_ != hipSuccess) return hip_failed(e_, #expr);   \
  } while (0)

extern "C" {

asgd_status asgd_fp4_quantize(const asgd_matrix* x, const asgd_fp4* q, void* hip_stream) {
  TRY(check_matrix(x, "x"));
  TRY(check_fp4(q, "q"));
  if (x->n_rows != q->n_rows || x->n_cols != q->n_cols) return set_error(ASGD_EINVAL, "x and q differ in shape");
  TRY(check_stream(hip_stream));
  TRY(check_device(x->data, "x.data"));
  TRY(check_device(q->codes, "q.codes"));
  TRY(check_device(q->scales, "q.scales"));
  LAUNCH(launch_fp4_quantize(x->dtype, x->data, x->ld, x->n_rows, x->n_cols, q->codes, q->scales,
                             (hipStream_t)hip_stream));
  return ASGD_OK;
}

asgd_status asgd_fp4_dequantize(const asgd_fp4* q, const asgd_matrix* out, void* hip_stream) {
  TRY(check_fp4(q, "q"));
  TRY(check_matrix(out, "out"));
  if (out->n_rows != q->n_rows || out->n_cols != q->n_cols) return set_error(ASGD_EINVAL, "q and out differ in shape");
  TRY(check_stream(hip_stream));
  TRY(check_device(q->codes, "q.codes"));
  TRY(check_device(q->scales, "q.scales"));
  TRY(check_device(out->data, "out.data"));
  LAUNCH(launch_fp4_dequantize(q->codes, q->scales, q->n_rows, q->n_cols, out->dtype, out->data, out->ld,
                               (hipStream_t)hip_stream));
  return ASGD_OK;
}

asgd_status asgd_fp4_logits(const asgd_matrix* h, const asgd_fp4* h4, const asgd_fp4* w, const float* bias,
                            const asgd_matrix* z, void* hip_stream) {
  if (!h == !h4) return set_error(ASGD_EINVAL, "exactly one of h and h4 must be given");
  TRY(h ? check_matrix(h, "h") : check_fp4(h4, "h4"));
  TRY(check_fp4(w, "w"));
  TRY(check_matrix(z, "z"));
  const int rows = h ? h->n_rows : h4->n_rows, cols = h ? h->n_cols : h4->n_cols;
  if (cols != HID || w->n_cols != HID) return set_error(ASGD_EINVAL, "the hidden rows and w must have 128 columns");
  if (z->n_rows != rows || z->n_cols != w->n_rows) return set_error(ASGD_EINVAL, "z must be [rows x labels]");
  if (h && h->dtype != ASGD_BF16) return set_error(ASGD_EINVAL, "h must be bf16");
  if (h && ((uintptr_t)h->data % 16 || h->ld % 8)) return set_error(ASGD_EINVAL, "h's rows must be 16-byte aligned");
  if ((uintptr_t)bias % 4) return set_error(ASGD_EINVAL, "bias must be 4-byte aligned");
  TRY(check_stream(hip_stream));
  TRY(check_device(h ? h->data : h4->codes, "the hidden rows"));
  if (h4) TRY(check_device(h4->scales, "h4.scales"));
  TRY(check_device(w->codes, "w.codes"));
  TRY(check_device(w->scales, "w.scales"));
  if (bias) TRY(check_device(bias, "bias"));
  TRY(check_device(z->data, "z.data"));
  const Fp4Rows a{h ? h->data : nullptr, h ? h->ld : 0, h4 ? h4->codes : nullptr, h4 ? h4->scales : nullptr};
  LAUNCH(launch_fp4_logits(a, rows, w->codes, w->scales, bias, w->n_rows, z->dtype, z->data, z->ld,
                           (hipStream_t)hip_stream));
  return ASGD_OK;
}

static asgd_status check_sizes(int32_t n_rows, int32_t n_cols, int32_t k, int max_k, size_t* bytes) {
  if (!bytes) return set_error(ASGD_EINVAL, "bytes is NULL");
  if (n_rows < 1 || n_cols < 1) return set_error(ASGD_EINVAL, "n_rows and n_cols must be >= 1");
  if (n_rows > kMaxRows || n_cols >= kMaxLabels)
    return set_error(ASGD_ERANGE, "n_rows must be <= 2^20 and n_cols < 2^22");
  if (k < 1 || k > max_k) return set_error(ASGD_EINVAL, max_k == RANK_MAX_K ? "k must be in [1, 64]" : "k must be in [1, 512]");
  return ASGD_OK;
}

asgd_status asgd_logits_topk_workspace(int32_t n_rows, int32_t n_cols, int32_t k, size_t* bytes) {
  TRY(check_sizes(n_rows, n_cols, k, RANK_MAX_K, bytes));
  *bytes = rank_ws_bytes(rank_shape(n_rows, n_cols), n_rows, k);
  return ASGD_OK;
}

asgd_status asgd_logits_topk(const asgd_matrix* z, const asgd_logit_rules* rules, int32_t k, int32_t* ids,
                             float* scores, float* lse, void* ws, size_t ws_bytes, void* hip_stream) {
  TRY(check_matrix(z, "z"));
  if (k < 1 || k > RANK_MAX_K) return set_error(ASGD_EINVAL, "k must be in [1, 64]");
  TRY(check_rules(rules, z->n_rows, z->n_cols));
  if (!ids) return set_error(ASGD_EINVAL, "ids is NULL");
  if (((uintptr_t)ids | (uintptr_t)scores | (uintptr_t)lse) % 4)
    return set_error(ASGD_EINVAL, "ids, scores and lse must be 4-byte aligned");
  const RankShape sh = rank_shape(z->n_rows, z->n_cols);
  TRY(check_workspace(ws, ws_bytes, rank_ws_bytes(sh, z->n_rows, k)));
  TRY(check_stream(hip_stream));
  TRY(check_device(z->data, "z.data"));
  TRY(check_rules_memory(rules));
  TRY(check_device(ids, "ids"));
  if (scores) TRY(check_device(scores, "scores"));
  if (lse) TRY(check_device(lse, "lse"));
  LAUNCH(launch_rank(z->dtype, z->data, z->ld, z->n_rows, z->n_cols, rules_dev(rules, 0), k, sh, ids, scores, lse, ws,
                     (hipStream_t)hip_stream));
  return ASGD_OK;
}

asgd_status asgd_distill_workspace(int32_t n_rows, int32_t n_cols, int32_t k, size_t* bytes) {
  TRY(check_sizes(n_rows, n_cols, k, DISTILL_MAX_K, bytes));
  *bytes = distill_ws_bytes(distill_splits(n_rows, n_cols), n_rows, k);
  return ASGD_OK;
}

asgd_status asgd_distill(const asgd_matrix* z, const int32_t* t_ids, const float* t_logits, int32_t k,
                         float temperature, const float* weights, float* loss_rows, const asgd_matrix* grad,
                         void* ws, size_t ws_bytes, void* hip_stream) {
  TRY(check_matrix(z, "z"));
  if (k < 1 || k > DISTILL_MAX_K) return set_error(ASGD_EINVAL, "k must be in [1, 512]");
  TRY(check_temperature(temperature));
  if (!t_ids || !t_logits || !loss_rows) return set_error(ASGD_EINVAL, "t_ids, t_logits and loss_rows must be non-NULL");
  if (((uintptr_t)t_ids | (uintptr_t)t_logits | (uintptr_t)loss_rows | (uintptr_t)weights) % 4)
    return set_error(ASGD_EINVAL, "t_ids, t_logits, weights and loss_rows must be 4-byte aligned");
  if (grad) {
    TRY(check_matrix(grad, "grad"));
    if (grad->n_rows != z->n_rows || grad->n_cols != z->n_cols || grad->dtype != z->dtype)
      return set_error(ASGD_EINVAL, "grad differs from z in shape or type");
    const bool same = grad->data == z->data && grad->ld == z->ld;
    if (!same && (uintptr_t)grad->data < end_of(z) && (uintptr_t)z->data < end_of(grad))
      return set_error(ASGD_EINVAL, "grad overlaps z without being z");
  }
  const int splits = distill_splits(z->n_rows, z->n_cols);
  TRY(check_workspace(ws, ws_bytes, distill_ws_bytes(splits, z->n_rows, k)));
  TRY(check_stream(hip_stream));
  TRY(check_device(z->data, "z.data"));
  TRY(check_device(t_ids, "t_ids"));
  TRY(check_device(t_logits, "t_logits"));
  if (weights) TRY(check_device(weights, "weights"));
  TRY(check_device(loss_rows, "loss_rows"));
  if (grad) TRY(check_device(grad->data, "grad.data"));
  const DistillJob j{z->data, z->ld, z->n_rows, z->n_cols, z->n_cols, t_ids, t_logits, k, temperature, weights, loss_rows,
                     grad ? grad->data : nullptr, grad ? grad->ld : 0};
  LAUNCH(launch_distill(z->dtype, j, splits, ws, (hipStream_t)hip_stream));
  return ASGD_OK;
}

}  // extern "C"

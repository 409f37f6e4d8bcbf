// Entry points for dense layers, dropout and the label loss on the caller's matrices (include/asgd.h,
// "A network of the caller's own"): argument checks and launches.
#include <math.h>

#include "../../include/asgd.h"
#include "asgd_kernels.h"
#include "ops_check.h"

using namespace asgd;

namespace {

#define TRY(expr)             \
  do {                        \
    asgd_status s_ = (expr);  \
    if (s_) return s_;        \
  } while (0)
#define LAUNCH(expr)                                      \
  do {                                                    \
    hipError_t e_ = (expr);                               \
    if (e_ != hipSuccess) return hip_failed(e_, #expr);   \
  } while (0)

int elem_bytes(int dtype) { return dtype == ASGD_F32 ? 4 : 2; }

MatDev mat_dev(const asgd_matrix* a) {
  if (!a) return MatDev{};
  return MatDev{a->data, a->ld, a->dtype};
}

// Bytes that an argument spans: rows of `width` bytes, `step` apart.
struct Span {
  uintptr_t at;
  int64_t rows, width, step;
};
Span span_of(const asgd_matrix* a) {
  const int es = elem_bytes(a->dtype);
  return Span{(uintptr_t)a->data, a->n_rows, (int64_t)a->n_cols * es, a->ld * es};
}
Span span_of(const float* p, int64_t n) { return Span{(uintptr_t)p, 1, 4 * n, 4 * n}; }

// Whether two arguments share a byte (columns of one buffer side by side do not).
bool meet(const Span& a, const Span& b) {
  if (!a.at || !b.at) return false;
  const uintptr_t ea = a.at + (a.rows - 1) * a.step + a.width, eb = b.at + (b.rows - 1) * b.step + b.width;
  if (a.at >= eb || b.at >= ea) return false;
  if (a.rows == 1 && b.rows == 1) return true;
  if (a.rows > 1 && b.rows > 1 && a.step != b.step) return true;
  const int64_t step = a.rows > 1 ? a.step : b.step;  // (one row lies between rows or meets them)
  const int64_t d = (int64_t)((a.at < b.at ? b.at - a.at : step - (int64_t)((a.at - b.at) % step)) % step);
  return d < a.width || d + b.width > step;
}
bool meet(const asgd_matrix* a, const asgd_matrix* b) { return a && b && meet(span_of(a), span_of(b)); }
// Whether they do and are not the same matrix.
bool meet_partly(const asgd_matrix* a, const asgd_matrix* b) {
  return meet(a, b) && !(a->data == b->data && (a->ld == b->ld || a->n_rows == 1) && a->dtype == b->dtype);
}

asgd_status check_shape(const asgd_matrix* a, const char* name, int rows, int cols) {
  TRY(check_matrix(a, name));
  if (a->n_rows != rows || a->n_cols != cols) return set_error_named(ASGD_EINVAL, name, " has another shape");
  return ASGD_OK;
}

asgd_status check_drop(double p) {
  if (!(p >= 0.0) || !(p < 1.0)) return set_error(ASGD_EINVAL, "the dropout probability must be in [0, 1)");
  return ASGD_OK;
}

uint64_t splitmix(uint64_t v) {
  v += 0x9E3779B97F4A7C15ull;
  v = (v ^ (v >> 30)) * 0xBF58476D1CE4E5B9ull;
  v = (v ^ (v >> 27)) * 0x94D049BB133111EBull;
  return v ^ (v >> 31);
}

DropDev drop_dev(double p, uint64_t seed) {
  return DropDev{splitmix(seed), (uint32_t)floor(p * 4294967296.0), (float)(1.0 / (1.0 - p))};
}

// Columns that a product is summed over: the offsets of a tile's copies are 32 bits, which its 256 rows of 4 MiB fill.
asgd_status check_sum(const asgd_matrix* a, const char* name) {
  if (a->n_cols > 1 << 20) return set_error_named(ASGD_ERANGE, name, ": more than 2^20 columns");
  return ASGD_OK;
}

// x [m x k] and w [n x k] of a layer.
asgd_status check_layer(const asgd_matrix* x, const asgd_matrix* w) {
  TRY(check_matrix(x, "x"));
  TRY(check_matrix(w, "w"));
  if (x->n_cols != w->n_cols) return set_error(ASGD_EINVAL, "x and w differ in columns");
  if (x->dtype != w->dtype) return set_error(ASGD_EINVAL, "x and w differ in type");
  return check_sum(x, "x");
}

asgd_status check_epilogue(const asgd_epilogue* e) {
  if (!e) return ASGD_OK;
  if (e->act < ASGD_ACT_NONE || e->act > ASGD_ACT_SILU) return set_error(ASGD_EINVAL, "epilogue.act is unknown");
  if ((uintptr_t)e->bias % 4) return set_error(ASGD_EINVAL, "epilogue.bias must be 4-byte aligned");
  return check_drop(e->drop);
}

asgd_status check_rows(const asgd_matrix* h, const asgd_matrix* w) {
  TRY(check_matrix(h, "h"));
  TRY(check_matrix(w, "w", true));
  if (h->n_cols != w->n_cols) return set_error(ASGD_EINVAL, "h and w differ in columns");
  if (h->dtype != w->dtype) return set_error(ASGD_EINVAL, "h and w differ in type");
  return check_sum(h, "h");
}

// The current device, which everything has to be on.
struct Device {
  int id = -1;
  asgd_status find() {
    const hipError_t e = hipGetDevice(&id);
    return e == hipSuccess ? ASGD_OK : hip_failed(e, "hipGetDevice");
  }
  asgd_status has(const void* p, const char* name) const { return p ? check_device_is(id, p, name) : ASGD_OK; }
  asgd_status has(const asgd_matrix* a, const char* name) const { return a ? has((const void*)a->data, name) : ASGD_OK; }
};

}  // namespace

extern "C" {

asgd_status asgd_dense_workspace(const asgd_matrix* x, const asgd_matrix* w, size_t* bytes) {
  if (!bytes) return set_error(ASGD_EINVAL, "bytes is NULL");
  TRY(check_layer(x, w));
  *bytes = dense_ws_bytes(x->dtype, mat_dev(x), mat_dev(w), x->n_rows, w->n_rows, x->n_cols);
  return ASGD_OK;
}

asgd_status asgd_dense(const asgd_matrix* x, const asgd_matrix* w, const asgd_epilogue* ep, const asgd_matrix* pre,
                       const asgd_matrix* y, void* ws, size_t ws_bytes, void* hip_stream) {
  TRY(check_layer(x, w));
  TRY(check_epilogue(ep));
  const int m = x->n_rows, n = w->n_rows;
  TRY(check_shape(y, "y", m, n));
  if (pre) TRY(check_shape(pre, "pre", m, n));
  const asgd_matrix* res = ep ? ep->residual : nullptr;
  if (res) TRY(check_shape(res, "epilogue.residual", m, n));
  const Span bias = span_of(ep ? ep->bias : nullptr, n);
  if (meet(y, x) || meet(y, w) || meet_partly(y, res) || meet(span_of(y), bias))
    return set_error(ASGD_EINVAL, "y overlaps an input (it may be the residual itself)");
  if (pre && (meet(pre, x) || meet(pre, w) || meet(pre, y) || meet(pre, res) || meet(span_of(pre), bias)))
    return set_error(ASGD_EINVAL, "pre overlaps another matrix");
  TRY(check_workspace(ws, ws_bytes, dense_ws_bytes(x->dtype, mat_dev(x), mat_dev(w), m, n, x->n_cols)));
  Device dev;
  TRY(dev.find());
  TRY(check_stream(hip_stream));
  TRY(dev.has(x, "x.data"));
  TRY(dev.has(w, "w.data"));
  TRY(dev.has(y, "y.data"));
  TRY(dev.has(pre, "pre.data"));
  TRY(dev.has(res, "epilogue.residual.data"));
  TRY(dev.has(ep ? ep->bias : nullptr, "epilogue.bias"));
  DenseJob j{x->dtype, mat_dev(x), mat_dev(w), m, n, x->n_cols, {}};
  if (ep) {
    j.epi.bias = ep->bias;
    j.epi.act = ep->act;
    j.epi.drop = drop_dev(ep->drop, ep->seed);
  }
  j.epi.res = mat_dev(res);
  j.epi.pre = mat_dev(pre);
  j.epi.y = mat_dev(y);
  LAUNCH(launch_dense(j, ws, (hipStream_t)hip_stream));
  return ASGD_OK;
}

asgd_status asgd_dense_backward_workspace(const asgd_matrix* x, const asgd_matrix* w, size_t* bytes) {
  if (!bytes) return set_error(ASGD_EINVAL, "bytes is NULL");
  TRY(check_layer(x, w));
  *bytes = dense_grad_ws_bytes(x->dtype, mat_dev(x), mat_dev(w), x->n_rows, w->n_rows, x->n_cols);
  return ASGD_OK;
}

asgd_status asgd_dense_backward(const asgd_matrix* dy, const asgd_matrix* x, const asgd_matrix* w,
                                const asgd_matrix* pre, const asgd_epilogue* ep, const asgd_matrix* dx,
                                const asgd_matrix* dw, float* db, void* ws, size_t ws_bytes, void* hip_stream) {
  TRY(check_layer(x, w));
  TRY(check_epilogue(ep));
  const int m = x->n_rows, n = w->n_rows, k = x->n_cols, act = ep ? ep->act : ASGD_ACT_NONE;
  TRY(check_shape(dy, "dy", m, n));
  if (act != ASGD_ACT_NONE && !pre) return set_error(ASGD_EINVAL, "the activation's gradient needs pre");
  if (pre) TRY(check_shape(pre, "pre", m, n));
  if (!dx && !dw && !db) return set_error(ASGD_EINVAL, "dx, dw and db are all NULL");
  if (dx) TRY(check_shape(dx, "dx", m, k));
  if (dw) TRY(check_shape(dw, "dw", n, k));
  if ((uintptr_t)db % 4) return set_error(ASGD_EINVAL, "db must be 4-byte aligned");
  const Span dbs = span_of(db, n);
  for (const asgd_matrix* in : {dy, x, w, pre})
    if (meet(dx, in) || meet(dw, in) || (in && meet(span_of(in), dbs)))
      return set_error(ASGD_EINVAL, "a gradient overlaps an input");
  if (meet(dx, dw) || (dx && meet(span_of(dx), dbs)) || (dw && meet(span_of(dw), dbs)))
    return set_error(ASGD_EINVAL, "gradients overlap");
  TRY(check_workspace(ws, ws_bytes, dense_grad_ws_bytes(x->dtype, mat_dev(x), mat_dev(w), m, n, k)));
  Device dev;
  TRY(dev.find());
  TRY(check_stream(hip_stream));
  TRY(dev.has(dy, "dy.data"));
  TRY(dev.has(x, "x.data"));
  TRY(dev.has(w, "w.data"));
  TRY(dev.has(pre, "pre.data"));
  TRY(dev.has(dx, "dx.data"));
  TRY(dev.has(dw, "dw.data"));
  TRY(dev.has(db, "db"));
  const DenseGradJob j{x->dtype, mat_dev(dy), mat_dev(pre), mat_dev(x), mat_dev(w), mat_dev(dx), mat_dev(dw), db, m, n, k,
                       act, ep ? drop_dev(ep->drop, ep->seed) : DropDev{}};
  LAUNCH(launch_dense_grad(j, ws, (hipStream_t)hip_stream));
  return ASGD_OK;
}

asgd_status asgd_dropout(const asgd_matrix* x, double p, uint64_t seed, const asgd_matrix* residual,
                         const asgd_matrix* y, void* hip_stream) {
  TRY(check_matrix(x, "x"));
  TRY(check_drop(p));
  TRY(check_shape(y, "y", x->n_rows, x->n_cols));
  if (residual) TRY(check_shape(residual, "residual", x->n_rows, x->n_cols));
  if (meet_partly(y, x) || meet_partly(y, residual))
    return set_error(ASGD_EINVAL, "y overlaps an input without being it");
  Device dev;
  TRY(dev.find());
  TRY(check_stream(hip_stream));
  TRY(dev.has(x, "x.data"));
  TRY(dev.has(y, "y.data"));
  TRY(dev.has(residual, "residual.data"));
  LAUNCH(launch_dropout(mat_dev(x), mat_dev(residual), mat_dev(y), drop_dev(p, seed), x->n_rows, x->n_cols,
                        (hipStream_t)hip_stream));
  return ASGD_OK;
}

asgd_status asgd_label_loss_workspace(const asgd_matrix* h, const asgd_matrix* w, int32_t gradients, size_t* bytes) {
  if (!bytes) return set_error(ASGD_EINVAL, "bytes is NULL");
  TRY(check_rows(h, w));
  *bytes = label_loss_ws_bytes(h->dtype, mat_dev(h), mat_dev(w), h->n_rows, w->n_rows, h->n_cols, gradients != 0);
  return ASGD_OK;
}

asgd_status asgd_label_loss(const asgd_matrix* h, const asgd_matrix* w, const float* bias, const asgd_csr* y,
                            const float* weights, float* loss_rows, float* lse, const asgd_matrix* dh,
                            const asgd_matrix* dw, float* db, void* ws, size_t ws_bytes, void* hip_stream) {
  TRY(check_rows(h, w));
  const int B = h->n_rows, L = w->n_rows, D = h->n_cols;
  if (!y) return set_error(ASGD_EINVAL, "y is NULL");
  TRY(check_list(y, "y", B, L, false));
  if (!loss_rows) return set_error(ASGD_EINVAL, "loss_rows is NULL");
  if (((uintptr_t)bias | (uintptr_t)weights | (uintptr_t)loss_rows | (uintptr_t)lse | (uintptr_t)db) % 4)
    return set_error(ASGD_EINVAL, "bias, weights, loss_rows, lse and db must be 4-byte aligned");
  if (dh) TRY(check_shape(dh, "dh", B, D));
  if (dw) {
    TRY(check_matrix(dw, "dw", true));
    if (dw->n_rows != L || dw->n_cols != D) return set_error(ASGD_EINVAL, "dw has another shape");
  }
  // what is written, against what is read and against each other
  const Span out[] = {span_of(loss_rows, B), span_of(lse, B), span_of(db, L), dh ? span_of(dh) : Span{}, dw ? span_of(dw) : Span{}};
  const Span in[] = {span_of(h), span_of(w), span_of(bias, L), span_of(weights, B), span_of((const float*)y->indptr, B + 1),
                     span_of((const float*)(y->nnz ? y->indices : nullptr), y->nnz)};
  for (int i = 0; i < 5; ++i) {
    for (const Span& s : in)
      if (meet(out[i], s)) return set_error(ASGD_EINVAL, "an output overlaps an input");
    for (int k = 0; k < i; ++k)
      if (meet(out[i], out[k])) return set_error(ASGD_EINVAL, "outputs overlap");
  }
  const bool grads = dh || dw || db;
  TRY(check_workspace(ws, ws_bytes, label_loss_ws_bytes(h->dtype, mat_dev(h), mat_dev(w), B, L, D, grads)));
  Device dev;
  TRY(dev.find());
  TRY(check_stream(hip_stream));
  TRY(dev.has(h, "h.data"));
  TRY(dev.has(w, "w.data"));
  TRY(dev.has(y->indptr, "y.indptr"));
  TRY(dev.has(y->nnz ? y->indices : nullptr, "y.indices"));
  TRY(dev.has(bias, "bias"));
  TRY(dev.has(weights, "weights"));
  TRY(dev.has(loss_rows, "loss_rows"));
  TRY(dev.has(lse, "lse"));
  TRY(dev.has(db, "db"));
  TRY(dev.has(dh, "dh.data"));
  TRY(dev.has(dw, "dw.data"));
  const LossJob j{h->dtype, mat_dev(h), mat_dev(w), B, L, D, bias, list_dev(y, 0), weights, loss_rows, lse, mat_dev(dh),
                  mat_dev(dw), db};
  LAUNCH(launch_label_loss(j, ws, (hipStream_t)hip_stream));
  return ASGD_OK;
}

}  // extern "C"

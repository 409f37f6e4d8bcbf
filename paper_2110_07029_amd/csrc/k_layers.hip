// Dense layers of any width with everything in the product's epilogue, their gradients, and dropout
// from a counter.
//
//   forward   A = X W^T + b ; Y = R + drop(act(A))
//   backward  dA = act'(A) drop(dY) (once, rounded to the operands' type, with the sums of its columns
//             in fp32 for db) ; dX = dA W ; dW = dA^T X
//   dropout   y = r + x / (1 - p) where 32 bits of splitmix64(key ^ (row 2^22 + column / 2)) are p 2^32 or more:
//             the mask is a function of seed and place, so that the backward pass forms it again
//
// The three products are tile_product.h's; few rows or few tiles split k over workgroups, whose sums
// meet in k_join.
#include <math.h>

#include <mutex>
#include <set>

#include "tile_plan.h"

namespace asgd {

hipError_t tp_allow_lds(const void* fn, int lds) {
  static std::mutex lock;
  static std::set<std::pair<const void*, int>> done;  // (kernel, device)
  int dev = 0;
  hipError_t e = hipGetDevice(&dev);
  if (e != hipSuccess) return e;
  try {
    const std::lock_guard<std::mutex> hold(lock);
    if (done.count({fn, dev})) return hipSuccess;
    e = hipFuncSetAttribute(fn, hipFuncAttributeMaxDynamicSharedMemorySize, lds);
    if (e == hipSuccess) done.insert({fn, dev});
  } catch (...) {  // (no memory for the note: set it again the next time)
  }
  return e;
}

// ---- rows out of line -----------------------------------------------------------------
template <typename T>
__global__ __launch_bounds__(256) void k_pack(const T* __restrict__ src, int64_t ld, int64_t rows, int cols,
                                              T* __restrict__ dst, int64_t ldp) {
  constexpr int V = 16 / (int)sizeof(T);
  typedef T vec __attribute__((ext_vector_type(V)));
  const int64_t per_row = ldp / V, total = rows * per_row;
  for (int64_t e = blockIdx.x * 256ll + threadIdx.x; e < total; e += 256ll * gridDim.x) {
    const int64_t r = e / per_row;
    const int c = (int)(e % per_row) * V;
    vec v;
#pragma unroll
    for (int i = 0; i < V; ++i) v[i] = c + i < cols ? src[r * ld + c + i] : (T)0.0f;
    *reinterpret_cast<vec*>(dst + r * ldp + c) = v;
  }
}

hipError_t launch_pack(int dtype, const MatDev& src, int64_t rows, int cols, void* dst, hipStream_t st) {
  const int64_t ldp = tp_packed_cols(dtype, cols), chunks = rows * ldp * elem_size(dtype) / 16;
  const int64_t want = ceil_div(chunks, 256);
  const dim3 grid((unsigned)(want < 4096 ? want : 4096));
  if (dtype == 0)
    hipLaunchKernelGGL(k_pack<float>, grid, dim3(256), 0, st, (const float*)src.data, src.ld, rows, cols, (float*)dst, ldp);
  else  // (16 bits are 16 bits)
    hipLaunchKernelGGL(k_pack<f16>, grid, dim3(256), 0, st, (const f16*)src.data, src.ld, rows, cols, (f16*)dst, ldp);
  return hipGetLastError();
}

// ---- slabs --------------------------------------------------------------------------------
// 256 / P groups of 8 columns per workgroup, P threads each, which take every P-th slab and meet in LDS (many slabs of few
// sums: 256 slabs of 256 x 128 take 25 us with one thread per group).
template <bool FULL, int P>
__global__ __launch_bounds__(256) void k_join(StoreArgs a, int splits, int m, int n, const float* __restrict__ live) {
  constexpr int GROUPS = 256 / P;
  __shared__ f32x4 meet[P > 1 ? 512 : 1];
  const int64_t per_row = (n + 7) / 8, total = m * per_row;
  const float alpha = FULL ? 1.0f : a.alpha * (a.alpha_dev ? *a.alpha_dev : 1.0f);
  const int which = threadIdx.x % GROUPS, part = threadIdx.x / GROUPS;
  for (int64_t e0 = blockIdx.x * (int64_t)GROUPS; e0 < total; e0 += (int64_t)GROUPS * gridDim.x) {
    const int64_t e = e0 + which, row = e / per_row;
    const int col = (int)(e % per_row) * 8;
    f32x4 lo{0.0f, 0.0f, 0.0f, 0.0f}, hi = lo;
    if (e < total) {
      const float* p = a.part + row * a.ldp + col + part * a.slab;
#pragma unroll 4
      for (int s = part; s < splits; s += P, p += P * a.slab) {
        lo += *reinterpret_cast<const f32x4*>(p);
        hi += *reinterpret_cast<const f32x4*>(p + 4);
      }
    }
    if constexpr (P > 1) {
      __syncthreads();
      meet[threadIdx.x] = lo;
      meet[256 + threadIdx.x] = hi;
      __syncthreads();
      if (part) continue;
#pragma unroll
      for (int k = 1; k < P; ++k) {
        lo += meet[k * GROUPS + which];
        hi += meet[256 + k * GROUPS + which];
      }
    }
    if (e >= total) continue;
    float v[8] = {lo[0], lo[1], lo[2], lo[3], hi[0], hi[1], hi[2], hi[3]};
    const int c = n - col < 8 ? n - col : 8;
    if constexpr (FULL) {
      float b[8];
      bias8(a.epi.bias, col, c, b);
      dense_out8(a.epi, b, row, col, c, v);
    } else {
      const bool zero = live && live[row] == 0.0f;
#pragma unroll
      for (int i = 0; i < 8; ++i) v[i] = zero ? 0.0f : v[i] * alpha;
      store8(a.epi.y, row, col, c, v);
    }
  }
}

hipError_t launch_join(const StoreArgs& a, int splits, int m, int n, bool full, const float* live, hipStream_t st) {
  const int p = splits >= 32 ? 16 : splits >= 8 ? 4 : 1;
  const int64_t want = ceil_div((int64_t)m * ((n + 7) / 8), 256 / p);
  const dim3 grid((unsigned)(want < 8192 ? want : 8192));
  auto go = [&](auto fn) { hipLaunchKernelGGL(fn, grid, dim3(256), 0, st, a, splits, m, n, live); };
  if (full) p == 16 ? go(k_join<true, 16>) : p == 4 ? go(k_join<true, 4>) : go(k_join<true, 1>);
  else p == 16 ? go(k_join<false, 16>) : p == 4 ? go(k_join<false, 4>) : go(k_join<false, 1>);
  return hipGetLastError();
}

// 64 columns per workgroup, sixteen waves take every sixteenth row.
__global__ __launch_bounds__(1024) void k_column_sums(const float* __restrict__ part, int rows, int64_t ld, int n,
                                                      float alpha, const float* alpha_dev, float* __restrict__ y) {
  __shared__ float s[16][64];
  const int lane = threadIdx.x & 63, w = threadIdx.x >> 6;
  const int64_t col = blockIdx.x * 64ll + lane;
  float v = 0.0f;
  if (col < n) {
#pragma unroll 4
    for (int r = w; r < rows; r += 16) v += part[r * ld + col];
  }
  s[w][lane] = v;
  __syncthreads();
  if (w == 0 && col < n) {
    float t = 0.0f;
#pragma unroll
    for (int i = 0; i < 16; ++i) t += s[i][lane];
    y[col] = t * alpha * (alpha_dev ? *alpha_dev : 1.0f);
  }
}

hipError_t launch_column_sums(const float* part, int rows, int64_t ld, int n, float alpha, const float* alpha_dev,
                              float* y, hipStream_t st) {
  hipLaunchKernelGGL(k_column_sums, dim3((unsigned)ceil_div(n, 64)), dim3(1024), 0, st, part, rows, ld, n, alpha, alpha_dev, y);
  return hipGetLastError();
}

// ---- forward ------------------------------------------------------------------------------
namespace {

constexpr int MAX_SPLITS = 64;

size_t slab_bytes(const TpPlan& p) {
  return p.job.splits > 1 ? round256((size_t)p.job.splits * p.job.m * ceil_div(p.job.n, 8) * 8 * 4) : 0;
}

struct Carve {  // places in the workspace, in order
  char* at;
  void* take(size_t n) {
    char* p = at;
    at += round256(n);
    return p;
  }
};

// `a` in place, or laid out anew in the workspace.
hipError_t operand(int dtype, const MatDev& a, int64_t rows, int cols, Carve* c, hipStream_t st, TpOperand* out) {
  if (tp_in_place(dtype, a, cols)) {
    *out = tp_operand(dtype, a.data, a.ld, rows, cols);
    return hipSuccess;
  }
  void* p = c->take(tp_packed_bytes(dtype, rows, cols));
  const int64_t ldp = tp_packed_cols(dtype, cols);
  *out = tp_operand(dtype, p, ldp, rows, ldp);
  return launch_pack(dtype, a, rows, cols, p, st);
}
size_t operand_bytes(int dtype, const MatDev& a, int64_t rows, int cols) {
  return tp_in_place(dtype, a, cols) ? 0 : tp_packed_bytes(dtype, rows, cols);
}

template <template <class> class Epi, bool AK, bool BK>
hipError_t any_type(int dtype, const TpPlan& p, const StoreArgs& a, hipStream_t st) {
  if (dtype == 0) return tp_launch<float, AK, BK, Epi>(p, a, st);
  if (dtype == 1) return tp_launch<bf16, AK, BK, Epi>(p, a, st);
  return tp_launch<f16, AK, BK, Epi>(p, a, st);
}

// C = A B^T through the epilogue, by way of slabs where k is split.
enum { DENSE, KROWS, KCOLS };
hipError_t product(int dtype, int kind, TpPlan p, const TpOperand& x, const TpOperand& y, StoreArgs a, Carve c,
                   hipStream_t st) {
  p.job.a = x;
  p.job.b = y;
  a.part = nullptr;
  if (p.job.splits > 1) {
    a.ldp = ceil_div(p.job.n, 8) * 8;
    a.slab = a.ldp * p.job.m;
    a.part = (float*)c.take(slab_bytes(p));
  }
  const hipError_t e =
      kind == DENSE ? any_type<EpiDense, true, true>(dtype, p, a, st) : launch_plain(dtype, kind == KROWS, p, a, st);
  if (e != hipSuccess || p.job.splits == 1) return e;
  return launch_join(a, p.job.splits, p.job.m, p.job.n, kind == DENSE, nullptr, st);
}

}  // namespace

hipError_t launch_plain(int dtype, bool a_krows, const TpPlan& p, const StoreArgs& a, hipStream_t st) {
  return a_krows ? any_type<EpiPlain, true, false>(dtype, p, a, st) : any_type<EpiPlain, false, false>(dtype, p, a, st);
}

size_t dense_ws_bytes(int dtype, const MatDev& x, const MatDev& w, int m, int n, int k) {
  return operand_bytes(dtype, x, m, k) + operand_bytes(dtype, w, n, k) + slab_bytes(tp_plan(dtype, m, n, k, MAX_SPLITS));
}

hipError_t launch_dense(const DenseJob& j, void* ws, hipStream_t st) {
  Carve c{(char*)ws};
  TpOperand x, w;
  hipError_t e = operand(j.dtype, j.x, j.m, j.k, &c, st, &x);
  if (e == hipSuccess) e = operand(j.dtype, j.w, j.n, j.k, &c, st, &w);
  if (e != hipSuccess) return e;
  StoreArgs a{};
  a.epi = j.epi;
  return product(j.dtype, DENSE, tp_plan(j.dtype, j.m, j.n, j.k, MAX_SPLITS), x, w, a, c, st);
}

// ---- backward ------------------------------------------------------------------------------
// dA = act'(pre) drop(dy), rounded to T (the operand of both products; its own rounding is of the size of their
// outputs'), into da (zeros up to ldd), and per row block the sums of its columns before the rounding.  `lpr` lanes of 8
// columns per row, the block's other lanes on further rows.
struct DaArgs {
  MatDev dy, pre;
  int act;
  DropDev drop;
  int m, n, rows_wg, lpr;
  int64_t ldd;
};
template <typename T>
__global__ __launch_bounds__(256) void k_dense_da(DaArgs a, T* __restrict__ da, float* __restrict__ part) {
  typedef T vec8 __attribute__((ext_vector_type(8)));
  __shared__ float s[256 * 8];
  const int tid = threadIdx.x, l = tid % a.lpr, g = tid / a.lpr, groups = 256 / a.lpr;
  const int col = ((int)blockIdx.x * a.lpr + l) * 8;
  const int r0 = (int)blockIdx.y * a.rows_wg, r1 = min(a.m, r0 + a.rows_wg);
  const int c = max(0, min(8, a.n - col));
  float sum[8] = {};
  if (c > 0)
    for (int r = r0 + g; r < r1; r += groups) {
      float v[8];
      load8(a.dy, r, col, c, v);
      if (a.act) {
        float p[8];
        load8(a.pre, r, col, c, p);
#pragma unroll
        for (int i = 0; i < 8; ++i) v[i] *= act_slope(a.act, p[i]);
      }
      if (a.drop.below) drop8(a.drop, r, col, v);
#pragma unroll
      for (int i = 0; i < 8; ++i) sum[i] += v[i];
      if (da) {
        if constexpr (sizeof(T) == 4) {
          f32x4* q = reinterpret_cast<f32x4*>(da + r * a.ldd + col);
          q[0] = f32x4{v[0], v[1], v[2], v[3]};
          if (a.ldd - col >= 8) q[1] = f32x4{v[4], v[5], v[6], v[7]};
        } else {
          vec8 o;
#pragma unroll
          for (int i = 0; i < 8; ++i) o[i] = i < c ? (T)v[i] : (T)0.0f;
          *reinterpret_cast<vec8*>(da + r * a.ldd + col) = o;
        }
      }
    }
  if (!part) return;
#pragma unroll
  for (int i = 0; i < 8; ++i) s[tid * 8 + i] = sum[i];
  __syncthreads();
  for (int i = tid; i < a.lpr * 8; i += 256) {
    const int cc = (int)blockIdx.x * a.lpr * 8 + i;
    if (cc >= a.n) continue;
    float t = 0.0f;
    for (int k = 0; k < groups; ++k) t += s[k * a.lpr * 8 + i];
    part[(int64_t)blockIdx.y * a.n + cc] = t;
  }
}

namespace {

int da_rows_wg(int m) {
  const int64_t r = ceil_div(m, 128);
  return (int)(r < 32 ? 32 : r);
}

}  // namespace

size_t dense_grad_ws_bytes(int dtype, const MatDev& x, const MatDev& w, int m, int n, int k) {
  const size_t da = tp_packed_bytes(dtype, m, n), part = round256(ceil_div(m, da_rows_wg(m)) * (size_t)n * 4);
  const size_t dx = slab_bytes(tp_plan(dtype, m, k, n, MAX_SPLITS)), dw = slab_bytes(tp_plan(dtype, n, k, m, MAX_SPLITS));
  return da + part + operand_bytes(dtype, x, m, k) + operand_bytes(dtype, w, n, k) + (dx > dw ? dx : dw);
}

hipError_t launch_dense_grad(const DenseGradJob& j, void* ws, hipStream_t st) {
  Carve c{(char*)ws};
  hipError_t e;
  const int64_t ldd = tp_packed_cols(j.dtype, j.n);
  const bool products = j.dx.data || j.dw.data;
  const bool same = !j.act && !j.drop.below && j.dy.dtype == j.dtype && tp_in_place(j.dtype, j.dy, j.n);
  TpOperand da = tp_operand(j.dtype, j.dy.data, j.dy.ld, j.m, j.n);
  void* dst = nullptr;
  if (products && !same) {
    dst = c.take(tp_packed_bytes(j.dtype, j.m, j.n));
    da = tp_operand(j.dtype, dst, ldd, j.m, ldd);
  }
  if (dst || j.db) {
    DaArgs a{j.dy, j.pre, j.act, j.drop, j.m, j.n, da_rows_wg(j.m), 64, ldd};
    while (a.lpr > 8 && a.lpr * 4 >= j.n) a.lpr /= 2;
    const int blocks = (int)ceil_div(j.m, a.rows_wg);
    float* part = j.db ? (float*)c.take((size_t)blocks * j.n * 4) : nullptr;
    const dim3 grid((unsigned)ceil_div(j.n, 8 * a.lpr), blocks);
    if (j.dtype == 0)
      hipLaunchKernelGGL(k_dense_da<float>, grid, dim3(256), 0, st, a, (float*)dst, part);
    else if (j.dtype == 1)
      hipLaunchKernelGGL(k_dense_da<bf16>, grid, dim3(256), 0, st, a, (bf16*)dst, part);
    else
      hipLaunchKernelGGL(k_dense_da<f16>, grid, dim3(256), 0, st, a, (f16*)dst, part);
    e = hipGetLastError();
    if (e == hipSuccess && j.db) e = launch_column_sums(part, blocks, j.n, j.n, 1.0f, nullptr, j.db, st);
    if (e != hipSuccess) return e;
  }
  StoreArgs a{};
  a.alpha = 1.0f;
  if (j.dx.data) {
    TpOperand w;
    Carve d = c;
    e = operand(j.dtype, j.w, j.n, j.k, &d, st, &w);
    if (e != hipSuccess) return e;
    a.epi.y = j.dx;
    e = product(j.dtype, KROWS, tp_plan(j.dtype, j.m, j.k, j.n, MAX_SPLITS), da, w, a, d, st);
    if (e != hipSuccess) return e;
  }
  if (j.dw.data) {
    TpOperand x;
    Carve d = c;
    e = operand(j.dtype, j.x, j.m, j.k, &d, st, &x);
    if (e != hipSuccess) return e;
    a.epi.y = j.dw;
    return product(j.dtype, KCOLS, tp_plan(j.dtype, j.n, j.k, j.m, MAX_SPLITS), da, x, a, d, st);
  }
  return hipSuccess;
}

// ---- dropout -----------------------------------------------------------------------------
__global__ __launch_bounds__(256) void k_dropout(MatDev x, MatDev res, MatDev y, DropDev d, int rows, int cols) {
  const int64_t per_row = (cols + 7) / 8, total = rows * per_row;
  for (int64_t e = blockIdx.x * 256ll + threadIdx.x; e < total; e += 256ll * gridDim.x) {
    const int64_t row = e / per_row;
    const int col = (int)(e % per_row) * 8, c = cols - col < 8 ? cols - col : 8;
    float v[8], r[8];
    load8(x, row, col, c, v);
    if (res.data) load8(res, row, col, c, r);
    if (d.below) drop8(d, row, col, v);
    if (res.data) {
#pragma unroll
      for (int i = 0; i < 8; ++i) v[i] += r[i];
    }
    store8(y, row, col, c, v);
  }
}

hipError_t launch_dropout(const MatDev& x, const MatDev& res, const MatDev& y, const DropDev& d, int rows, int cols,
                          hipStream_t st) {
  const int64_t want = ceil_div((int64_t)rows * ((cols + 7) / 8), 256);
  const dim3 grid((unsigned)(want < 16384 ? want : 16384));
  hipLaunchKernelGGL(k_dropout, grid, dim3(256), 0, st, x, res, y, d, rows, cols);
  return hipGetLastError();
}

}  // namespace asgd

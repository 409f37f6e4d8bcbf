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
// meet in k_join.  In bf16, GELU, dropout 0.1, a residual and A kept, 8,192 rows, 4,096 of 1,024 columns: 120 to 144 us by
// card, of which the product is 65 (69 GFLOP; the library's alone takes 58) and the epilogue 55 (random bits 21, GELU 20;
// 201 MB read and written are 40 at a copy's rate): a tile's products and another's epilogue meet on a compute unit, but do
// not add up to one.  Its gradients 202 to 222: dA 58 (random bits and GELU's slope; 201 MB), dX 75, dW 81 (69 GFLOP each;
// the library's 61 and 67), joining the slabs of dW 8.
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
struct PackJobs {
  PackJob j[2];
};
// One or two matrices, side by side in the grid's y.
template <typename T>
__global__ __launch_bounds__(256) void k_pack(PackJobs jobs) {
  constexpr int V = 16 / (int)sizeof(T);
  typedef T vec __attribute__((ext_vector_type(V)));
  const PackJob& j = jobs.j[blockIdx.y];
  const int64_t per_row = (j.cols + V - 1) / V, total = j.rows * per_row;
  for (int64_t e = blockIdx.x * 256ll + threadIdx.x; e < total; e += 256ll * gridDim.x) {
    const int64_t r = e / per_row;
    const int c = (int)(e % per_row) * V;
    const T* src = (const T*)j.src + r * j.ld + c;
    vec v;
    if (c + V <= j.cols && ((uintptr_t)src & 15) == 0) {
      v = *reinterpret_cast<const vec*>(src);
    } else {
#pragma unroll
      for (int i = 0; i < V; ++i) v[i] = c + i < j.cols ? src[i] : (T)0.0f;
    }
    reinterpret_cast<vec*>(j.dst)[e] = v;
  }
}

hipError_t launch_pack(int dtype, const PackJob* jobs, int n, hipStream_t st) {
  PackJobs p{};
  int64_t want = 1;
  for (int i = 0; i < n; ++i) {
    p.j[i] = jobs[i];
    const int64_t w = ceil_div(jobs[i].rows * tp_packed_cols(dtype, jobs[i].cols) * elem_size(dtype) / 16, 256);
    if (w > want) want = w;
  }
  const dim3 grid((unsigned)(want < 4096 ? want : 4096), n);
  if (dtype == 0)
    hipLaunchKernelGGL(k_pack<float>, grid, dim3(256), 0, st, p);
  else  // (16 bits are 16 bits)
    hipLaunchKernelGGL(k_pack<f16>, grid, dim3(256), 0, st, p);
  return hipGetLastError();
}

// ---- slabs --------------------------------------------------------------------------------
// 256 / P groups of 8 columns per workgroup, P threads each, which take every P-th slab and meet in LDS (many slabs of few
// sums: 256 slabs of 256 x 128 take 25 us with one thread per group).
template <bool FULL, int P>
__global__ __launch_bounds__(256) void k_join(StoreArgs a, int splits, int m, int n) {
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
      const bool zero = a.live && a.live[row] == 0.0f;
#pragma unroll
      for (int i = 0; i < 8; ++i) v[i] = zero ? 0.0f : v[i] * alpha;
      store8(a.epi.y, row, col, c, v);
    }
  }
}

hipError_t launch_join(const StoreArgs& a, int splits, int m, int n, bool full, hipStream_t st) {
  const int p = splits >= 32 ? 16 : splits >= 8 ? 4 : 1;
  const int64_t want = ceil_div((int64_t)m * ((n + 7) / 8), 256 / p);
  const dim3 grid((unsigned)(want < 8192 ? want : 8192));
  auto go = [&](auto fn) { hipLaunchKernelGGL(fn, grid, dim3(256), 0, st, a, splits, m, n); };
  if (full) p == 16 ? go(k_join<true, 16>) : p == 4 ? go(k_join<true, 4>) : go(k_join<true, 1>);
  else p == 16 ? go(k_join<false, 16>) : p == 4 ? go(k_join<false, 4>) : go(k_join<false, 1>);
  return hipGetLastError();
}

// 64 columns per workgroup of 256 or more threads, whose waves take turns at the rows.
__device__ __forceinline__ void column_sums(const SumJob& j, int block, float* s) {
  const int lane = threadIdx.x & 63, w = threadIdx.x >> 6, waves = blockDim.x >> 6;
  const int64_t col = block * 64ll + lane;
  float v = 0.0f;
  if (col < j.n) {
#pragma unroll 4
    for (int r = w; r < j.rows; r += waves) v += j.part[r * j.ld + col];
  }
  s[threadIdx.x] = v;
  __syncthreads();
  if (w == 0 && col < j.n) {
    float t = 0.0f;
    for (int i = 0; i < waves; ++i) t += s[64 * i + lane];
    j.y[col] = t * j.alpha * (j.alpha_dev ? *j.alpha_dev : 1.0f);
  }
}
__global__ __launch_bounds__(1024) void k_column_sums(SumJob j) {
  __shared__ float s[1024];
  column_sums(j, blockIdx.x, s);
}

hipError_t launch_column_sums(const SumJob& j, hipStream_t st) {
  if (!j.y) return hipSuccess;
  hipLaunchKernelGGL(k_column_sums, dim3((unsigned)ceil_div(j.n, 64)), dim3(1024), 0, st, j);
  return hipGetLastError();
}

// Both products and the sums in one launch: small ones are a few microseconds each, most of it the launch.
template <typename T, class S>
__global__ __launch_bounds__(S::THREADS) void k_pair(TpJob jx, StoreArgs ax, int nx, TpJob jy, StoreArgs ay, int ny, SumJob sums) {
  extern __shared__ __attribute__((aligned(16))) char smem[];
  const int b = blockIdx.x;
  if (b < nx)
    tp_tile<T, true, false, S, EpiPlain<S>>(jx, ax, b, smem);
  else if (b < nx + ny)
    tp_tile<T, false, false, S, EpiPlain<S>>(jy, ay, b - nx, smem);
  else
    column_sums(sums, b - nx - ny, reinterpret_cast<float*>(smem));
}

template <typename T, class S>
static hipError_t pair_launch(const PairJob& p, hipStream_t st) {
  const auto fn = k_pair<T, S>;
  constexpr int loop = S::NBUF * S::BUF, out = S::WAVES * S::OUT, lds = loop > out ? loop : out;
  const hipError_t e = tp_allow_lds((const void*)fn, lds);
  if (e != hipSuccess) return e;
  const int nx = p.x.job.a.base ? tp_blocks(p.x.job) : 0, ny = p.y.job.a.base ? tp_blocks(p.y.job) : 0;
  const int ns = p.sums.y ? (int)ceil_div(p.sums.n, 64) : 0;
  hipLaunchKernelGGL(fn, dim3(nx + ny + ns), dim3(S::THREADS), lds, st, p.x.job, p.ax, nx, p.y.job, p.ay, ny, p.sums);
  return hipGetLastError();
}
template <class S>
static hipError_t pair_type(int dtype, const PairJob& p, hipStream_t st) {
  if (dtype == 0) return pair_launch<float, S>(p, st);
  if (dtype == 1) return pair_launch<bf16, S>(p, st);
  return pair_launch<f16, S>(p, st);
}

hipError_t launch_pair(int dtype, const PairJob& p, hipStream_t st) {
  const bool x = p.x.job.a.base, y = p.y.job.a.base;
  hipError_t e = hipSuccess;
  const bool several = x + y + (p.sums.y != nullptr) > 1 && (x || y);
  const int shape = !several ? TP_LARGE : x && y && p.x.shape != p.y.shape ? TP_LARGE : (x ? p.x : p.y).shape;
  if (shape == TP_TINY) {
    e = pair_type<TpTiny>(dtype, p, st);
  } else if (shape == TP_SMALL) {
    e = pair_type<TpSmall>(dtype, p, st);
  } else {
    e = launch_column_sums(p.sums, st);
    if (e == hipSuccess && x) e = launch_plain(dtype, true, p.x, p.ax, st);
    if (e == hipSuccess && y) e = launch_plain(dtype, false, p.y, p.ay, st);
  }
  // (slabs that were added to are joined by the caller when all of them are there)
  if (e == hipSuccess && x && p.ax.part && !p.ax.keep)
    e = launch_join(p.ax, p.x.job.splits, p.x.job.m, p.x.job.n, false, st);
  if (e == hipSuccess && y && p.ay.part && !p.ay.keep)
    e = launch_join(p.ay, p.y.job.splits, p.y.job.m, p.y.job.n, false, st);
  return e;
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

// Operands in place, or laid out anew in the workspace (both in one launch).
hipError_t operands(int dtype, const MatDev* const* a, const int64_t* rows, int cols, int n, Carve* c, TpOperand* out,
                    hipStream_t st) {
  PackJob jobs[2];
  int packs = 0;
  for (int i = 0; i < n; ++i) {
    if (tp_in_place(dtype, *a[i], cols)) {
      out[i] = tp_operand(dtype, a[i]->data, a[i]->ld, rows[i], cols);
      continue;
    }
    void* p = c->take(tp_packed_bytes(dtype, rows[i], cols));
    const int64_t ldp = tp_packed_cols(dtype, cols);
    out[i] = tp_operand(dtype, p, ldp, rows[i], ldp);
    jobs[packs++] = PackJob{a[i]->data, a[i]->ld, rows[i], cols, p};
  }
  return packs ? launch_pack(dtype, jobs, packs, st) : hipSuccess;
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

// Slabs for the splits of a product.
void take_slabs(const TpPlan& p, StoreArgs* a, Carve* c) {
  if (p.job.splits < 2) return;
  a->ldp = ceil_div(p.job.n, 8) * 8;
  a->slab = a->ldp * p.job.m;
  a->part = (float*)c->take(slab_bytes(p));
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
  const MatDev* const mats[] = {&j.x, &j.w};
  const int64_t rows[] = {j.m, j.n};
  TpOperand o[2];
  hipError_t e = operands(j.dtype, mats, rows, j.k, 2, &c, o, st);
  if (e != hipSuccess) return e;
  StoreArgs a{};
  a.epi = j.epi;
  TpPlan p = tp_plan(j.dtype, j.m, j.n, j.k, MAX_SPLITS);
  p.job.a = o[0];
  p.job.b = o[1];
  take_slabs(p, &a, &c);
  e = any_type<EpiDense, true, true>(j.dtype, p, a, st);
  if (e != hipSuccess || !a.part) return e;
  return launch_join(a, p.job.splits, j.m, j.n, true, st);
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
        slope8(a.act, p, v);
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

// Rows per workgroup: some 4,096 workgroups (1,024 of them: 10 us more for 8,192 x 4,096), sums of 512 row blocks at most.
int da_rows_wg(int m, int n) {
  const int64_t cols = ceil_div(n, 512), blocks = ceil_div(4096, cols) < 512 ? ceil_div(4096, cols) : 512;
  const int64_t r = ceil_div(m, blocks);
  return (int)(r < 16 ? 16 : r);
}

}  // namespace

size_t dense_grad_ws_bytes(int dtype, const MatDev& x, const MatDev& w, int m, int n, int k) {
  const size_t da = tp_packed_bytes(dtype, m, n), part = round256(ceil_div(m, da_rows_wg(m, n)) * (size_t)n * 4);
  const size_t dx = slab_bytes(tp_plan(dtype, m, k, n, MAX_SPLITS)), dw = slab_bytes(tp_plan(dtype, n, k, m, MAX_SPLITS));
  return da + part + operand_bytes(dtype, x, m, k) + operand_bytes(dtype, w, n, k) + dx + dw;
}

hipError_t launch_dense_grad(const DenseGradJob& j, void* ws, hipStream_t st) {
  Carve c{(char*)ws};
  hipError_t e;
  PairJob p{};
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
    DaArgs a{j.dy, j.pre, j.act, j.drop, j.m, j.n, da_rows_wg(j.m, j.n), 64, ldd};
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
    if ((e = hipGetLastError()) != hipSuccess) return e;
    if (j.db) p.sums = SumJob{part, blocks, j.n, j.n, 1.0f, nullptr, j.db};
  }
  // x is needed for dw, w for dx
  const MatDev* mats[2];
  int64_t rows[2];
  int n = 0;
  if (j.dx.data) { mats[n] = &j.w; rows[n++] = j.n; }
  if (j.dw.data) { mats[n] = &j.x; rows[n++] = j.m; }
  TpOperand o[2];
  if ((e = operands(j.dtype, mats, rows, j.k, n, &c, o, st)) != hipSuccess) return e;
  p.ax.alpha = p.ay.alpha = 1.0f;
  if (j.dx.data) {
    p.x = tp_plan(j.dtype, j.m, j.k, j.n, MAX_SPLITS);
    p.x.job.a = da;
    p.x.job.b = o[0];
    p.ax.epi.y = j.dx;
    take_slabs(p.x, &p.ax, &c);
  }
  if (j.dw.data) {
    p.y = tp_plan(j.dtype, j.n, j.k, j.m, MAX_SPLITS);
    p.y.job.a = da;
    p.y.job.b = o[n - 1];
    p.ay.epi.y = j.dw;
    take_slabs(p.y, &p.ay, &c);
  }
  return launch_pair(j.dtype, p, st);
}

// ---- dropout -----------------------------------------------------------------------------
// One pass, 8 columns a thread; bound by memory (16,384 x 4,096 in bf16 with a residual: 403 MB in 72 us, 5.6 TB/s).
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

// Launch shapes of the tiled products (tile_product.h), the epilogue that dense layers and stored
// products share, and operands that are laid out anew where the caller's rows are out of line.
#pragma once

#include "rows_dev.h"
#include "tile_product.h"

namespace asgd {

using TpLarge = TpShape<256, 256, 2, 4, 2>;
using TpMedium = TpShape<128, 128, 2, 2, 2>;
using TpSmall = TpShape<64, 64, 2, 2, 3>;
using TpFew = TpShape<32, 128, 1, 4, 3>;
using TpTiny = TpShape<32, 32, 1, 1, 8, 4>;

enum { TP_LARGE = 0, TP_MEDIUM = 1, TP_SMALL = 2, TP_FEW = 3, TP_TINY = 4 };
constexpr int TP_BM[] = {256, 128, 64, 32, 32}, TP_BN[] = {256, 128, 64, 128, 32};

// Up to so many steps of k large tiles spend too much of their time around the loop: gradients of 732 rows, 26,436
// labels, width 763 (12 steps) 333 us with them, 264 without; a layer of 8,192 x 4,096 with 16 steps 120, 124 without.
constexpr int SHORT_K = 12;

struct TpPlan {
  int shape;
  TpJob job;
};

inline int64_t ceil_div(int64_t a, int64_t b) { return (a + b - 1) / b; }
inline int elem_size(int dtype) { return dtype == 0 ? 4 : 2; }

// Shape and splits of a product of m x n over k; max_splits 1: the epilogue needs whole sums.
//   large tiles   where they fill the chip and k is long enough that what surrounds the loop (1 workgroup per CU) is
//                 little; also where few of them with a long k are worth their slabs
//   medium, small where they fill it, with k split if that takes a long k and (medium) enough work to pay for the slabs
//   few           up to 32 rows of many columns; tiny: everything else, latency counts
// (The label loss of 326 rows, 82,407 labels, width 538, whose dz W has 326 x 538 sums over 82,407: 548 us with tiny tiles
// for them, 354 with medium ones.)
inline TpPlan tp_plan(int dtype, int m, int n, int64_t k, int max_splits) {
  TpPlan p{};
  TpJob& j = p.job;
  j.m = m;
  j.n = n;
  j.k = k;
  const int kb = TP_STEP / elem_size(dtype);
  const int64_t large = ceil_div(m, 256) * ceil_div(n, 256), medium = ceil_div(m, 128) * ceil_div(n, 128);
  const int64_t small = ceil_div(m, 64) * ceil_div(n, 64), steps = ceil_div(k, kb);
  int64_t most = steps / 8 < max_splits ? steps / 8 : max_splits;
  if (most < 1 || steps < 24) most = 1;
  const bool split_large = large >= 48 && large < 192 && max_splits > 1 && k * large >= 8192ll * 256;
  // (fp32 takes longer for the same slabs; tiles that would be a quarter emptier than small ones stay small.  The label loss in
  // fp32 of 995 rows, 6,929 labels, width 1,208: 803 us from 1e10 on, 676 from 5e9; of 556 rows, 253,146 labels, width 128
  // 2,116, and 2,262 from 1e9.)
  const bool much = (double)m * n * k >= (dtype == 0 ? 5e9 : 1e10) && 16 * medium <= 5 * small;
  p.shape = m <= 32                                           ? (n > 192 * 128 ? TP_FEW : TP_TINY)
            : (large >= 192 && steps > SHORT_K) || split_large ? TP_LARGE
            : medium >= 192 || (much && medium * most >= 256)  ? TP_MEDIUM
            : small * most >= 128                              ? TP_SMALL
                                                               : TP_TINY;
  j.tiles_m = (int)ceil_div(m, TP_BM[p.shape]);
  j.tiles_n = (int)ceil_div(n, TP_BN[p.shape]);
  const int64_t tiles = (int64_t)j.tiles_m * j.tiles_n;
  // splits of k cost a launch that joins them: long k of few tiles alone
  int64_t s = 1;
  if (split_large) s = 256 / tiles;
  else if (p.shape != TP_LARGE && tiles <= 256) s = 512 / tiles;
  s = s < most ? s : most;
  if (s < 1) s = 1;
  const int64_t per = ceil_div(steps, s);
  j.splits = (int)ceil_div(steps, per);
  j.split_k = per * kb;
  j.group = 8 < j.tiles_m ? 8 : j.tiles_m;
  return p;
}

// Lets a kernel have `lds` bytes of dynamic LDS on the current device.
hipError_t tp_allow_lds(const void* fn, int lds);

template <typename T, bool AK, bool BK, class S, class Epi>
hipError_t tp_launch_shape(const TpJob& j, const typename Epi::Args& ea, hipStream_t st) {
  constexpr int loop = S::NBUF * S::BUF, out = Epi::BLOCKS * S::WAVES * S::OUT;
  constexpr int lds = (loop > out ? loop : out) + Epi::TAIL;
  static_assert(lds <= 160 * 1024, "LDS of a compute unit");
  const auto fn = k_tile_product<T, AK, BK, S, Epi>;
  const hipError_t e = tp_allow_lds((const void*)fn, lds);
  if (e != hipSuccess) return e;
  // (a launch has less than 2^32 threads)
  constexpr int MOST = 1 << 22;
  TpJob part = j;
  for (int64_t b = 0; b < tp_blocks(j); b += MOST) {
    part.block0 = (int)b;
    const int64_t n = tp_blocks(j) - b < MOST ? tp_blocks(j) - b : MOST;
    hipLaunchKernelGGL(fn, dim3((unsigned)n), dim3(S::THREADS), lds, st, part, ea);
    const hipError_t r = hipGetLastError();
    if (r != hipSuccess) return r;
  }
  return hipSuccess;
}

template <typename T, bool AK, bool BK, template <class> class Epi>
hipError_t tp_launch(const TpPlan& p, const typename Epi<TpLarge>::Args& ea, hipStream_t st) {
  if (p.shape == TP_LARGE) return tp_launch_shape<T, AK, BK, TpLarge, Epi<TpLarge>>(p.job, ea, st);
  if (p.shape == TP_SMALL) return tp_launch_shape<T, AK, BK, TpSmall, Epi<TpSmall>>(p.job, ea, st);
  if (p.shape == TP_MEDIUM) return tp_launch_shape<T, AK, BK, TpMedium, Epi<TpMedium>>(p.job, ea, st);
  if (p.shape == TP_TINY) return tp_launch_shape<T, AK, BK, TpTiny, Epi<TpTiny>>(p.job, ea, st);
  return tp_launch_shape<T, AK, BK, TpFew, Epi<TpFew>>(p.job, ea, st);
}

// The same plan for fewer columns.
inline void tp_narrow(TpPlan* p, int n) {
  p->job.n = n;
  p->job.tiles_n = (int)ceil_div(n, TP_BN[p->shape]);
}

// ---- operands in place or laid out anew ---------------------------------------------------
// Rows can be read in place if they are made of whole 16-byte chunks and close enough for a tile's
// offsets to fit 31 bits.
inline bool tp_in_place(int dtype, const MatDev& a, int cols) {
  const int es = elem_size(dtype);
  return ((uintptr_t)a.data | (uint64_t)(a.ld * es)) % 16 == 0 && (int64_t)cols * es % 16 == 0 && a.ld * es <= (1 << 22);
}
inline int64_t tp_packed_cols(int dtype, int cols) { return ceil_div(cols, 16 / elem_size(dtype)) * (16 / elem_size(dtype)); }
inline size_t round256(size_t n) { return (n + 255) / 256 * 256; }
inline size_t tp_packed_bytes(int dtype, int64_t rows, int cols) {
  return round256((size_t)(rows * tp_packed_cols(dtype, cols) * elem_size(dtype)));
}
inline TpOperand tp_operand(int dtype, const void* data, int64_t ld, int64_t rows, int64_t cols) {
  const int es = elem_size(dtype);
  return TpOperand{(const char*)data, ld * es, ((rows - 1) * ld + cols) * es};
}
// dst [rows x packed cols] = src, zeros behind its columns.
struct PackJob {
  const void* src;
  int64_t ld, rows;
  int cols;
  void* dst;
};
hipError_t launch_pack(int dtype, const PackJob* jobs, int n, hipStream_t st);  // n <= 2

// ---- the epilogue of dense layers and of stored products ---------------------------------
// Sums of one split go to a slab of floats of their own (part, [splits][m x ldp]), added to what is
// there with `add`; whole sums go out through dense_out8 (FULL) or scaled by alpha and *alpha_dev.
struct StoreArgs {
  DenseEpi epi;
  float* part;
  int64_t ldp, slab;
  int add, keep;  // keep: the slabs are joined by the caller
  float alpha;
  const float* alpha_dev;
  const float* live;  // or null: rows whose entry is 0 become zeros
};

template <class S, bool FULL>
struct EpiStore {
  using Args = StoreArgs;
  static constexpr int BLOCKS = 1, TAIL = 0;
  static constexpr int LPR = S::WCOLS / 8, RPP = 64 / LPR;  // lanes per row, rows per pass
  const StoreArgs& a;
  int m, n, c;
  float* part;
  float alpha;
  float b[FULL ? 8 : 1];
  __device__ EpiStore(const StoreArgs& args, const TpJob& j, int, int col0, int split, int wave, int lane)
      : a(args), m(j.m), n(j.n) {
    part = a.part ? a.part + split * a.slab : nullptr;
    alpha = FULL ? 1.0f : a.alpha * (a.alpha_dev ? *a.alpha_dev : 1.0f);
    const int col = col0 + wave % S::WN * S::WCOLS + 8 * (lane % LPR);
    c = n - col < 8 ? n - col : 8;
    if constexpr (FULL) bias8(a.epi.bias, col, c, b);
  }
  __device__ void begin(char*) {}
  __device__ __forceinline__ void block(const f32x16 (&acc)[S::TN], int row0, int colw, float* out, int, int lane) {
    tp_stage<S>(acc, out, lane);
    const int col = colw + 8 * (lane % LPR);
    if (c > 0) {
#pragma unroll 1  // (four copies of the epilogue's code are enough)
      for (int p = 0; p < 32 / RPP; ++p) {
        const int r = p * RPP + lane / LPR;
        if (row0 + r >= m) break;
        float v[8];
        tp_staged8<S>(out, r, 8 * (lane % LPR), v);
        put(row0 + r, col, v);
      }
    }
    __builtin_amdgcn_fence(__ATOMIC_SEQ_CST, "wavefront");
  }
  __device__ __forceinline__ void put(int row, int col, float v[8]) {
    if (part) {  // (ldp covers whole groups of 8 columns)
      f32x4* p = reinterpret_cast<f32x4*>(part + row * a.ldp + col);
      f32x4 lo{v[0], v[1], v[2], v[3]}, hi{v[4], v[5], v[6], v[7]};
      if (a.add) {
        lo += p[0];
        hi += p[1];
      }
      p[0] = lo;
      p[1] = hi;
      return;
    }
    if constexpr (FULL) {
      dense_out8(a.epi, b, row, col, c, v);
    } else {
#pragma unroll
      for (int i = 0; i < 8; ++i) v[i] = a.live && a.live[row] == 0.0f ? 0.0f : v[i] * alpha;
      store8(a.epi.y, row, col, c, v);
    }
  }
  __device__ void end(int, int, int, int, int) {}
};
template <class S>
using EpiDense = EpiStore<S, true>;
template <class S>
using EpiPlain = EpiStore<S, false>;

// The product with the plain epilogue: a has k along its rows (a_krows) or across them, b across them.
hipError_t launch_plain(int dtype, bool a_krows, const TpPlan& p, const StoreArgs& a, hipStream_t st);
// Adds the slabs of a product and puts the sums out as the epilogue would.
hipError_t launch_join(const StoreArgs& a, int splits, int m, int n, bool full, hipStream_t st);
// y[j] = alpha *alpha_dev sum_i part[i][j], i < rows; y null: nothing.
struct SumJob {
  const float* part;
  int rows;
  int64_t ld;
  int n;
  float alpha;
  const float* alpha_dev;
  float* y;
};
hipError_t launch_column_sums(const SumJob& s, hipStream_t st);
// What both gradients of a product take: a x (k along a's rows) and a^T y (k across), either with its operands null
// for none, and sums; in one launch where the products are small.  Products that split k are joined.
struct PairJob {
  TpPlan x, y;
  StoreArgs ax, ay;
  SumJob sums;
};
hipError_t launch_pair(int dtype, const PairJob& p, hipStream_t st);

}  // namespace asgd

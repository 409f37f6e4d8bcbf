// Softmax cross-entropy over a label matrix, in pieces of the labels, without the logits, and its
// gradients.
//
//   z_ij = h_i . w_j + b_j ;  lse_i = ln sum_j e^z_ij ;  n_i = valid entries of row i's list
//   loss_i = lse_i - (1 / n_i) sum of z_iy over the entries
//   dz_ij = weight_i (e^(z_ij - lse_i) - c_ij / n_i), c_ij how often j stands in the list
//   dh = dz W ; dw = dz^T h ; db = 1^T dz
//
//   product 1     z in tiles; per row and tile the maximum and the sum of exponentials
//   k_loss_rows   n_i; lse; the target logits as products of their own; loss; for gradients the largest |weight| and a
//                 copy of h in which rows without labels are zeros (what they hold must not reach dw)
//   per piece of labels:
//     product 2   z again, dz formed in fp32 from it, the targets taken off in place; its column sums
//                 for db in fp32; dz rounded to the operands' type in the workspace
//     products 3, 4   dz W onto slabs of dh, dz^T h: the piece's rows of dw; column sums for db
//   k_join        dh
//
// Rows of 16 bits up to 128 wide take other kernels for product 1, and for the gradients where there are up to 256 of them or
// many labels (k_label_narrow.hip).
//
// 4,096 rows, 32,001 labels, width 2,048 in bf16: 1,930 to 2,090 us for four products of 537 GFLOP, 1.03 to 1.11 PFLOP/s
// (the library's product of 8,192 cubed reaches 1.39 with k along both operands' rows, 1.21 and 1.08 in the forms that the
// gradients' products have).  Forming z twice is the fourth product; storing dz of all labels would take 262 MB, and a loss
// that is only read needs no dz at all.  dz in 16 bits is
// rounded once, with the target in it (p and the target may nearly cancel); fp16 holds it times 2^15 over the
// largest weight, so that probabilities of a row of that weight stay normal down to 2^-29, and of a row of 1/x of it down to
// x 2^-29: one scale for all, since the products sum over rows.
#include <float.h>
#include <math.h>

#include "label_loss_dev.h"

namespace asgd {

namespace {

// Of dz at a time: the products read it from the last cache (256 MB), and pieces are large enough to fill the chip (4,096 rows,
// 32,001 labels, width 2,048: 2,151 us with 64 MiB, 2,078 with 128, 2,079 with 512).
constexpr int64_t PIECE_BYTES = 128ll << 20;
constexpr int MAX_SLABS = 64;
typedef unsigned u32x4 __attribute__((ext_vector_type(4)));

// Entries of row i that count: ids in [0, L).
__device__ __forceinline__ int entry(const IdLists& y, int q, int L) {
  const int id = y.indices[q];
  return (unsigned)id < (unsigned)L ? id : -1;
}

}  // namespace

// ---- product 1 -------------------------------------------------------------------------------------
struct LseArgs {
  const float* bias;
  float2* part;  // [B][tiles_n]
};

// The tile's biases in LDS (zeros without, and past the last column): a lane's accumulators hold columns
// 32 b + 8 q + 4 g + 0..3 of its wave's.
template <class S>
__device__ __forceinline__ void tile_bias(const float* bias, int c0, int n, float* to) {
  for (int c = threadIdx.x; c < S::BN; c += S::THREADS) to[c] = bias && c0 + c < n ? bias[c0 + c] : 0.0f;
}

// All in the accumulators: a lane has half of a wave's columns of its row.
template <class S>
struct EpiLse {
  using Args = LseArgs;
  static constexpr int BLOCKS = 1, TAIL = S::WN * S::BM * 8 + S::BN * 4;
  const LseArgs& a;
  int m, n, row0, col0, tile, tiles;
  float2* ms;   // [WN][BM]
  float* bias;  // [BN]
  __device__ EpiLse(const LseArgs& args, const TpJob& j, int r0, int c0, int, int wave, int lane)
      : a(args), m(j.m), n(j.n), row0(r0), col0(c0), tile(c0 / S::BN), tiles(j.tiles_n) {}
  __device__ void begin(char* tail) {
    ms = reinterpret_cast<float2*>(tail);
    bias = reinterpret_cast<float*>(tail + S::WN * S::BM * 8);
    tile_bias<S>(a.bias, col0, n, bias);  // (the loop's barriers lie between)
  }
  __device__ __forceinline__ void block(const f32x16 (&acc)[S::TN], int r0, int colw, float*, int wave, int lane) {
    float v[S::TN][16], top = -INFINITY;
    const bool edge = colw + S::WCOLS > n;  // (the same for the whole wave)
    const int g = lane >> 5;
#pragma unroll
    for (int b = 0; b < S::TN; ++b)
#pragma unroll
      for (int q = 0; q < 4; ++q) {
        const f32x4 t = *reinterpret_cast<const f32x4*>(bias + colw - col0 + 32 * b + 8 * q + 4 * g);
#pragma unroll
        for (int i = 0; i < 4; ++i) {
          float& x = v[b][4 * q + i];
          x = acc[b][4 * q + i] + t[i];
          if (edge && colw + 32 * b + 8 * q + 4 * g + i >= n) x = -INFINITY;
          top = fmaxf(top, x);
        }
      }
    top = fmaxf(top, __builtin_bit_cast(float, lane_xor<32>(__builtin_bit_cast(unsigned, top), lane)));
    const float base = top == -INFINITY ? 0.0f : top;
    float s[4] = {};
#pragma unroll
    for (int b = 0; b < S::TN; ++b)
#pragma unroll
      for (int r = 0; r < 16; ++r) s[r & 3] += exp_fast(v[b][r] - base);
    float t = (s[0] + s[1]) + (s[2] + s[3]);
    t += __builtin_bit_cast(float, lane_xor<32>(__builtin_bit_cast(unsigned, t), lane));
    if (lane < 32) ms[(wave % S::WN) * S::BM + r0 - row0 + lane] = make_float2(top, t);
  }
  __device__ void end(int, int, int, int, int tid) {
    __syncthreads();
    for (int r = tid; r < S::BM; r += S::THREADS) {
      if (row0 + r >= m) continue;
      float top = -INFINITY, s = 0.0f;
#pragma unroll
      for (int k = 0; k < S::WN; ++k) top = fmaxf(top, ms[k * S::BM + r].x);
      const float base = top == -INFINITY ? 0.0f : top;
#pragma unroll
      for (int k = 0; k < S::WN; ++k) s += ms[k * S::BM + r].y * exp_fast(ms[k * S::BM + r].x - base);
      a.part[(int64_t)(row0 + r) * tiles + tile] = make_float2(top, s);
    }
  }
};

// ---- lse and loss --------------------------------------------------------------------------------
// One workgroup per row.  Target logits are products of their own, 16 lanes each (h and w as the products read them: whole
// 16-byte pieces).  With `scale` one workgroup more, the first, finds the gradients' scale: the largest finite |weight| of rows
// that have labels, 1 / B without weights; it reads eight rows a thread at once (one at a
// time, gradients of 2^20 rows of width 16 in rising order of weight waited for it: 7.9 ms, 5.7 so).
template <typename T>
__global__ __launch_bounds__(256) void k_loss_rows(const float2* __restrict__ part, int tiles, TpOperand h, TpOperand w,
                                                   int D, int L, const float* __restrict__ bias, IdLists y,
                                                   float* __restrict__ share, float* __restrict__ top_ws,
                                                   float* __restrict__ inv, float* __restrict__ lse_out, float* __restrict__ loss, int B,
                                                   const float* __restrict__ weights, float* __restrict__ scale,
                                                   T* __restrict__ hp, int64_t ldp) {
  constexpr int V = 16 / (int)sizeof(T);
  typedef T vec __attribute__((ext_vector_type(V)));
  const int i = (int)blockIdx.x - (scale ? 1 : 0), tid = threadIdx.x, lane = tid & 63, wave = tid >> 6;
  __shared__ float sm[4], ss[4], st[4];
  __shared__ int sn[4];
  if (i < 0) {
    float v = 0.0f;
    if (weights && y.indptr)
      for (int r0 = tid; r0 < B; r0 += 256 * 8) {
        float a[8];
        int q0[8], q1[8];
        bool live[8] = {}, more = true;
#pragma unroll
        for (int k = 0; k < 8; ++k) {
          const int r = min(r0 + 256 * k, B - 1);
          a[k] = fabsf(weights[r]);
          label_range(y, r, &q0[k], &q1[k]);
        }
        while (more) {  // an entry of each row that may matter, until one counts
          int id[8];
          more = false;
#pragma unroll
          for (int k = 0; k < 8; ++k) {
            const bool look = !live[k] && a[k] > v && a[k] < INFINITY && q0[k] < q1[k];
            id[k] = look ? entry(y, q0[k]++, L) : -1;
            more |= look;
          }
#pragma unroll
          for (int k = 0; k < 8; ++k) live[k] |= id[k] >= 0;
        }
#pragma unroll
        for (int k = 0; k < 8; ++k)
          if (live[k]) v = fmaxf(v, a[k]);
      }
    v = wave_max(v);
    if (lane == 0) sm[wave] = v;
    __syncthreads();
    if (tid == 0) *scale = weights ? fmaxf(fmaxf(sm[0], sm[1]), fmaxf(sm[2], sm[3])) : 1.0f / (float)B;
    return;
  }
  const float2* p = part + (int64_t)i * tiles;
  float top = -INFINITY;
  for (int k = tid; k < tiles; k += 256) top = fmaxf(top, p[k].x);
  float t = 0.0f;
  int n = 0;
  const T* hr = (const T*)(h.base + i * h.ld);
  if (y.indptr) {
    int q0, q1;
    label_range(y, i, &q0, &q1);
    const int l = tid & 15;
    constexpr int E = 4;  // entries on their way at once (75 of them in 1,024 rows: 13 us one at a time)
    for (int o = tid >> 4; o < q1 - q0; o += 16 * E) {
      int id[E];
      float d[E];
#pragma unroll
      for (int e = 0; e < E; ++e) {
        id[e] = o + 16 * e < q1 - q0 ? entry(y, q0 + o + 16 * e, L) : -1;
        d[e] = 0.0f;
      }
      for (int c = V * l; c < D; c += V * 16) {
        const vec a = *reinterpret_cast<const vec*>(hr + c);
        vec b[E];
#pragma unroll
        for (int e = 0; e < E; ++e)  // (a place without entry reads row 0, for nothing)
          b[e] = *reinterpret_cast<const vec*>(w.base + (id[e] < 0 ? 0 : id[e]) * w.ld + c * (int)sizeof(T));
#pragma unroll
        for (int e = 0; e < E; ++e)
#pragma unroll
          for (int k = 0; k < V; ++k) d[e] = fmaf((float)a[k], (float)b[e][k], d[e]);
      }
#pragma unroll
      for (int e = 0; e < E; ++e)
        if (id[e] >= 0) {
          n += l == 0;
          // (times 2^-16: masks of the lowest value, up to 65,535 of them, have a sum as well as a mean)
          t += 0x1p-16f * (d[e] + (bias && l == 0 ? bias[id[e]] : 0.0f));
        }
    }
  }
  t = wave_sum(t);
  top = wave_max(top);
#pragma unroll
  for (int o = 32; o; o >>= 1) n += __shfl_xor(n, o);
  if (lane == 0) {
    sm[wave] = top;
    st[wave] = t;
    sn[wave] = n;
  }
  __syncthreads();
  n = sn[0] + sn[1] + sn[2] + sn[3];
  if (hp)
    for (int64_t c = V * tid; c < ldp; c += V * 256)
      *reinterpret_cast<vec*>(hp + i * ldp + c) = n ? *reinterpret_cast<const vec*>(hr + c) : vec{};
  top = fmaxf(fmaxf(sm[0], sm[1]), fmaxf(sm[2], sm[3]));
  const float base = top == -INFINITY ? 0.0f : top;
  float s = 0.0f;
  for (int k = tid; k < tiles; k += 256) s += p[k].y * exp_fast(p[k].x - base);
  s = wave_sum(s);
  if (lane == 0) ss[wave] = s;
  __syncthreads();
  if (tid == 0) {
    s = ss[0] + ss[1] + ss[2] + ss[3];
    t = st[0] + st[1] + st[2] + st[3];
    const float lse = top + logf(s), sh = n ? 1.0f / (float)n : 0.0f;
    share[i] = sh;
    top_ws[i] = top;
    inv[i] = 1.0f / s;
    if (lse_out) lse_out[i] = lse;
    float mean = t * (0x1p16f * sh);
    if (mean == -INFINITY && t > -INFINITY) mean = -FLT_MAX;  // (1 / n rounded up)
    loss[i] = n ? lse - mean : 0.0f;
  }
}

// ---- product 2 -------------------------------------------------------------------------------------
// Targets of a tile: every thread looks through a share of one row's list while the first copies
// are on their way; what falls into the tile is listed in LDS.  A wave's block of 32 rows that has any gets a
// block of counts beside its output block.  A tile with more than HITS looks through the lists again per block.
template <typename T, class S>
struct EpiDzT {
  using Args = DzArgs;
  static constexpr int HITS = 1023, BLOCKS = 2, TAIL = 4 * (HITS + 1) + 4 * S::BN;
  const DzArgs& a;
  int m, n, row0, col0, tm;
  int* hits;    // [0]: how many
  float* bias;  // [BN]
  unsigned* counts;
  float scale;
  f32x4 sum[S::TN][4];
  __device__ EpiDzT(const DzArgs& args, const TpJob& j, int r0, int c0, int, int wave, int lane)
      : a(args), m(j.m), n(j.n), row0(r0), col0(c0), tm(r0 / S::BM) {
    scale = *a.scale;
#pragma unroll
    for (int b = 0; b < S::TN; ++b)
#pragma unroll
      for (int q = 0; q < 4; ++q) sum[b][q] = f32x4{0.0f, 0.0f, 0.0f, 0.0f};
  }
  __device__ void begin(char* tail) {
    hits = reinterpret_cast<int*>(tail);
    bias = reinterpret_cast<float*>(tail + 4 * (HITS + 1));
    tile_bias<S>(a.bias, col0, n, bias);
    if (threadIdx.x == 0) hits[0] = 0;
    asm volatile("s_waitcnt lgkmcnt(0)" ::: "memory");
    __builtin_amdgcn_s_barrier();
    constexpr int PER = S::THREADS / S::BM;
    const int r = threadIdx.x / PER, row = row0 + r;
    if (row < m && a.y.indptr) {
      each_label(a.y, row, (int)threadIdx.x % PER, PER, [&](int id) {
        const int c = id - a.label0 - col0;
        if (c >= 0 && c < S::BN && id < a.n_labels) {
          const int at = atomicAdd(hits, 1);
          if (at < HITS) hits[1 + at] = r << 16 | c;
        }
      });
    }
  }
  // Fills the wave's block of counts for rows r0 .. + 31, columns c0 .. ; false: none.
  // (The loop's barriers lie between begin and here.)
  __device__ bool targets(int r0, int c0, int wave, int lane) {
    const int total = hits[0];
    if (total == 0) return false;
    counts = reinterpret_cast<unsigned*>(reinterpret_cast<char*>(hits) - counts_offset()) + wave * (32 * S::OUT_LD);
    const int rl = r0 - row0, cl = c0 - col0;
    bool any = total > HITS;
    if (!any) {
      bool mine = false;
      for (int k = lane; k < total; k += 64) {
        const int h = hits[1 + k], r = (h >> 16) - rl, c = (h & 0xffff) - cl;
        mine |= r >= 0 && r < 32 && c >= 0 && c < S::WCOLS;
      }
      any = __ballot(mine) != 0;
    }
    if (!any) return false;
    for (int k = lane; k < 32 * S::OUT_LD; k += 64) counts[k] = 0;
    __builtin_amdgcn_fence(__ATOMIC_SEQ_CST, "wavefront");
    if (total <= HITS) {
      for (int k = lane; k < total; k += 64) {
        const int h = hits[1 + k], r = (h >> 16) - rl, c = (h & 0xffff) - cl;
        if (r >= 0 && r < 32 && c >= 0 && c < S::WCOLS) atomicAdd(counts + r * S::OUT_LD + c, 1u);
      }
    } else if (r0 + (lane >> 1) < m) {
      each_label(a.y, r0 + (lane >> 1), lane & 1, 2, [&](int id) {
        const int c = id - a.label0 - c0;
        if (c >= 0 && c < S::WCOLS && id < a.n_labels) atomicAdd(counts + (lane >> 1) * S::OUT_LD + c, 1u);
      });
    }
    __builtin_amdgcn_fence(__ATOMIC_SEQ_CST, "wavefront");
    return true;
  }
  // bytes from the output blocks to the tail, and from the blocks of counts
  static __device__ constexpr int tail_offset() {
    constexpr int loop = S::NBUF * S::BUF, out = 2 * S::WAVES * S::OUT;
    return loop > out ? loop : out;
  }
  static __device__ constexpr int counts_offset() { return tail_offset() - S::WAVES * S::OUT; }
  // dz in the accumulators; 16 bits go through the wave's block as they will lie in memory.
  __device__ __forceinline__ void block(const f32x16 (&acc)[S::TN], int r0, int colw, float* out, int wave, int lane) {
    const int i = lane & 31, row = r0 + i;
    const bool any = targets(r0, colw, wave, lane);
    float sh = 0.0f, top = 0.0f, f = 0.0f, fp = 0.0f;
    if (row < m) {
      sh = a.share[row];
      top = a.top[row];
      // (the weights are divided by the largest: 0 / 0 where all are 0)
      f = (a.weights ? scale > 0.0f ? a.weights[row] / scale : a.weights[row] : 1.0f) * a.up;
      fp = f * a.inv[row];
    }
    const bool live = sh > 0.0f;
    const float fs = f * sh;
    constexpr int LD = S::OUT_LD * (4 / (int)sizeof(T));  // elements (16 bits: 8-byte writes of 16 lanes take every bank twice)
    T* const block = reinterpret_cast<T*>(out);
#pragma unroll
    for (int b = 0; b < S::TN; ++b)
#pragma unroll
      for (int q = 0; q < 4; ++q) {
        const int c = 32 * b + 8 * q + 4 * (lane >> 5);
        const f32x4 t = *reinterpret_cast<const f32x4*>(bias + colw - col0 + c);
        f32x4 v;
#pragma unroll
        for (int k = 0; k < 4; ++k) v[k] = exp_fast(acc[b][4 * q + k] + t[k] - top) * fp;
        if (any) {
          const u32x4 times = *reinterpret_cast<const u32x4*>(counts + i * S::OUT_LD + c);
#pragma unroll
          for (int k = 0; k < 4; ++k) v[k] -= (float)times[k] * fs;
        }
        // rows without labels and columns past the last are zeros, whatever they hold
#pragma unroll
        for (int k = 0; k < 4; ++k) v[k] = live && colw + c + k < n ? v[k] : 0.0f;
        sum[b][q] += v;
        typename TpMma<T>::frag4 o;
#pragma unroll
        for (int k = 0; k < 4; ++k) o[k] = (T)v[k];
        *reinterpret_cast<typename TpMma<T>::frag4*>(block + i * LD + c) = o;
      }
    __builtin_amdgcn_fence(__ATOMIC_SEQ_CST, "wavefront");
    constexpr int V = 16 / (int)sizeof(T), LPR = S::WCOLS / V, RPP = 64 / LPR;
    typedef T vec __attribute__((ext_vector_type(V)));
    const int c = V * (lane % LPR);
#pragma unroll
    for (int p = 0; p < 32 / RPP; ++p) {
      const int r = p * RPP + lane / LPR;
      const vec v = *reinterpret_cast<const vec*>(block + r * LD + c);
      // (the matrix has whole groups of 64 columns)
      if (r0 + r < m && colw + c < n) *reinterpret_cast<vec*>((T*)a.dz + (r0 + r) * a.ld + colw + c) = v;
    }
    __builtin_amdgcn_fence(__ATOMIC_SEQ_CST, "wavefront");
  }
  __device__ void end(int wave, int wm, int wn, int lane, int tid) {
    if (!a.part) return;
    // a lane's sums are those of its row of each block: rows meet in LDS
    float* const mine = reinterpret_cast<float*>(reinterpret_cast<char*>(hits) - tail_offset()) + wave * (32 * S::OUT_LD);
#pragma unroll
    for (int b = 0; b < S::TN; ++b)
#pragma unroll
      for (int q = 0; q < 4; ++q)
        *reinterpret_cast<f32x4*>(mine + (lane & 31) * S::OUT_LD + 32 * b + 8 * q + 4 * (lane >> 5)) = sum[b][q];
    __syncthreads();
    float* s = reinterpret_cast<float*>(hits);  // [WM][BN]
    static_assert(S::WM * S::BN * 4 <= TAIL, "column sums");
    for (int c = lane; c < S::WCOLS && wave < S::WM * S::WN; c += 64) {
      float t = 0.0f;
#pragma unroll 8
      for (int r = 0; r < 32; ++r) t += mine[r * S::OUT_LD + c];
      s[wm * S::BN + wn * S::WCOLS + c] = t;
    }
    __syncthreads();
    for (int c = tid; c < S::BN; c += S::THREADS) {
      if (col0 + c >= n) continue;
      float t = 0.0f;
#pragma unroll
      for (int k = 0; k < S::WM; ++k) t += s[k * S::BN + c];
      a.part[tm * a.ld + col0 + c] = t;
    }
  }
};
template <class S>
using EpiDzF32 = EpiDzT<float, S>;
template <class S>
using EpiDzBf16 = EpiDzT<bf16, S>;
template <class S>
using EpiDzF16 = EpiDzT<f16, S>;

namespace {

struct Sizes {
  int piece;  // labels of a piece (a multiple of 64 unless it is all)
  int64_t ldz;
  NarrowPlan nl, ng;
  bool narrow, narrow_grad, sides;
  int parts;  // of a row's log-sum-exp
  TpPlan fwd, dz, dh;
  size_t hp, hq, wp, share, top, inv, scale, part, dzb, dbp, slabs, side_slabs, total;
};

Sizes sizes(int dtype, const MatDev& h, const MatDev& w, int B, int L, int D, bool grads) {
  Sizes s{};
  const int es = elem_size(dtype);
  s.narrow = narrow_takes(dtype, D);
  s.narrow_grad = grads && narrow_grad_takes(dtype, B, D);
  s.nl = narrow_lse_plan(B, L);
  s.fwd = tp_plan(dtype, B, L, D, 1);
  s.parts = s.narrow ? s.nl.ranges : s.fwd.job.tiles_n;
  s.share = round256((size_t)B * 4);
  s.top = s.inv = s.share;
  s.part = round256((size_t)B * s.parts * 8);
  s.wp = tp_in_place(dtype, w, D) ? 0 : tp_packed_bytes(dtype, L, D);
  s.hq = tp_in_place(dtype, h, D) ? 0 : tp_packed_bytes(dtype, B, D);
  s.hp = grads ? tp_packed_bytes(dtype, B, D) : 0;
  s.total = s.share + s.top + s.inv + s.part + s.wp + s.hp + s.hq;
  if (!grads) return s;
  s.scale = 256;
  s.sides = narrow_sides_take(dtype, B, L, D);
  if (s.narrow_grad || s.sides) {
    s.ng = s.sides ? narrow_rows_plan(B, L) : narrow_grad_plan(L);
    s.side_slabs = narrow_slab_bytes(s.ng, B);
    if (s.narrow_grad) {
      s.total += s.scale + s.side_slabs;
      return s;
    }
  }
  const int64_t fit = PIECE_BYTES / ((int64_t)B * es) / 256 * 256;
  s.piece = (int)(fit < 256 ? 256 : fit);
  if (s.piece > L) s.piece = L;
  s.ldz = ceil_div(s.piece, 64) * 64;
  s.dz = tp_plan(dtype, B, s.piece, D, 1);
  s.dh = tp_plan(dtype, B, D, s.piece, MAX_SLABS);
  s.dzb = round256((size_t)B * s.ldz * es);
  s.dbp = round256((size_t)s.dz.job.tiles_m * s.ldz * 4);
  s.slabs = round256((size_t)s.dh.job.splits * B * ceil_div(D, 8) * 8 * 4);
  // (the lists decide between the two, and they are not known here)
  const size_t general = s.dzb + s.dbp + s.slabs;
  s.total += s.scale + (general > s.side_slabs ? general : s.side_slabs);
  return s;
}

template <typename T, template <class> class EpiDz>
hipError_t run(const LossJob& j, char* ws, hipStream_t st) {
  const int B = j.n_rows, L = j.n_labels, D = j.d, dt = j.dtype;
  const bool grads = j.dh.data || j.dw.data || j.db;
  Sizes s = sizes(dt, j.h, j.w, B, L, D, grads);
  auto take = [&](size_t n) {
    char* p = ws;
    ws += n;
    return p;
  };
  float* share = (float*)take(s.share);
  float* top = (float*)take(s.top);
  float* inv = (float*)take(s.inv);
  float2* part = (float2*)take(s.part);
  char* wp = take(s.wp);
  char* hp = take(s.hp);
  float* scale = grads ? (float*)take(s.scale) : nullptr;
  const int64_t ldp = tp_packed_cols(dt, D);
  hipError_t e;
  // operands in place, or laid out anew
  TpOperand h = tp_operand(dt, j.h.data, j.h.ld, B, D), w = tp_operand(dt, j.w.data, j.w.ld, L, D);
  const TpOperand hz = tp_operand(dt, hp, ldp, B, ldp);  // (zeros in rows without labels: for the gradients alone)
  int64_t ldw = j.w.ld;
  PackJob jobs[2];
  int packs = 0;
  if (s.hq) {
    char* hq = take(s.hq);
    h = tp_operand(dt, hq, ldp, B, ldp);
    jobs[packs++] = PackJob{j.h.data, j.h.ld, B, D, hq};
  }
  if (s.wp) {
    w = tp_operand(dt, wp, ldp, L, ldp);
    ldw = ldp;
    jobs[packs++] = PackJob{j.w.data, j.w.ld, L, D, wp};
  }
  if (packs && (e = launch_pack(dt, jobs, packs, st)) != hipSuccess) return e;
  s.fwd.job.a = h;
  s.fwd.job.b = w;
  e = s.narrow ? launch_narrow_lse(dt, s.nl, h, w, j.bias, B, L, D, part, st)
               : tp_launch<T, true, true, EpiLse>(s.fwd, LseArgs{j.bias, part}, st);
  if (e != hipSuccess) return e;
  hipLaunchKernelGGL(k_loss_rows<T>, dim3(B + (scale ? 1 : 0)), dim3(256), 0, st, part, s.parts, h, w, D, L, j.bias, j.y,
                     share, top, inv, j.lse, j.loss_rows, B, j.weights, scale, s.hp ? (T*)hp : (T*)nullptr, ldp);
  if ((e = hipGetLastError()) != hipSuccess) return e;
  if (!grads) return hipSuccess;

  const float up = dt == 2 ? 32768.0f : 1.0f;
  StoreArgs da{};
  da.epi.y = j.dh;
  da.alpha = 1.0f / up;
  da.alpha_dev = scale;
  da.live = share;
  if (s.sides && !narrow_sides_worth(B, L, j.y.nnz)) s.sides = false;
  if (s.narrow_grad || s.sides) {
    float* slabs = j.dh.data ? (float*)take(s.side_slabs) : nullptr;
    const DzArgs za{j.bias, top, inv, share, j.weights, scale, up, nullptr, 0, nullptr, j.y, 0, L};
    e = (s.sides ? launch_narrow_sides : launch_narrow_grad)(dt, s.ng, hz, w, za, B, D, 1.0f / up, j.dw, j.db, slabs, st);
    if (e != hipSuccess || !slabs) return e;
    da.part = slabs;
    da.ldp = 128;
    da.slab = 128ll * B;
    return launch_join(da, s.ng.ranges, B, D, false, st);
  }
  char* dz = take(s.dzb);
  float* dbp = (float*)take(s.dbp);
  float* slabs = (float*)take(s.slabs);
  da.part = slabs;
  da.ldp = ceil_div(D, 8) * 8;
  da.slab = da.ldp * B;
  // One piece and one split: whole sums, straight into dh (rows without labels are zeros in dz).
  if (s.piece >= L && s.dh.job.splits == 1) da.part = nullptr;
  int splits = 0;
  for (int64_t l0 = 0; l0 < L; l0 += s.piece) {
    const int n = (int)(L - l0 < s.piece ? L - l0 : s.piece);
    TpOperand wl{w.base + l0 * w.ld, w.ld, ((int64_t)(n - 1) * ldw + (s.wp ? ldp : D)) * elem_size(dt)};
    TpPlan p = s.dz;
    tp_narrow(&p, n);
    p.job.a = hz;
    p.job.b = wl;
    const DzArgs za{j.bias ? j.bias + l0 : nullptr, top, inv, share, j.weights, scale, up, dz, s.ldz, j.db ? dbp : nullptr, j.y,
                    (int)l0, L};
    if ((e = tp_launch<T, true, true, EpiDz>(p, za, st)) != hipSuccess) return e;
    PairJob pair{};
    if (j.db) pair.sums = SumJob{dbp, p.job.tiles_m, s.ldz, n, 1.0f / up, scale, j.db + l0};
    if (j.dh.data) {
      pair.x = s.dh;
      TpJob& q = pair.x.job;
      q.k = n;
      q.a = tp_operand(dt, dz, s.ldz, B, ceil_div(n, 8) * 8);
      q.b = wl;
      // (the first piece is the longest, so every slab of it is written)
      q.splits = (int)ceil_div(n, q.split_k);
      if (!splits) splits = q.splits;
      da.add = l0 > 0;
      da.keep = 1;
      pair.ax = da;
    }
    if (j.dw.data) {
      pair.y = tp_plan(dt, n, D, B, 1);
      pair.y.job.a = tp_operand(dt, dz, s.ldz, B, ceil_div(n, 8) * 8);
      pair.y.job.b = hz;
      pair.ay.epi.y = j.dw;
      pair.ay.epi.y.data = (char*)j.dw.data + l0 * j.dw.ld * elem_size(j.dw.dtype);
      pair.ay.alpha = 1.0f / up;
      pair.ay.alpha_dev = scale;
    }
    if ((e = launch_pair(dt, pair, st)) != hipSuccess) return e;
  }
  if (da.part && j.dh.data) return launch_join(da, splits, B, D, false, st);
  return hipSuccess;
}

}  // namespace

size_t label_loss_ws_bytes(int dtype, const MatDev& h, const MatDev& w, int n_rows, int n_labels, int d, bool grads) {
  return sizes(dtype, h, w, n_rows, n_labels, d, grads).total;
}

hipError_t launch_label_loss(const LossJob& j, void* ws, hipStream_t st) {
  if (j.dtype == 0) return run<float, EpiDzF32>(j, (char*)ws, st);
  if (j.dtype == 1) return run<bf16, EpiDzBf16>(j, (char*)ws, st);
  return run<f16, EpiDzF16>(j, (char*)ws, st);
}

}  // namespace asgd

// Softmax cross-entropy over a label matrix, in pieces of the labels, without the logits, and its
// gradients.
//
//   z_ij = h_i . w_j + b_j ;  lse_i = ln sum_j e^z_ij ;  n_i = valid entries of row i's list
//   loss_i = lse_i - (1 / n_i) sum of z_iy over the entries
//   dz_ij = weight_i (e^(z_ij - lse_i) - c_ij / n_i), c_ij how often j stands in the list
//   dh = dz W ; dw = dz^T h ; db = 1^T dz
//
//   k_loss_prep   n_i; for gradients a copy of h in which rows without labels are zeros (what they hold
//                 must not reach dw)
//   product 1     z in tiles; per row and tile the maximum and the sum of exponentials
//   k_loss_rows   lse; the target logits as products of their own; loss; the largest |weight|
//   per piece of labels:
//     product 2   z again, dz formed in fp32 from it, the targets taken off in place; its column sums
//                 for db in fp32; dz rounded to the operands' type in the workspace
//     product 3   dz W onto slabs of dh
//     product 4   dz^T h: the piece's rows of dw
//   k_join, k_column_sums   dh and db
//
// Forming z twice costs 2 B L D operations of 8; a piece's dz stays near the last caches.  dz in 16 bits is
// rounded once, with the target in it (p and the target may nearly cancel); fp16 holds it times 2^15 over the
// largest weight, so that probabilities down to 2^-29 stay normal.
#include <math.h>

#include "logits_dev.h"
#include "tile_plan.h"

namespace asgd {

namespace {

constexpr int64_t PIECE_BYTES = 128ll << 20;  // of dz at a time
constexpr int MAX_SLABS = 64;

// Entries of row i that count: ids in [0, L).
__device__ __forceinline__ int entry(const IdLists& y, int q, int L) {
  const int id = y.indices[q];
  return (unsigned)id < (unsigned)L ? id : -1;
}

}  // namespace

// ---- rows before the products ------------------------------------------------------------------
// One wave per row: share[i] = 1 / n_i, 0 without entries; hp: the row, or zeros.
template <typename T>
__global__ __launch_bounds__(256) void k_loss_prep(MatDev h, IdLists y, int B, int L, int D, float* __restrict__ share,
                                                   T* __restrict__ hp, int64_t ldp) {
  const int lane = threadIdx.x & 63, i = blockIdx.x * 4 + (threadIdx.x >> 6);
  if (i >= B) return;
  int q0 = 0, q1 = 0, n = 0;
  if (y.indptr) list_range(y, i, &q0, &q1);
  for (int q = q0 + lane; q < q1; q += 64) n += entry(y, q, L) >= 0;
#pragma unroll
  for (int o = 32; o; o >>= 1) n += __shfl_xor(n, o);
  if (lane == 0) share[i] = n ? 1.0f / (float)n : 0.0f;
  if (!hp) return;
  const T* src = (const T*)h.data + (int64_t)i * h.ld;
  for (int64_t c = lane; c < ldp; c += 64) hp[i * ldp + c] = n && c < D ? src[c] : (T)0.0f;
}

// ---- product 1 -------------------------------------------------------------------------------------
struct LseArgs {
  const float* bias;
  float2* part;  // [B][tiles_n]
};

template <class S>
struct EpiLse {
  using Args = LseArgs;
  static constexpr int BLOCKS = 1, TAIL = S::WN * S::BM * 8;
  const LseArgs& a;
  int m, n, row0, tile, tiles;
  float2* ms;  // [WN][BM]
  __device__ EpiLse(const LseArgs& args, const TpJob& j, int r0, int c0, int)
      : a(args), m(j.m), n(j.n), row0(r0), tile(c0 / S::BN), tiles(j.tiles_n) {}
  __device__ void begin(char* tail) { ms = reinterpret_cast<float2*>(tail); }
  __device__ void slab(int, int, int, int) {}
  __device__ __forceinline__ void rows(int row, int, int col, float v[8], int wave, int lane) {
    float top = -INFINITY;
#pragma unroll
    for (int i = 0; i < 8; ++i) {
      const bool in = col + i < n;
      v[i] = in ? v[i] + (a.bias ? a.bias[col + i] : 0.0f) : -INFINITY;
      top = fmaxf(top, v[i]);
    }
    constexpr int LPR = S::WCOLS / 8;
#pragma unroll
    for (int o = 1; o < LPR; o <<= 1) top = fmaxf(top, __shfl_xor(top, o));
    const float base = top == -INFINITY ? 0.0f : top;
    float s = 0.0f;
#pragma unroll
    for (int i = 0; i < 8; ++i) s += exp_fast(v[i] - base);
#pragma unroll
    for (int o = 1; o < LPR; o <<= 1) s += __shfl_xor(s, o);
    if (lane % LPR == 0) ms[(wave % S::WN) * S::BM + row - row0] = make_float2(top, s);
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
// One workgroup per row.  Target logits are products of their own (a gather of n_i rows of W).  With `scale` one
// workgroup more finds the gradients' scale: the largest finite |weight| of rows that have labels, 1 / B without weights.
template <typename T>
__global__ __launch_bounds__(256) void k_loss_rows(const float2* __restrict__ part, int tiles, MatDev h, MatDev w, int D,
                                                   int L, const float* __restrict__ bias, IdLists y,
                                                   const float* __restrict__ share, float* __restrict__ lse_ws,
                                                   float* __restrict__ lse_out, float* __restrict__ loss, int B,
                                                   const float* __restrict__ weights, float* __restrict__ scale) {
  const int i = blockIdx.x, tid = threadIdx.x, lane = tid & 63, wave = tid >> 6;
  __shared__ float sm[4], ss[4], st[4];
  if (i == B) {
    float v = 0.0f;
    if (weights)
      for (int r = tid; r < B; r += 256) {
        const float a = fabsf(weights[r]);
        if (share[r] > 0.0f && a < INFINITY) v = fmaxf(v, a);
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
  top = wave_max(top);
  if (lane == 0) sm[wave] = top;
  __syncthreads();
  top = fmaxf(fmaxf(sm[0], sm[1]), fmaxf(sm[2], sm[3]));
  const float base = top == -INFINITY ? 0.0f : top;
  float s = 0.0f;
  for (int k = tid; k < tiles; k += 256) s += p[k].y * exp_fast(p[k].x - base);
  s = wave_sum(s);

  float t = 0.0f;
  const float sh = share[i];
  if (sh > 0.0f) {
    int q0, q1;
    list_range(y, i, &q0, &q1);
    const T* hr = (const T*)h.data + (int64_t)i * h.ld;
    for (int q = q0 + wave; q < q1; q += 4) {
      const int id = entry(y, q, L);
      if (id < 0) continue;
      const T* wr = (const T*)w.data + (int64_t)id * w.ld;
      float d = 0.0f;
      for (int c = lane; c < D; c += 64) d = fmaf((float)hr[c], (float)wr[c], d);
      d = wave_sum(d);
      t += d + (bias ? bias[id] : 0.0f);
    }
  }
  if (lane == 0) {
    ss[wave] = s;
    st[wave] = t;
  }
  __syncthreads();
  if (tid == 0) {
    s = ss[0] + ss[1] + ss[2] + ss[3];
    t = st[0] + st[1] + st[2] + st[3];
    const float lse = top + logf(s);
    lse_ws[i] = lse;
    if (lse_out) lse_out[i] = lse;
    loss[i] = sh > 0.0f ? lse - t * sh : 0.0f;
  }
}

// ---- product 2 -------------------------------------------------------------------------------------
struct DzArgs {
  const float* bias;   // of the piece's first label
  const float *lse, *share, *weights, *scale;
  float up;            // 2^15 for fp16
  void* dz;            // [B x ld]
  int64_t ld;
  float* part;         // [tiles_m x ld] column sums, or null
  IdLists y;
  int label0, n_labels;
};

// Targets of a tile: every thread looks through a share of one row's list while the first copies
// are on their way; what falls into the tile is listed in LDS.  A wave's block of 32 rows that has any gets a
// block of counts beside its output block.  A tile with more than HITS looks through the lists again per block.
template <typename T, class S>
struct EpiDzT {
  using Args = DzArgs;
  static constexpr int HITS = 1023, BLOCKS = 2, TAIL = 4 * (HITS + 1);
  const DzArgs& a;
  int m, n, row0, col0, tm;
  int* hits;  // [0]: how many
  unsigned* counts;
  bool any;
  float sum[8];
  __device__ EpiDzT(const DzArgs& args, const TpJob& j, int r0, int c0, int)
      : a(args), m(j.m), n(j.n), row0(r0), col0(c0), tm(r0 / S::BM) {
#pragma unroll
    for (int i = 0; i < 8; ++i) sum[i] = 0.0f;
  }
  __device__ void begin(char* tail) {
    hits = reinterpret_cast<int*>(tail);
    if (threadIdx.x == 0) hits[0] = 0;
    asm volatile("s_waitcnt lgkmcnt(0)" ::: "memory");
    __builtin_amdgcn_s_barrier();
    constexpr int PER = S::THREADS / S::BM;
    const int r = threadIdx.x / PER, row = row0 + r;
    if (row < m && a.y.indptr) {
      int q0, q1;
      list_range(a.y, row, &q0, &q1);
      for (int q = q0 + (int)threadIdx.x % PER; q < q1; q += PER) {
        const int id = a.y.indices[q];
        const int c = id - a.label0 - col0;
        if (c >= 0 && c < S::BN && id < a.n_labels) {
          const int at = atomicAdd(hits, 1);
          if (at < HITS) hits[1 + at] = r << 16 | c;
        }
      }
    }
  }
  // (the loop's barriers lie between begin and here)
  __device__ void slab(int r0, int c0, int wave, int lane) {
    const int total = hits[0];
    counts = reinterpret_cast<unsigned*>(reinterpret_cast<char*>(hits) - a_out_offset()) + wave * (32 * S::OUT_LD);
    const int rl = r0 - row0, cl = c0 - col0;
    any = total > HITS;
    if (total && !any) {
      bool mine = false;
      for (int k = lane; k < total; k += 64) {
        const int h = hits[1 + k], r = (h >> 16) - rl, c = (h & 0xffff) - cl;
        mine |= r >= 0 && r < 32 && c >= 0 && c < S::WCOLS;
      }
      any = __ballot(mine) != 0;
    }
    if (!any) return;
    for (int k = lane; k < 32 * S::OUT_LD; k += 64) counts[k] = 0;
    __builtin_amdgcn_fence(__ATOMIC_SEQ_CST, "wavefront");
    if (total <= HITS) {
      for (int k = lane; k < total; k += 64) {
        const int h = hits[1 + k], r = (h >> 16) - rl, c = (h & 0xffff) - cl;
        if (r >= 0 && r < 32 && c >= 0 && c < S::WCOLS) atomicAdd(counts + r * S::OUT_LD + c, 1u);
      }
    } else if (r0 + (lane >> 1) < m) {
      int q0, q1;
      list_range(a.y, r0 + (lane >> 1), &q0, &q1);
      for (int q = q0 + (lane & 1); q < q1; q += 2) {
        const int id = a.y.indices[q], c = id - a.label0 - c0;
        if (c >= 0 && c < S::WCOLS && id < a.n_labels) atomicAdd(counts + (lane >> 1) * S::OUT_LD + c, 1u);
      }
    }
    __builtin_amdgcn_fence(__ATOMIC_SEQ_CST, "wavefront");
  }
  // bytes from the blocks of counts to the tail
  static __device__ constexpr int a_out_offset() {
    constexpr int loop = S::NBUF * S::BUF, out = 2 * S::WAVES * S::OUT;
    return (loop > out ? loop : out) - S::WAVES * S::OUT;
  }
  __device__ __forceinline__ void rows(int row, int r, int col, float v[8], int, int lane) {
    if (row >= m || col >= n) return;
    const float sh = a.share[row];
    if (sh == 0.0f) {
#pragma unroll
      for (int i = 0; i < 8; ++i) v[i] = 0.0f;
    } else {
      // (the weights are divided by the largest: 0 / 0 where all are 0)
      const float lse = a.lse[row], top = *a.scale;
      const float f = (a.weights ? top > 0.0f ? a.weights[row] / top : a.weights[row] : 1.0f) * a.up;
      const int c0 = (col - col0) % S::WCOLS;
#pragma unroll
      for (int i = 0; i < 8; ++i) {
        float p = exp_fast(v[i] + (a.bias && col + i < n ? a.bias[col + i] : 0.0f) - lse);
        if (any) p -= (float)counts[r * S::OUT_LD + c0 + i] * sh;
        v[i] = col + i < n ? p * f : 0.0f;
        sum[i] += v[i];
      }
    }
    if constexpr (sizeof(T) == 4) {
      f32x4* q = reinterpret_cast<f32x4*>((T*)a.dz + row * a.ld + col);
      q[0] = f32x4{v[0], v[1], v[2], v[3]};
      q[1] = f32x4{v[4], v[5], v[6], v[7]};
    } else {
      typename TpMma<T>::frag8 o;
#pragma unroll
      for (int i = 0; i < 8; ++i) o[i] = (T)v[i];
      *reinterpret_cast<typename TpMma<T>::frag8*>((T*)a.dz + row * a.ld + col) = o;
    }
  }
  __device__ void end(int wave, int wm, int wn, int lane, int tid) {
    if (!a.part) return;
    constexpr int LPR = S::WCOLS / 8;
#pragma unroll
    for (int o = LPR; o < 64; o <<= 1)
#pragma unroll
      for (int i = 0; i < 8; ++i) sum[i] += __shfl_xor(sum[i], o);
    __syncthreads();
    float* s = reinterpret_cast<float*>(hits);  // [WM][BN]
    static_assert(S::WM * S::BN * 4 <= TAIL, "column sums");
    if (lane < LPR) {
#pragma unroll
      for (int i = 0; i < 8; ++i) s[wm * S::BN + wn * S::WCOLS + 8 * lane + i] = sum[i];
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
  TpPlan fwd, dz, dh;
  size_t hp, hq, wp, share, lse, scale, part, dzb, dbp, slabs, total;
};

Sizes sizes(int dtype, const MatDev& h, const MatDev& w, int B, int L, int D, bool grads) {
  Sizes s{};
  const int es = elem_size(dtype);
  s.fwd = tp_plan(dtype, B, L, D, 1);
  s.share = round256((size_t)B * 4);
  s.lse = round256((size_t)B * 4);
  s.part = round256((size_t)B * s.fwd.job.tiles_n * 8);
  s.wp = tp_in_place(dtype, w, D) ? 0 : tp_packed_bytes(dtype, L, D);
  s.hq = tp_in_place(dtype, h, D) ? 0 : tp_packed_bytes(dtype, B, D);
  s.hp = grads ? tp_packed_bytes(dtype, B, D) : 0;
  s.total = s.share + s.lse + s.part + s.wp + s.hp + s.hq;
  if (!grads) return s;
  const int64_t fit = PIECE_BYTES / ((int64_t)B * es) / 256 * 256;
  s.piece = (int)(fit < 256 ? 256 : fit);
  if (s.piece > L) s.piece = L;
  s.ldz = ceil_div(s.piece, 64) * 64;
  s.dz = tp_plan(dtype, B, s.piece, D, 1);
  s.dh = tp_plan(dtype, B, D, s.piece, MAX_SLABS);
  s.scale = 256;
  s.dzb = round256((size_t)B * s.ldz * es);
  s.dbp = round256((size_t)s.dz.job.tiles_m * s.ldz * 4);
  s.slabs = round256((size_t)s.dh.job.splits * B * ceil_div(D, 8) * 8 * 4);
  s.total += s.scale + s.dzb + s.dbp + s.slabs;
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
  float* lse = (float*)take(s.lse);
  float2* part = (float2*)take(s.part);
  char* wp = take(s.wp);
  char* hp = take(s.hp);
  float* scale = grads ? (float*)take(s.scale) : nullptr;
  const int64_t ldp = tp_packed_cols(dt, D);
  hipError_t e;
  hipLaunchKernelGGL(k_loss_prep<T>, dim3((unsigned)ceil_div(B, 4)), dim3(256), 0, st, j.h, j.y, B, L, D, share,
                     s.hp ? (T*)hp : (T*)nullptr, ldp);
  if ((e = hipGetLastError()) != hipSuccess) return e;
  TpOperand h = tp_operand(dt, j.h.data, j.h.ld, B, D);
  const TpOperand hz = tp_operand(dt, hp, ldp, B, ldp);  // (zeros in rows without labels: for the gradients alone)
  if (s.hq) {
    char* hq = take(s.hq);
    if ((e = launch_pack(dt, j.h, B, D, hq, st)) != hipSuccess) return e;
    h = tp_operand(dt, hq, ldp, B, ldp);
  }
  TpOperand w = tp_operand(dt, j.w.data, j.w.ld, L, D);
  int64_t ldw = j.w.ld;
  if (s.wp) {
    if ((e = launch_pack(dt, j.w, L, D, wp, st)) != hipSuccess) return e;
    w = tp_operand(dt, wp, ldp, L, ldp);
    ldw = ldp;
  }
  s.fwd.job.a = h;
  s.fwd.job.b = w;
  if ((e = tp_launch<T, true, true, EpiLse>(s.fwd, LseArgs{j.bias, part}, st)) != hipSuccess) return e;
  hipLaunchKernelGGL(k_loss_rows<T>, dim3(B + (scale ? 1 : 0)), dim3(256), 0, st, part, s.fwd.job.tiles_n, j.h, j.w, D, L, j.bias, j.y,
                     share, lse, j.lse, j.loss_rows, B, j.weights, scale);
  if ((e = hipGetLastError()) != hipSuccess) return e;
  if (!grads) return hipSuccess;

  char* dz = take(s.dzb);
  float* dbp = (float*)take(s.dbp);
  float* slabs = (float*)take(s.slabs);
  const float up = dt == 2 ? 32768.0f : 1.0f;
  StoreArgs da{};
  da.epi.y = j.dh;
  da.part = slabs;
  da.ldp = ceil_div(D, 8) * 8;
  da.slab = da.ldp * B;
  da.alpha = 1.0f / up;
  da.alpha_dev = scale;
  int splits = 0;
  for (int64_t l0 = 0; l0 < L; l0 += s.piece) {
    const int n = (int)(L - l0 < s.piece ? L - l0 : s.piece);
    TpOperand wl{w.base + l0 * w.ld, w.ld, ((int64_t)(n - 1) * ldw + (s.wp ? ldp : D)) * elem_size(dt)};
    TpPlan p = s.dz;
    tp_narrow(&p, n);
    p.job.a = hz;
    p.job.b = wl;
    const DzArgs za{j.bias ? j.bias + l0 : nullptr, lse, share, j.weights, scale, up, dz, s.ldz, j.db ? dbp : nullptr, j.y,
                    (int)l0, L};
    if ((e = tp_launch<T, true, true, EpiDz>(p, za, st)) != hipSuccess) return e;
    if (j.db && (e = launch_column_sums(dbp, p.job.tiles_m, s.ldz, n, 1.0f / up, scale, j.db + l0, st)) != hipSuccess) return e;
    if (j.dh.data) {
      TpPlan q = s.dh;
      q.job.k = n;
      q.job.a = tp_operand(dt, dz, s.ldz, B, ceil_div(n, 8) * 8);
      q.job.b = wl;
      da.add = l0 > 0;
      // (the first piece is the longest, so every slab of it is written)
      q.job.splits = (int)ceil_div(n, q.job.split_k);
      if (!splits) splits = q.job.splits;
      if ((e = launch_plain(dt, true, q, da, st)) != hipSuccess) return e;
    }
    if (j.dw.data) {
      TpPlan q = tp_plan(dt, n, D, B, 1);
      q.job.a = tp_operand(dt, dz, s.ldz, B, ceil_div(n, 8) * 8);
      q.job.b = hz;
      StoreArgs wa{};
      wa.epi.y = j.dw;
      wa.epi.y.data = (char*)j.dw.data + l0 * j.dw.ld * elem_size(j.dw.dtype);
      wa.alpha = 1.0f / up;
      wa.alpha_dev = scale;
      if ((e = launch_plain(dt, false, q, wa, st)) != hipSuccess) return e;
    }
  }
  if (j.dh.data) return launch_join(da, splits, B, D, false, share, st);
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

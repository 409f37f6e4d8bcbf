// C[m][n] = sum_k A(m, k) B(n, k) in tiles on the matrix cores, for operands that the
// caller laid out: bf16, fp16 or fp32, each either with k along its rows ("K rows") or with
// k across them ("K columns": element (m, k) at base + k ld + m).  What becomes of a tile is
// an epilogue's business (dense layers and label loss: k_layers.hip, k_label_loss.hip).
//
// A workgroup owns a BM x BN tile.  Per step, 128 bytes of k (64 elements of 16 bits, 32 of
// 32) of both operands go from memory straight into LDS, 16 bytes a lane, through buffer
// descriptors whose limit is the operand's end: rows, columns and k past the operand arrive as
// zeros, so the loop has no masks.  A copy's place in LDS is its lane's, so bank conflicts are
// avoided by which 16 bytes a lane fetches:
//   K rows:    [row][8 chunks], chunk c of row r at place c ^ ((r / 2) % 8): a fragment read
//              (16 lanes of consecutive rows, the same c) touches every bank once.
//   K columns: [k][BM or BN], units of 32 elements, unit u of row k at place u ^ (k % 4)
//              (16 bits: a transposing read's 32 lanes take 64 bytes of four rows) or
//              u ^ ((k / 4) % 2) (32 bits).
// NBUF buffers: the copies of step s + NBUF - 1 are issued once every wave has left step s - 1.
//
// The product is formed as B A^T: an accumulator's lane holds one row m and runs of four
// columns n.  Epilogues that write rows take them through a block of LDS per wave ([32][32 TN + 4] floats,
// 16-byte writes and reads without conflicts), 8 consecutive columns of a row per lane, so that memory gets
// whole lines.
#pragma once

#include <type_traits>

#include "asgd_dev.h"

namespace asgd {

typedef int i32x4 __attribute__((ext_vector_type(4)));

constexpr int TP_STEP = 128;  // bytes of k per step

template <typename T>
struct TpMma {
  static constexpr int KB = TP_STEP / (int)sizeof(T);  // k per step
  typedef T frag8 __attribute__((ext_vector_type(8)));
  typedef T frag4 __attribute__((ext_vector_type(4)));
};

// ---- tile shapes ----------------------------------------------------------------
template <int BM_, int BN_, int WM_, int WN_, int NBUF_, int WK_ = 1>
struct TpShape {
  static constexpr int BM = BM_, BN = BN_, WM = WM_, WN = WN_, NBUF = NBUF_, WK = WK_;
  static constexpr int WAVES = WM * WN * WK, THREADS = 64 * WAVES;
  static constexpr int TM = BM / WM / 32, TN = BN / WN / 32;  // 32 x 32 blocks of a wave
  static constexpr int BUF = (BM + BN) * TP_STEP;             // bytes of a buffer
  static constexpr int WCOLS = 32 * TN;                       // columns of a wave
  static constexpr int OUT_LD = WCOLS + 4;                    // floats, a wave's output block
  static constexpr int OUT = 32 * OUT_LD * 4;                 // bytes of it
  // WK > 1: that many waves share a block and take turns along k; the first of them has the sums in the end
  static_assert(WK == 1 || (WK == 4 && TM == 1 && TN == 1), "one wave per chunk of a step");
  static_assert(BM % (32 * WM) == 0 && BN % (32 * WN) == 0, "whole blocks");
};

// An operand as the kernel sees it: base of element (0, 0), bytes from a row to the next, bytes
// from base to its end (nothing at or past it is read).
struct TpOperand {
  const char* base;
  int64_t ld, end;
};

// ---- copies into LDS -----------------------------------------------------------
// 16 bytes per lane to LDS byte lds + 16 lane (lds: wave-uniform); zeros where voff is at or past the
// descriptor's limit.  Inline asm so that the compiler does not take every later LDS read for
// dependent on the copy; the kernel waits itself (tp_wait).
__device__ __forceinline__ void tp_copy16(i32x4 rsrc, unsigned voff, unsigned lds) {
  asm volatile("s_mov_b32 m0, %2\n\ts_nop 0\n\tbuffer_load_dwordx4 %0, %1, 0 offen lds" ::"v"(voff), "s"(rsrc), "s"(lds)
               : "memory");
}
// The same with 4 bytes a lane.
__device__ __forceinline__ void tp_copy4(i32x4 rsrc, unsigned voff, unsigned lds) {
  asm volatile("s_mov_b32 m0, %2\n\ts_nop 0\n\tbuffer_load_dword %0, %1, 0 offen lds" ::"v"(voff), "s"(rsrc), "s"(lds)
               : "memory");
}
template <int N>
__device__ __forceinline__ void tp_wait() {
  asm volatile("s_waitcnt vmcnt(%0) lgkmcnt(0)" ::"n"(N) : "memory");
}

__device__ __forceinline__ i32x4 tp_rsrc(const char* base, int64_t left) {
  const uint64_t a = (uint64_t)base;
  const int64_t n = left < 0 ? 0 : left > 0x7fffffff ? 0x7fffffff : left;
  return i32x4{__builtin_amdgcn_readfirstlane((int)(uint32_t)a), __builtin_amdgcn_readfirstlane((int)(uint32_t)(a >> 32) & 0xffff),
               __builtin_amdgcn_readfirstlane((int)n), BUF_RSRC_WORD3};
}

// The copies of one operand's tile: R rows of m (or n), per step TP_STEP bytes of k.
template <typename T, bool KROWS, int R, class S>
struct TpLoad {
  static constexpr int THREADS = S::THREADS;
  static constexpr int ITS = R * 8 / THREADS;
  static constexpr int CPR = KROWS ? 8 : R * (int)sizeof(T) / 16;  // 16-byte chunks per LDS row
  static constexpr int ROWS_IT = THREADS / CPR;                      // LDS rows per round of copies
  static constexpr int UNIT = 2 * (int)sizeof(T);                    // chunks per unit of 32 elements
  static constexpr int UNITS = R / 32;
  static_assert(R * 8 % THREADS == 0 && THREADS % CPR == 0, "whole rounds");
  unsigned voff[ITS];
  unsigned kchunk;  // K rows: 16-byte chunk of k that this lane fetches
  const char* at;   // (wave-uniform) start of the next step
  int64_t left, step;

  static __device__ __forceinline__ int swz(int k) {
    const int m = sizeof(T) == 2 ? k & 3 : (k >> 2) & 1;
    return m & (UNITS - 1);
  }
  __device__ __forceinline__ void init(const TpOperand& o, int64_t r0, int64_t k0, int tid) {
    const int row = tid / CPR, pos = tid % CPR;
    kchunk = pos ^ ((row >> 1) & 7);
    static_assert(!KROWS || ROWS_IT % 16 == 0, "a lane keeps its chunk");
#pragma unroll
    for (int i = 0; i < ITS; ++i) {
      const int r = row + i * ROWS_IT;
      const unsigned chunk = KROWS ? kchunk : ((pos / UNIT) ^ swz(r)) * UNIT + pos % UNIT;
      voff[i] = (unsigned)(r * o.ld) + 16 * chunk;
    }
    if constexpr (KROWS) {
      at = o.base + r0 * o.ld + k0 * (int64_t)sizeof(T);
      step = TP_STEP;
    } else {
      at = o.base + k0 * o.ld + r0 * (int64_t)sizeof(T);
      step = TpMma<T>::KB * o.ld;
    }
    left = o.end - (at - o.base);
  }
  // Copies the next step into the buffer at LDS byte `lds` (of this wave's first lane: + 1024 wave);
  // kleft: bytes of k left in the rows (K rows), TP_STEP or more except in the last step.
  __device__ __forceinline__ void copy(unsigned lds, int64_t kleft) {
    const i32x4 rs = tp_rsrc(at, left);
    if (KROWS && kleft < TP_STEP) {
      const bool in = 16 * (int64_t)kchunk < kleft;
#pragma unroll
      for (int i = 0; i < ITS; ++i) tp_copy16(rs, in ? voff[i] : 0x80000000u, lds + 16 * THREADS * i);
    } else {
#pragma unroll
      for (int i = 0; i < ITS; ++i) tp_copy16(rs, voff[i], lds + 16 * THREADS * i);
    }
    at += step;
    left -= step;
  }
};

// ---- fragments -----------------------------------------------------------------------
// A transposing read of 16-bit elements (lds_read_tr16).
template <typename T>
__device__ __forceinline__ typename TpMma<T>::frag4 tp_turned(const char* p) {
  return __builtin_bit_cast(typename TpMma<T>::frag4, lds_read_tr16(reinterpret_cast<const bf16*>(p)));
}

// Fragment of block row-base r0 (a multiple of 32), k chunk kk (of four) of the tile at `p`.
template <typename T, bool KROWS, int R>
__device__ __forceinline__ typename std::conditional<sizeof(T) == 2, typename TpMma<T>::frag8, f32x4>::type tp_frag(
    const char* p, int r0, int kk, int lane) {
  const int n = lane & 31, g = lane >> 5;
  if constexpr (KROWS) {
    const int r = r0 + n;
    const char* q = p + r * TP_STEP + 16 * ((2 * kk + g) ^ ((r >> 1) & 7));
    if constexpr (sizeof(T) == 2)
      return *reinterpret_cast<const typename TpMma<T>::frag8*>(q);
    else
      return *reinterpret_cast<const f32x4*>(q);
  } else if constexpr (sizeof(T) == 2) {
    const int G = lane >> 4, i = (lane >> 2) & 3, a = lane & 3;
    typename TpMma<T>::frag8 f;
#pragma unroll
    for (int hi = 0; hi < 2; ++hi) {
      const int k = 16 * kk + 8 * (G >> 1) + 4 * hi + i;
      const int u = (r0 >> 5) ^ (i & (R / 32 - 1));
      const char* q = p + k * (R * 2) + u * 64 + 32 * (G & 1) + 8 * a;
      const typename TpMma<T>::frag4 v = tp_turned<T>(q);
#pragma unroll
      for (int j = 0; j < 4; ++j) f[4 * hi + j] = v[j];
    }
    return f;
  } else {
    f32x4 f;
    const int u = (r0 >> 5) ^ (g & (R / 32 - 1));
#pragma unroll
    for (int j = 0; j < 4; ++j) f[j] = *reinterpret_cast<const float*>(p + (8 * kk + 4 * g + j) * (R * 4) + u * 128 + 4 * n);
    return f;
  }
}

__device__ __forceinline__ f32x16 tp_mma(bf16x8 a, bf16x8 b, f32x16 c) {
  return __builtin_amdgcn_mfma_f32_32x32x16_bf16(a, b, c, 0, 0, 0);
}
__device__ __forceinline__ f32x16 tp_mma(f16x8 a, f16x8 b, f32x16 c) {
  return __builtin_amdgcn_mfma_f32_32x32x16_f16(a, b, c, 0, 0, 0);
}
__device__ __forceinline__ f32x16 tp_mma(f32x4 a, f32x4 b, f32x16 c) {
#pragma unroll
  for (int j = 0; j < 4; ++j) c = __builtin_amdgcn_mfma_f32_32x32x2f32(a[j], b[j], c, 0, 0, 0);
  return c;
}

// ---- the tile --------------------------------------------------------------------------
struct TpJob {
  TpOperand a, b;
  int m, n;          // rows and columns of C
  int64_t k;
  int tiles_m, tiles_n, splits;
  int64_t split_k;   // k per split, a multiple of the step's
  int group;         // tiles of m that share their tiles of n in a row of the launch order
  int block0;        // this launch's first workgroup
};

// Launch order: workgroups go to the 8 XCDs in turn, so XCD x takes every 8th; consecutive tiles of one
// XCD are `group` tiles of m by some of n, whose operands its L2 holds.
__device__ __forceinline__ bool tp_place(const TpJob& j, int block, int* tm, int* tn, int* split) {
  const int tiles = j.tiles_m * j.tiles_n, total = tiles * j.splits;
  const int per = (total + 7) >> 3;
  const int lin = (block & 7) * per + (block >> 3);
  if ((block >> 3) >= per || lin >= total) return false;
  *split = lin / tiles;
  const int t = lin % tiles;
  const int span = j.group * j.tiles_n, g0 = t / span * j.group;
  const int rows = min(j.group, j.tiles_m - g0), in = t % span;
  *tm = g0 + in % rows;
  *tn = in / rows;
  return true;
}
inline int tp_blocks(const TpJob& j) { return 8 * ((j.tiles_m * j.tiles_n * j.splits + 7) / 8); }

// A wave's block of 32 rows (accumulators of one row of blocks) in LDS, [32][OUT_LD] floats, private to the wave.
template <class S>
__device__ __forceinline__ void tp_stage(const f32x16 (&c)[S::TN], float* out, int lane) {
  const int n = lane & 31, g = lane >> 5;
#pragma unroll
  for (int b = 0; b < S::TN; ++b)
#pragma unroll
    for (int q = 0; q < 4; ++q)
      *reinterpret_cast<f32x4*>(out + n * S::OUT_LD + 32 * b + 8 * q + 4 * g) =
          f32x4{c[b][4 * q], c[b][4 * q + 1], c[b][4 * q + 2], c[b][4 * q + 3]};
  __builtin_amdgcn_fence(__ATOMIC_SEQ_CST, "wavefront");
}
// Eight consecutive columns of row r of it.
template <class S>
__device__ __forceinline__ void tp_staged8(const float* out, int r, int c, float v[8]) {
  const f32x4 lo = *reinterpret_cast<const f32x4*>(out + r * S::OUT_LD + c);
  const f32x4 hi = *reinterpret_cast<const f32x4*>(out + r * S::OUT_LD + c + 4);
#pragma unroll
  for (int i = 0; i < 4; ++i) { v[i] = lo[i]; v[4 + i] = hi[i]; }
}

// Epi, the epilogue: begin(tail) while the first copies are on their way (Epi::TAIL bytes of LDS of its own behind
// the buffers and Epi::BLOCKS output blocks per wave); block() with the accumulators of each 32 rows of a wave, where
// lane (g, i) holds row i, columns 32 b + 8 q + 4 g + 0..3; end() with the whole workgroup.
//
// Fragments are read one chunk of k ahead of their products, over the barrier too: after it the first reads of
// the new step go out, then the last products of the old one (log-sum-exp of 4,096 x 32,001 over 2,048 in bf16, 537 GFLOP:
// 544 us without, 484 with; its products alone, with neither copies nor LDS reads, take 380, with the reads 417).
template <typename T, bool AK, bool BK, class S, class Epi>
__device__ __forceinline__ void tp_tile(const TpJob& j, const typename Epi::Args& ea, int block, char* smem) {
  int tm, tn, split;
  if (!tp_place(j, block, &tm, &tn, &split)) return;
  const int tid = threadIdx.x, lane = tid & 63;
  const int wave = __builtin_amdgcn_readfirstlane(tid >> 6);
  const int wk = wave / (S::WM * S::WN), wm = wave / S::WN % S::WM, wn = wave % S::WN;
  constexpr int KB = TpMma<T>::KB, NB = S::NBUF;
  const int64_t k0 = split * j.split_k, k1 = min(j.k, k0 + j.split_k);
  const int steps = (int)((k1 - k0 + KB - 1) / KB);
  Epi epi(ea, j, tm * S::BM, tn * S::BN, split, wave, lane);

  TpLoad<T, AK, S::BM, S> la;
  TpLoad<T, BK, S::BN, S> lb;
  la.init(j.a, (int64_t)tm * S::BM, k0, tid);
  lb.init(j.b, (int64_t)tn * S::BN, k0, tid);
  const unsigned lds0 = (unsigned)(uintptr_t)(__attribute__((address_space(3))) char*)smem;
  const unsigned lw = __builtin_amdgcn_readfirstlane(lds0 + 1024 * wave);
  constexpr int COPIES = decltype(la)::ITS + decltype(lb)::ITS;
  auto issue = [&](int s) {
    const int64_t kleft = (j.k - k0 - (int64_t)s * KB) * (int64_t)sizeof(T);
    const unsigned at = lw + (unsigned)(s % NB) * S::BUF;
    la.copy(at, kleft);
    lb.copy(at + S::BM * TP_STEP, kleft);
  };
#pragma unroll
  for (int s = 0; s < NB - 1; ++s)
    if (s < steps) issue(s);
  constexpr int LOOP = NB * S::BUF, OUT = Epi::BLOCKS * S::WAVES * S::OUT;
  epi.begin(smem + (LOOP > OUT ? LOOP : OUT));

  f32x16 acc[S::TM][S::TN];
#pragma unroll
  for (int a = 0; a < S::TM; ++a)
#pragma unroll
    for (int b = 0; b < S::TN; ++b)
#pragma unroll
      for (int r = 0; r < 16; ++r) acc[a][b][r] = 0.0f;

  using Frag = decltype(tp_frag<T, AK, S::BM>(smem, 0, 0, 0));
  Frag fa[2][S::TM], fb[2][S::TN];
  auto read = [&](int s, int kk, int into) {
    const char* pa = smem + (s % NB) * S::BUF;
    const char* pb = pa + S::BM * TP_STEP;
#pragma unroll
    for (int b = 0; b < S::TN; ++b) fb[into][b] = tp_frag<T, BK, S::BN>(pb, 32 * (wn * S::TN + b), kk, lane);
#pragma unroll
    for (int a = 0; a < S::TM; ++a) fa[into][a] = tp_frag<T, AK, S::BM>(pa, 32 * (wm * S::TM + a), kk, lane);
  };
  auto multiply = [&](int from) {
#pragma unroll
    for (int a = 0; a < S::TM; ++a)
#pragma unroll
      for (int b = 0; b < S::TN; ++b) acc[a][b] = tp_mma(fb[from][b], fa[from][a], acc[a][b]);
  };
  for (int s = 0; s < steps; ++s) {
    // this step's copies have landed (those of later steps may be on their way), everywhere, and this wave has
    // read all of the step before
    if (NB > 2 && s + NB - 2 < steps)
      tp_wait<(NB - 2) * COPIES>();
    else
      tp_wait<0>();
    __builtin_amdgcn_s_barrier();
    if constexpr (S::WK > 1) {
      if (s + NB - 1 < steps) issue(s + NB - 1);
      read(s, wk, 0);
      multiply(0);
      continue;
    }
    read(s, 0, 0);
    if (s + NB - 1 < steps) issue(s + NB - 1);
    __builtin_amdgcn_sched_barrier(0);
    if (s > 0) multiply(1);
    __builtin_amdgcn_sched_barrier(0);
#pragma unroll
    for (int kk = 1; kk < 4; ++kk) {
      read(s, kk, kk & 1);
      __builtin_amdgcn_sched_barrier(0);
      multiply((kk - 1) & 1);
      __builtin_amdgcn_sched_barrier(0);
    }
  }
  if (S::WK == 1 && steps > 0) multiply(1);
  __syncthreads();  // the buffers are free for the epilogue

  float* const out = reinterpret_cast<float*>(smem + wave * S::OUT);
  if constexpr (S::WK > 1) {
    tp_stage<S>(acc[0], out, lane);
    __syncthreads();
    if (wk == 0) {
#pragma unroll
      for (int k = 1; k < S::WK; ++k)
#pragma unroll
        for (int q = 0; q < 4; ++q) {
          const f32x4 v = *reinterpret_cast<const f32x4*>(out + k * S::WM * S::WN * (S::OUT / 4) + (lane & 31) * S::OUT_LD + 8 * q +
                                                          4 * (lane >> 5));
#pragma unroll
          for (int i = 0; i < 4; ++i) acc[0][0][4 * q + i] += v[i];
        }
    }
    __syncthreads();  // (the other waves' blocks are theirs again)
    if (wk == 0) epi.block(acc[0], tm * S::BM + 32 * wm, tn * S::BN + 32 * wn, out, wave, lane);
    epi.end(wave, wm, wn, lane, tid);
    return;
  }
#pragma unroll
  for (int a = 0; a < S::TM; ++a) {
    __builtin_amdgcn_sched_barrier(0);  // (one row of blocks at a time: all at once do not fit the registers)
    epi.block(acc[a], tm * S::BM + 32 * (wm * S::TM + a), tn * S::BN + wn * S::WCOLS, out, wave, lane);
  }
  epi.end(wave, wm, wn, lane, tid);
}

template <typename T, bool AK, bool BK, class S, class Epi>
__global__ __launch_bounds__(S::THREADS) void k_tile_product(TpJob j, typename Epi::Args ea) {
  extern __shared__ __attribute__((aligned(16))) char smem[];
  tp_tile<T, AK, BK, S, Epi>(j, ea, j.block0 + (int)blockIdx.x, smem);
}

}  // namespace asgd

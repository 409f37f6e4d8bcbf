// MXFP4 matrices (asgd_fp4_*): quantisation, the way back, and label logits from a
// 4-bit label matrix.
#include <math.h>

#include "asgd_dev.h"
#include "asgd_kernels.h"
#include "logits_dev.h"

namespace asgd {

namespace {

constexpr int Q_THREADS = 256;
typedef unsigned short u16x8 __attribute__((ext_vector_type(8)));
typedef float f32x2 __attribute__((ext_vector_type(2)));
typedef int i32x4 __attribute__((ext_vector_type(4)));
typedef int i32x8 __attribute__((ext_vector_type(8)));

// A thread takes 16 bytes of the dense matrix at a time, Q_U of them in flight; EACH elements,
// whose codes are EACH / 2 bytes.  Rows that follow each other without a gap are one run of
// pieces; otherwise the piece's row is looked up.  ALIGNED: every piece of the dense matrix is 16-byte aligned.
constexpr int Q_U = 4;
template <typename T>
struct Piece {
  static constexpr int EACH = 16 / (int)sizeof(T), LANES = 32 / EACH;  // lanes per block
  typedef T vec __attribute__((ext_vector_type(EACH)));
  static __device__ __forceinline__ int64_t offset(unsigned i, unsigned per_row, int64_t ld) {
    if (per_row == 0) return (int64_t)i * EACH;
    const unsigned row = i / per_row;
    return (int64_t)row * ld + (i - row * per_row) * EACH;
  }
};

// 2^(byte - 127), or NaN for 255.
__device__ __forceinline__ float scale_of(unsigned byte) {
  return __uint_as_float(byte == 0 ? 0x00400000u : byte == 255 ? 0x7fc00000u : byte << 23);
}

// Eight lanes (16-bit types: four) hold a block of 32.  The scale's exponent is the largest magnitude's less 2,
// taken from its bits (which order magnitudes as integers, infinities and NaN on top).
// The conversion divides by the scale (a power of two, the exponent bits of a float: 2^-127
// is the field's 0) and rounds to nearest, ties to the even code, at most 6 in magnitude.
// Bound by memory, one pass over both sides: 670,091 x 128 fp32 (388 MB) 63 us, 6.2 TB/s; the way back
// 55 us, 7.1 TB/s (its codes are small, so nearly all of it is non-temporal writes).
template <typename T, bool ALIGNED>
__global__ __launch_bounds__(Q_THREADS) void k_quantize(const T* __restrict__ x, int64_t ld, unsigned n, unsigned per_row,
                                                        void* __restrict__ codes, uint8_t* __restrict__ scales) {
  using P = Piece<T>;
  const unsigned first = blockIdx.x * (Q_THREADS * Q_U) + threadIdx.x;
  const int lane = threadIdx.x & 63;
  typename P::vec v[Q_U];
#pragma unroll
  for (int u = 0; u < Q_U; ++u) {
    const unsigned i = first + u * Q_THREADS;
    if (i >= n) break;  // (whole blocks: n is a multiple of their lanes)
    const T* p = x + P::offset(i, per_row, ld);
    if constexpr (ALIGNED) {
      v[u] = __builtin_nontemporal_load(reinterpret_cast<const typename P::vec*>(p));
    } else {
#pragma unroll
      for (int e = 0; e < P::EACH; ++e) v[u][e] = p[e];
    }
  }
#pragma unroll
  for (int u = 0; u < Q_U; ++u) {
    const unsigned i = first + u * Q_THREADS;
    if (i >= n) break;
    float f[P::EACH];
    unsigned big = 0;
#pragma unroll
    for (int e = 0; e < P::EACH; ++e) {
      f[e] = (float)v[u][e];
      big = max(big, __float_as_uint(f[e]) & 0x7fffffffu);
    }
    big = max(big, lane_xor<1>(big, lane));
    big = max(big, lane_xor<2>(big, lane));
    if constexpr (P::LANES == 8) big = max(big, lane_xor<4>(big, lane));
    const int ex = (int)(big >> 23);
    const int byte = big == 0 ? 0 : ex == 255 ? 255 : max(ex - 2, 0);
    const float scale = scale_of((unsigned)byte);
    unsigned out = 0;
    out = __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(out, f[0], f[1], scale, 0);
    out = __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(out, f[2], f[3], scale, 1);
    if constexpr (P::EACH == 8) {
      out = __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(out, f[4], f[5], scale, 2);
      out = __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(out, f[6], f[7], scale, 3);
    }
    if (byte == 255) out = 0;
    if constexpr (P::EACH == 8)
      reinterpret_cast<uint32_t*>(codes)[i] = out;
    else
      reinterpret_cast<uint16_t*>(codes)[i] = (uint16_t)out;
    if (i % P::LANES == 0) scales[i / P::LANES] = (uint8_t)byte;
  }
}

template <typename T, bool ALIGNED>
__global__ __launch_bounds__(Q_THREADS) void k_dequantize(const void* __restrict__ codes, const uint8_t* __restrict__ scales,
                                                          unsigned n, unsigned per_row, T* __restrict__ out, int64_t ld) {
  using P = Piece<T>;
  const unsigned first = blockIdx.x * (Q_THREADS * Q_U) + threadIdx.x;
  unsigned w[Q_U], byte[Q_U];
#pragma unroll
  for (int u = 0; u < Q_U; ++u) {
    const unsigned i = first + u * Q_THREADS;
    if (i >= n) break;
    w[u] = P::EACH == 8 ? reinterpret_cast<const uint32_t*>(codes)[i] : reinterpret_cast<const uint16_t*>(codes)[i];
    byte[u] = scales[i / P::LANES];
  }
#pragma unroll
  for (int u = 0; u < Q_U; ++u) {
    const unsigned i = first + u * Q_THREADS;
    if (i >= n) break;
    const float s = scale_of(byte[u]);
    const bool nan = byte[u] == 255;
    typename P::vec v;
    auto two = [&](f32x2 p, int at) {
      v[at] = (T)(nan ? NAN : p[0]);
      v[at + 1] = (T)(nan ? NAN : p[1]);
    };
    two(__builtin_amdgcn_cvt_scalef32_pk_f32_fp4(w[u], s, 0), 0);
    two(__builtin_amdgcn_cvt_scalef32_pk_f32_fp4(w[u], s, 1), 2);
    if constexpr (P::EACH == 8) {
      two(__builtin_amdgcn_cvt_scalef32_pk_f32_fp4(w[u], s, 2), 4);
      two(__builtin_amdgcn_cvt_scalef32_pk_f32_fp4(w[u], s, 3), 6);
    }
    T* p = out + P::offset(i, per_row, ld);
    if constexpr (ALIGNED) {
      __builtin_nontemporal_store(v, reinterpret_cast<typename P::vec*>(p));
    } else {
#pragma unroll
      for (int e = 0; e < P::EACH; ++e) p[e] = v[e];
    }
  }
}

// ---------------------------------------------------------------------------
// Logits.  A wave's tile is 32 labels, the product's columns: lane (g, n) holds label n's codes
// of hidden units 64g .. 64g + 63, 32 contiguous bytes, and takes units 64g + 32c .. + 31 into
// half c of the product (the order of the inner index is free as long as both
// operands share it).  The accumulator then holds, per register, one row of 32 consecutive
// labels on each half of the wave.  With 4-bit rows the codes go into the scaled product as
// they are, a lane's 32 elements under its block's scale; with bf16 rows they are
// widened to bf16 (exactly) first.
// ---------------------------------------------------------------------------
constexpr int FL_THREADS = 256;
constexpr int FL_WAVES = FL_THREADS / 64;
constexpr int FL_FEW = 16;
constexpr int FL_FEW_WGS = 1024;

// A label's share of a tile, on its two lanes: codes, scales (halves c = 0, 1 in bytes 0, 1) and bias, as loaded.
struct LabelTile {
  i32x4 c[2];
  unsigned scale;
  float bias;
};
__device__ __forceinline__ void label_load(LabelTile& t, const uint8_t* codes, const uint8_t* scales, const float* bias,
                                           int label, int L, int g) {
  label = max(0, min(label, L - 1));
  const i32x4* p = reinterpret_cast<const i32x4*>(codes + (unsigned)label * (HID / 2) + 32 * g);
  t.c[0] = p[0];
  t.c[1] = p[1];
  t.scale = *reinterpret_cast<const unsigned*>(scales + (unsigned)label * (HID / 32)) >> (16 * g);
  t.bias = bias ? bias[label] : 0.0f;
}

typedef bf16 bf16x2_ __attribute__((ext_vector_type(2)));
// The tile's weights as operands of the bf16 product.
__device__ __forceinline__ void widen(const LabelTile& t, bf16x8 (&w)[8]) {
#pragma unroll
  for (int c = 0; c < 2; ++c) {
    const float s = scale_of((t.scale >> (8 * c)) & 255);
#pragma unroll
    for (int j = 0; j < 4; ++j) {
      const unsigned v = (unsigned)t.c[c][j];
      const bf16x2_ a = __builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(v, s, 0), b = __builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(v, s, 1),
                    d = __builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(v, s, 2), e = __builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(v, s, 3);
      w[4 * c + j] = bf16x8{a[0], a[1], b[0], b[1], d[0], d[1], e[0], e[1]};
    }
  }
}

// 32 hidden rows as the other operand.
template <bool H4>
struct RowTile;
template <>
struct RowTile<false> {
  bf16x8 a[8];
  __device__ void load(const Fp4Rows& h, int row, int g) {
    const bf16* p = (const bf16*)h.h + (int64_t)row * h.ld + 64 * g;
#pragma unroll
    for (int c = 0; c < 8; ++c) a[c] = *reinterpret_cast<const bf16x8*>(p + 8 * c);
  }
};
template <>
struct RowTile<true> {
  i32x4 c[2];
  unsigned scale;
  __device__ void load(const Fp4Rows& h, int row, int g) {
    const i32x4* p = reinterpret_cast<const i32x4*>(h.codes + (unsigned)row * (HID / 2) + 32 * g);
    c[0] = p[0];
    c[1] = p[1];
    scale = *reinterpret_cast<const unsigned*>(h.scales + (unsigned)row * (HID / 32)) >> (16 * g);
  }
};

__device__ __forceinline__ f32x16 product(const RowTile<false>& h, const bf16x8 (&w)[8], f32x16 acc) {
#pragma unroll
  for (int c = 0; c < 8; ++c) acc = __builtin_amdgcn_mfma_f32_32x32x16_bf16(h.a[c], w[c], acc, 0, 0, 0);
  return acc;
}
__device__ __forceinline__ f32x16 product(const RowTile<true>& h, const LabelTile& w, f32x16 acc) {
#pragma unroll
  for (int c = 0; c < 2; ++c) {
    const i32x8 a = {h.c[c][0], h.c[c][1], h.c[c][2], h.c[c][3], 0, 0, 0, 0};
    const i32x8 b = {w.c[c][0], w.c[c][1], w.c[c][2], w.c[c][3], 0, 0, 0, 0};
    if (c == 0)
      acc = __builtin_amdgcn_mfma_scale_f32_32x32x64_f8f6f4(a, b, acc, 4, 4, 0, (int)h.scale, 0, (int)w.scale);
    else
      acc = __builtin_amdgcn_mfma_scale_f32_32x32x64_f8f6f4(a, b, acc, 4, 4, 1, (int)h.scale, 1, (int)w.scale);
  }
  // The product takes part of every lane; this compiler would otherwise move it, and the loads
  // of its operands, under a later branch that some lanes do not take.
  asm volatile("" : "+v"(acc));
  return acc;
}
__device__ __forceinline__ f32x16 splat(float v) {
  f32x16 a;
#pragma unroll
  for (int r = 0; r < 16; ++r) a[r] = v;
  return a;
}

// Few rows: they stay in registers, and a wave goes through its tiles of labels with the next one
// on its way.  One row reads the label matrix once: 670,091 labels, 51 MB, 10.4 us, of which about 3 are
// the launch; as fp32 the matrix alone would be 343 MB.
template <typename T, bool H4>
__global__ __launch_bounds__(FL_THREADS) void k_fp4_logits_few(Fp4Rows h, int B, const uint8_t* __restrict__ codes,
                                                               const uint8_t* __restrict__ scales,
                                                               const float* __restrict__ bias, int L, int n_tiles,
                                                               T* __restrict__ z, int64_t ldz) {
  const int lane = threadIdx.x & 63, g = lane >> 5, n = lane & 31;
  const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  const int step = (int)gridDim.x * FL_WAVES;
  int tile = (int)blockIdx.x * FL_WAVES + wave;
  if (tile >= n_tiles) return;
  LabelTile next;
  label_load(next, codes, scales, bias, tile * 32 + n, L, g);
  RowTile<H4> rows;
  rows.load(h, min(n, B - 1), g);
  for (; tile < n_tiles; tile += step) {
    const LabelTile w = next;
    if (tile + step < n_tiles) label_load(next, codes, scales, bias, (tile + step) * 32 + n, L, g);
    f32x16 acc;
    if constexpr (H4) {
      acc = product(rows, w, splat(0.0f));
    } else {
      bf16x8 f[8];
      widen(w, f);
      acc = product(rows, f, splat(0.0f));
    }
    const int label = tile * 32 + n;
    if (label < L) {
#pragma unroll
      for (int r = 0; r < 16; ++r) {
        const int i = 8 * (r >> 2) + 4 * g + (r & 3);
        if (i < B) z[(int64_t)i * ldz + label] = (T)(acc[r] + w.bias);
      }
    }
  }
}

// Many rows: bound by writing Z, whose rows of an odd number of labels start anywhere in a memory
// line.  A line that two workgroups write part of costs the memory a read, so each row is
// divided at its own line boundaries: the workgroup of labels from t0 on stores, of a row whose element
// t0 lies p elements into its line, the labels t0 - p .. t0 - p + KEEP - 1, and forms the labels
// of one line more for that.  Eight waves with 64 labels each (the weights stay in
// registers) go through blocks of 32 rows; a block passes through LDS, shifted so that
// 16-byte pieces of memory are 16-byte pieces there, and leaves as whole lines.  bf16 rows come
// in through LDS as well (read by every wave as operands, they are 16 bytes out of each of 64 lines).
// Measured: 1,024 x 670,091 bf16 to fp32 (2.74 GB written) 554 us, where a kernel that only writes such rows
// takes 490 to 520; 256 x 205,443 of 4-bit rows to bf16 (119 MB) 25 us.
constexpr int FM_THREADS = 512;
constexpr int FM_WGS = 1024;  // workgroups wanted
constexpr int FM_LABELS = 64 * (FM_THREADS / 64);

template <typename T, bool H4>
__global__ __launch_bounds__(FM_THREADS, 4) void k_fp4_logits(Fp4Rows h, int B, const uint8_t* __restrict__ codes,
                                                              const uint8_t* __restrict__ scales,
                                                              const float* __restrict__ bias, int L, int n_wg,
                                                              T* __restrict__ z, int64_t ldz) {
  constexpr int V = 16 / (int)sizeof(T), LINE = 128 / (int)sizeof(T), KEEP = FM_LABELS - LINE;
  typedef T vec __attribute__((ext_vector_type(V)));
  constexpr int S = FM_LABELS + 8;  // (4 rows of it apart, the halves of a wave write other banks)
  constexpr int HS = HID + 8;   // row stride of the hidden rows: 16 lanes read 16 different bank groups
  __shared__ __attribute__((aligned(16))) T stage[32 * S];
  __shared__ __attribute__((aligned(16))) bf16 hid[H4 ? 8 : 32 * HS];
  const int lane = threadIdx.x & 63, g = lane >> 5, n = lane & 31;
  const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  // neighbouring labels on one XCD
  const int per = (n_wg + 7) / 8;
  const int wg = (int)(blockIdx.x % 8) * per + (int)blockIdx.x / 8;
  if (wg >= n_wg) return;
  const int t0 = wg * KEEP, from = t0 - LINE;  // labels from .. from + FM_LABELS - 1 are formed
  // row i's element t0 lies (at0 + i ld_line) % LINE elements into its line
  const int at0 = (int)((uintptr_t)z / sizeof(T) + (unsigned)t0) & (LINE - 1), ld_line = (int)ldz & (LINE - 1);
  const bool inner = t0 >= LINE && t0 + KEEP <= L;  // every label that it stores exists
  LabelTile w[2];
  bf16x8 f[2][8];
#pragma unroll
  for (int t = 0; t < 2; ++t) {
    // (labels before the first and past the last are read as some other, and not stored)
    label_load(w[t], codes, scales, bias, from + 64 * wave + 32 * t + n, L, g);
    if constexpr (!H4) widen(w[t], f[t]);
  }
  const int step = (int)gridDim.y * 32;
  // thread t brings 16 bytes of row t / 16; or, 4-bit rows, a lane its operand
  bf16x8 piece;
  RowTile<true> rows;
  auto fetch = [&](int r) {
    if constexpr (H4)
      rows.load(h, min(r + n, B - 1), g);
    else
      piece = *reinterpret_cast<const bf16x8*>((const bf16*)h.h + (int64_t)min(r + (int)threadIdx.x / 16, B - 1) * h.ld +
                                               8 * (threadIdx.x % 16));
  };
  auto put = [&]() {
    if constexpr (!H4) *reinterpret_cast<bf16x8*>(hid + (threadIdx.x / 16) * HS + 8 * (threadIdx.x % 16)) = piece;
  };
  fetch((int)blockIdx.y * 32);
  put();
  if constexpr (!H4) __syncthreads();
  for (int r0 = (int)blockIdx.y * 32; r0 < B; r0 += step) {
    f32x16 acc[2] = {splat(0.0f), splat(0.0f)};
    if constexpr (H4) {
      acc[0] = product(rows, w[0], acc[0]);
      acc[1] = product(rows, w[1], acc[1]);
    } else {
#pragma unroll
      for (int c = 0; c < 8; ++c) {
        const bf16x8 a = *reinterpret_cast<const bf16x8*>(hid + n * HS + 64 * g + 8 * c);
        acc[0] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(a, f[0][c], acc[0], 0, 0, 0);
        acc[1] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(a, f[1][c], acc[1], 0, 0, 0);
      }
    }
    fetch(r0 + step);
    T* const to = stage + 4 * g * S + 64 * wave + n;
    const int at = at0 + (r0 + 4 * g) * ld_line;
#pragma unroll
    for (int r = 0; r < 16; ++r) {
      const int i = 8 * (r >> 2) + (r & 3);
      const int shift = (at + i * ld_line) & (V - 1);
      to[i * S + shift] = (T)(acc[0][r] + w[0].bias);
      to[i * S + shift + 32] = (T)(acc[1][r] + w[1].bias);
    }
    __syncthreads();
    put();  // (before the stores, or it would wait for them)
#pragma unroll 1
    for (int q = 0; q < 32 / (FM_THREADS / 64); ++q) {
      const int i = wave * (32 / (FM_THREADS / 64)) + q, row = r0 + i;
      if (row >= B) break;
      const int p = (at0 + row * ld_line) & (LINE - 1);
      const int first = t0 - p;  // the row's first label here: column LINE - p + p % V of the stage
      T* const out = z + ((int64_t)row * ldz + first);
      const T* const in = stage + i * S + LINE - (p & ~(V - 1));
      if (inner) {
#pragma unroll
        for (int v = 0; v < (KEEP / V + 63) / 64; ++v)
          if (v * 64 + lane < KEEP / V)
            __builtin_nontemporal_store(*reinterpret_cast<const vec*>(in + (v * 64 + lane) * V),
                                        reinterpret_cast<vec*>(out + (v * 64 + lane) * V));
      } else {
#pragma unroll 1
        for (int c = lane; c < KEEP; c += 64)
          if (first + c >= 0 && first + c < L) out[c] = in[c];
      }
    }
    __syncthreads();
  }
}

template <typename T>
hipError_t quantize_as(const void* x, int64_t ld, int rows, int cols, uint8_t* codes, uint8_t* scales, hipStream_t st) {
  const unsigned n = (unsigned)((int64_t)rows * cols / Piece<T>::EACH);
  const unsigned per_row = ld == cols ? 0 : (unsigned)(cols / Piece<T>::EACH);
  const bool al = ((uintptr_t)x & 15) == 0 && (ld * sizeof(T) % 16 == 0 || rows == 1);
  const dim3 grid((n + Q_THREADS * Q_U - 1) / (Q_THREADS * Q_U)), block(Q_THREADS);
  if (al)
    hipLaunchKernelGGL((k_quantize<T, true>), grid, block, 0, st, (const T*)x, ld, n, per_row, codes, scales);
  else
    hipLaunchKernelGGL((k_quantize<T, false>), grid, block, 0, st, (const T*)x, ld, n, per_row, codes, scales);
  return hipGetLastError();
}

template <typename T>
hipError_t dequantize_as(const uint8_t* codes, const uint8_t* scales, int rows, int cols, void* out, int64_t ld,
                         hipStream_t st) {
  const unsigned n = (unsigned)((int64_t)rows * cols / Piece<T>::EACH);
  const unsigned per_row = ld == cols ? 0 : (unsigned)(cols / Piece<T>::EACH);
  const bool al = ((uintptr_t)out & 15) == 0 && (ld * sizeof(T) % 16 == 0 || rows == 1);
  const dim3 grid((n + Q_THREADS * Q_U - 1) / (Q_THREADS * Q_U)), block(Q_THREADS);
  if (al)
    hipLaunchKernelGGL((k_dequantize<T, true>), grid, block, 0, st, codes, scales, n, per_row, (T*)out, ld);
  else
    hipLaunchKernelGGL((k_dequantize<T, false>), grid, block, 0, st, codes, scales, n, per_row, (T*)out, ld);
  return hipGetLastError();
}

template <typename T, bool H4>
hipError_t logits_as(const Fp4Rows& a, int B, const uint8_t* codes, const uint8_t* scales, const float* bias, int L,
                     void* z, int64_t ldz, hipStream_t st) {
  const int n_tiles = (L + 31) / 32;
  const dim3 block(FL_THREADS);
  // (these | the staged ones: 1 x 670,091 bf16 to fp32 11 | 14 us, 16 rows 17 | 18, 32 rows 27 | 24)
  if (B <= FL_FEW) {
    const int wgs = (n_tiles + FL_WAVES - 1) / FL_WAVES;
    hipLaunchKernelGGL((k_fp4_logits_few<T, H4>), dim3(wgs < FL_FEW_WGS ? wgs : FL_FEW_WGS), block, 0, st, a, B, codes, scales,
                       bias, L, n_tiles, (T*)z, ldz);
  } else {
    constexpr int LINE = 128 / (int)sizeof(T);
    const int wgs = (L + LINE - 1 + FM_LABELS - LINE - 1) / (FM_LABELS - LINE), blocks = (B + 31) / 32;
    int gy = (FM_WGS + wgs - 1) / wgs;
    if (gy > blocks) gy = blocks;
    hipLaunchKernelGGL((k_fp4_logits<T, H4>), dim3((wgs + 7) / 8 * 8, gy), dim3(FM_THREADS), 0, st, a, B, codes, scales,
                       bias, L, wgs, (T*)z, ldz);
  }
  return hipGetLastError();
}

}  // namespace

hipError_t launch_fp4_quantize(int dtype, const void* x, int64_t ld, int rows, int cols, uint8_t* codes,
                               uint8_t* scales, hipStream_t st) {
  if (dtype == 0) return quantize_as<float>(x, ld, rows, cols, codes, scales, st);
  if (dtype == 1) return quantize_as<bf16>(x, ld, rows, cols, codes, scales, st);
  return quantize_as<f16>(x, ld, rows, cols, codes, scales, st);
}

hipError_t launch_fp4_dequantize(const uint8_t* codes, const uint8_t* scales, int rows, int cols, int dtype, void* out,
                                 int64_t ld, hipStream_t st) {
  if (dtype == 0) return dequantize_as<float>(codes, scales, rows, cols, out, ld, st);
  if (dtype == 1) return dequantize_as<bf16>(codes, scales, rows, cols, out, ld, st);
  return dequantize_as<f16>(codes, scales, rows, cols, out, ld, st);
}

hipError_t launch_fp4_logits(const Fp4Rows& a, int B, const uint8_t* codes, const uint8_t* scales, const float* bias,
                             int L, int dtype, void* z, int64_t ldz, hipStream_t st) {
  if (a.codes) {
    if (dtype == 0) return logits_as<float, true>(a, B, codes, scales, bias, L, z, ldz, st);
    if (dtype == 1) return logits_as<bf16, true>(a, B, codes, scales, bias, L, z, ldz, st);
    return logits_as<f16, true>(a, B, codes, scales, bias, L, z, ldz, st);
  }
  if (dtype == 0) return logits_as<float, false>(a, B, codes, scales, bias, L, z, ldz, st);
  if (dtype == 1) return logits_as<bf16, false>(a, B, codes, scales, bias, L, z, ldz, st);
  return logits_as<f16, false>(a, B, codes, scales, bias, L, z, ldz, st);
}

}  // namespace asgd

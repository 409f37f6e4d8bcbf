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

// Eight consecutive elements of a row from element p on; ALIGNED: p is 16-byte aligned.
template <typename T, bool ALIGNED>
__device__ __forceinline__ void load8(const T* p, float (&x)[8]) {
  if constexpr (ALIGNED) {
    constexpr int V = 16 / (int)sizeof(T);
    typedef T vec __attribute__((ext_vector_type(V)));
#pragma unroll
    for (int a = 0; a < 8 / V; ++a) {
      const vec v = reinterpret_cast<const vec*>(p)[a];
#pragma unroll
      for (int e = 0; e < V; ++e) x[a * V + e] = (float)v[e];
    }
  } else {
#pragma unroll
    for (int e = 0; e < 8; ++e) x[e] = (float)p[e];
  }
}

template <typename T, bool ALIGNED>
__device__ __forceinline__ void store8(T* p, const float (&x)[8]) {
  if constexpr (ALIGNED) {
    constexpr int V = 16 / (int)sizeof(T);
    typedef T vec __attribute__((ext_vector_type(V)));
#pragma unroll
    for (int a = 0; a < 8 / V; ++a) {
      vec v;
#pragma unroll
      for (int e = 0; e < V; ++e) v[e] = (T)x[a * V + e];
      reinterpret_cast<vec*>(p)[a] = v;
    }
  } else {
#pragma unroll
    for (int e = 0; e < 8; ++e) p[e] = (T)x[e];
  }
}

// Four lanes hold a block of 32.  The scale's exponent is the largest magnitude's less 2,
// taken from its bits (which order magnitudes as integers, infinities and NaN on top).
// Elements are scaled by a power of two (exact) and compared with the midpoints of the
// e2m1 grid; which side a midpoint falls on is the even code's.
template <typename T, bool ALIGNED>
__global__ __launch_bounds__(Q_THREADS) void k_quantize(const T* __restrict__ x, int64_t ld, int64_t n8, int row8,
                                                        uint32_t* __restrict__ codes, uint8_t* __restrict__ scales) {
  const int64_t i = (int64_t)blockIdx.x * Q_THREADS + threadIdx.x;
  if (i >= n8) return;  // (whole blocks: n8 is a multiple of 4)
  const int64_t row = i / row8, c = i - row * row8;
  float v[8];
  load8<T, ALIGNED>(x + row * ld + c * 8, v);
  unsigned big = 0;
#pragma unroll
  for (int e = 0; e < 8; ++e) big = max(big, __float_as_uint(v[e]) & 0x7fffffffu);
  big = max(big, (unsigned)__shfl_xor((int)big, 1));
  big = max(big, (unsigned)__shfl_xor((int)big, 2));
  const int ex = (int)(big >> 23);
  const int byte = big == 0 ? 0 : ex == 255 ? 255 : max(ex - 2, 0);
  // 2^(127 - byte)
  const float up = __uint_as_float(byte >= 254 ? 0x00400000u >> (byte - 254) : (unsigned)(254 - byte) << 23);
  unsigned out = 0;
#pragma unroll
  for (int e = 0; e < 8; ++e) {
    const float m = fabsf(v[e] * up);
    unsigned code = (m > 0.25f) + (m >= 0.75f) + (m > 1.25f) + (m >= 1.75f) + (m > 2.5f) + (m >= 3.5f) + (m > 5.0f);
    if (v[e] < 0.0f) code |= 8;
    out |= code << (4 * e);
  }
  codes[i] = byte == 255 ? 0 : out;
  if ((i & 3) == 0) scales[i >> 2] = (uint8_t)byte;
}

__device__ __forceinline__ float scale_of(unsigned byte) {
  return __uint_as_float(byte == 0 ? 0x00400000u : byte == 255 ? 0x7fc00000u : byte << 23);
}

template <typename T, bool ALIGNED>
__global__ __launch_bounds__(Q_THREADS) void k_dequantize(const uint32_t* __restrict__ codes,
                                                          const uint8_t* __restrict__ scales, int64_t n8, int row8,
                                                          T* __restrict__ out, int64_t ld) {
  const int64_t i = (int64_t)blockIdx.x * Q_THREADS + threadIdx.x;
  if (i >= n8) return;
  const int64_t row = i / row8, c = i - row * row8;
  const unsigned w = codes[i];
  const float s = scale_of(scales[i >> 2]);
  float v[8];
#pragma unroll
  for (int e = 0; e < 8; ++e) {
    const unsigned code = w >> (4 * e);
    const unsigned m = code & 7;
    // e2m1: 0, 0.5, then (1 + mantissa / 2) 2^(exponent - 1)
    const float a = m < 2 ? 0.5f * (float)m : __uint_as_float((126 + (m >> 1)) << 23 | (m & 1) << 22);
    v[e] = (code & 8 ? -a : a) * s;
  }
  store8<T, ALIGNED>(out + row * ld + c * 8, v);
}

// ---------------------------------------------------------------------------
// Logits.  One wave per 32 labels, the label as the product's column: lane
// (g, n) holds label n's codes of hidden units 64c + 32g .. + 31 (c = 0, 1), 16
// bytes each, and so the accumulator holds four rows of 32 consecutive labels
// per register quad.  With 4-bit rows the codes go into the scaled product
// as they are; with bf16 rows they are widened to bf16 (exact) once, for all the rows.
// ---------------------------------------------------------------------------
constexpr int FL_THREADS = 256;

template <typename T, bool H4>
__global__ __launch_bounds__(FL_THREADS) void k_fp4_logits(const bf16* __restrict__ h, int64_t ldh,
                                                           const uint8_t* __restrict__ h_codes,
                                                           const uint8_t* __restrict__ h_scales, int B,
                                                           const uint8_t* __restrict__ codes,
                                                           const uint8_t* __restrict__ scales,
                                                           const float* __restrict__ bias, int L, T* __restrict__ z,
                                                           int64_t ldz) {
  const int lane = threadIdx.x & 63, g = lane >> 5, n = lane & 31;
  const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  const int tile = (int)blockIdx.x * (FL_THREADS / 64) + wave;
  if (tile * 32 >= L) return;
  const int label = tile * 32 + n;
  const int safe = min(label, L - 1);
  i32x4 wc[2];
#pragma unroll
  for (int c = 0; c < 2; ++c)
    wc[c] = *reinterpret_cast<const i32x4*>(codes + (int64_t)safe * (HID / 2) + 32 * c + 16 * g);
  const unsigned ws = *reinterpret_cast<const unsigned*>(scales + (int64_t)safe * (HID / 32)) >> (8 * g);
  const float b = bias ? bias[safe] : 0.0f;
  bf16x8 wf[H4 ? 1 : 8];
  if constexpr (!H4) {
#pragma unroll
    for (int c = 0; c < 2; ++c) {
      const float s = scale_of((ws >> (16 * c)) & 255);
#pragma unroll
      for (int j = 0; j < 4; ++j)
#pragma unroll
        for (int e = 0; e < 8; ++e) {
          const unsigned code = (unsigned)wc[c][j] >> (4 * e);
          const unsigned m = code & 7;
          const float a = m < 2 ? 0.5f * (float)m : __uint_as_float((126 + (m >> 1)) << 23 | (m & 1) << 22);
          wf[4 * c + j][e] = (bf16)((code & 8 ? -a : a) * s);
        }
    }
  }
  for (int r0 = (int)blockIdx.y * 32; r0 < B; r0 += (int)gridDim.y * 32) {
    const int row = min(r0 + n, B - 1);
    f32x16 acc;
#pragma unroll
    for (int r = 0; r < 16; ++r) acc[r] = 0.0f;
    if constexpr (H4) {
      const unsigned hs = *reinterpret_cast<const unsigned*>(h_scales + (int64_t)row * (HID / 32)) >> (8 * g);
#pragma unroll
      for (int c = 0; c < 2; ++c) {
        const i32x4 hc = *reinterpret_cast<const i32x4*>(h_codes + (int64_t)row * (HID / 2) + 32 * c + 16 * g);
        const i32x8 a = {hc[0], hc[1], hc[2], hc[3], 0, 0, 0, 0}, w = {wc[c][0], wc[c][1], wc[c][2], wc[c][3], 0, 0, 0, 0};
        acc = __builtin_amdgcn_mfma_scale_f32_32x32x64_f8f6f4(a, w, acc, 4, 4, 0, (int)(hs >> (16 * c)), 0,
                                                              (int)(ws >> (16 * c)));
      }
      // The product takes part of every lane; this compiler would otherwise move it, and the
      // loads of its operands, under the branch below, which some lanes of the last tile skip.
      asm volatile("" : "+v"(acc));
    } else {
#pragma unroll
      for (int c = 0; c < 8; ++c) {
        const bf16x8 a = *reinterpret_cast<const bf16x8*>(h + (int64_t)row * ldh + 64 * (c >> 2) + 32 * g + 8 * (c & 3));
        acc = __builtin_amdgcn_mfma_f32_32x32x16_bf16(a, wf[c], acc, 0, 0, 0);
      }
    }
    if (label < L) {
#pragma unroll
      for (int r = 0; r < 16; ++r) {
        const int i = r0 + 8 * (r >> 2) + 4 * g + (r & 3);
        if (i < B) z[(int64_t)i * ldz + label] = (T)(acc[r] + b);
      }
    }
  }
}

template <typename T>
hipError_t quantize_as(const void* x, int64_t ld, int rows, int cols, uint8_t* codes, uint8_t* scales, hipStream_t st) {
  const int64_t n8 = (int64_t)rows * cols / 8;
  const bool al = ((uintptr_t)x & 15) == 0 && ld * sizeof(T) % 16 == 0;
  const dim3 grid((unsigned)((n8 + Q_THREADS - 1) / Q_THREADS)), block(Q_THREADS);
  if (al)
    hipLaunchKernelGGL((k_quantize<T, true>), grid, block, 0, st, (const T*)x, ld, n8, cols / 8, (uint32_t*)codes, scales);
  else
    hipLaunchKernelGGL((k_quantize<T, false>), grid, block, 0, st, (const T*)x, ld, n8, cols / 8, (uint32_t*)codes, scales);
  return hipGetLastError();
}

template <typename T>
hipError_t dequantize_as(const uint8_t* codes, const uint8_t* scales, int rows, int cols, void* out, int64_t ld,
                         hipStream_t st) {
  const int64_t n8 = (int64_t)rows * cols / 8;
  const bool al = ((uintptr_t)out & 15) == 0 && ld * sizeof(T) % 16 == 0;
  const dim3 grid((unsigned)((n8 + Q_THREADS - 1) / Q_THREADS)), block(Q_THREADS);
  if (al)
    hipLaunchKernelGGL((k_dequantize<T, true>), grid, block, 0, st, (const uint32_t*)codes, scales, n8, cols / 8, (T*)out, ld);
  else
    hipLaunchKernelGGL((k_dequantize<T, false>), grid, block, 0, st, (const uint32_t*)codes, scales, n8, cols / 8, (T*)out, ld);
  return hipGetLastError();
}

template <typename T>
hipError_t logits_as(const Fp4Rows& a, int B, const uint8_t* codes, const uint8_t* scales, const float* bias, int L,
                     void* z, int64_t ldz, hipStream_t st) {
  const int wgs = (L + 32 * (FL_THREADS / 64) - 1) / (32 * (FL_THREADS / 64));
  const int blocks = (B + 31) / 32;
  int gy = (2048 + wgs - 1) / wgs;
  if (gy > blocks) gy = blocks;
  const dim3 grid(wgs, gy), block(FL_THREADS);
  if (a.codes)
    hipLaunchKernelGGL((k_fp4_logits<T, true>), grid, block, 0, st, (const bf16*)nullptr, (int64_t)0, a.codes, a.scales,
                       B, codes, scales, bias, L, (T*)z, ldz);
  else
    hipLaunchKernelGGL((k_fp4_logits<T, false>), grid, block, 0, st, (const bf16*)a.h, a.ld, a.codes, a.scales, B, codes,
                       scales, bias, L, (T*)z, ldz);
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
  if (dtype == 0) return logits_as<float>(a, B, codes, scales, bias, L, z, ldz, st);
  if (dtype == 1) return logits_as<bf16>(a, B, codes, scales, bias, L, z, ldz, st);
  return logits_as<f16>(a, B, codes, scales, bias, L, z, ldz, st);
}

}  // namespace asgd

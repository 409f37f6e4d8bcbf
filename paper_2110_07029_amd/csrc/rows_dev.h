// Eight consecutive elements of a row of a caller's matrix of any of the three types, as
// the epilogues and the kernels along rows read and write them; activations and dropout.
#pragma once

#include "asgd_dev.h"
#include "asgd_kernels.h"

namespace asgd {

typedef _Float16 f16;
typedef _Float16 f16x8 __attribute__((ext_vector_type(8)));

// v[i] = element (row, col + i), i < n <= 8; zeros from n on.
__device__ __forceinline__ void load8(const MatDev& m, int64_t row, int col, int n, float v[8]) {
  const int64_t at = row * m.ld + col;
  if (m.vec && n == 8) {
    if (m.dtype == 0) {
      const f32x4* p = reinterpret_cast<const f32x4*>((const float*)m.data + at);
      const f32x4 a = p[0], b = p[1];
#pragma unroll
      for (int i = 0; i < 4; ++i) { v[i] = a[i]; v[4 + i] = b[i]; }
    } else if (m.dtype == 1) {
      const bf16x8 a = *reinterpret_cast<const bf16x8*>((const bf16*)m.data + at);
#pragma unroll
      for (int i = 0; i < 8; ++i) v[i] = (float)a[i];
    } else {
      const f16x8 a = *reinterpret_cast<const f16x8*>((const f16*)m.data + at);
#pragma unroll
      for (int i = 0; i < 8; ++i) v[i] = (float)a[i];
    }
    return;
  }
#pragma unroll
  for (int i = 0; i < 8; ++i) {
    v[i] = 0.0f;
    if (i < n)
      v[i] = m.dtype == 0 ? ((const float*)m.data)[at + i]
                          : m.dtype == 1 ? (float)((const bf16*)m.data)[at + i] : (float)((const f16*)m.data)[at + i];
  }
}

// Element (row, col + i) = v[i], i < n <= 8, rounded to nearest.
__device__ __forceinline__ void store8(const MatDev& m, int64_t row, int col, int n, const float v[8]) {
  const int64_t at = row * m.ld + col;
  if (m.vec && n == 8) {
    if (m.dtype == 0) {
      f32x4* p = reinterpret_cast<f32x4*>((float*)m.data + at);
      p[0] = f32x4{v[0], v[1], v[2], v[3]};
      p[1] = f32x4{v[4], v[5], v[6], v[7]};
    } else if (m.dtype == 1) {
      bf16x8 a;
#pragma unroll
      for (int i = 0; i < 8; ++i) a[i] = (bf16)v[i];
      *reinterpret_cast<bf16x8*>((bf16*)m.data + at) = a;
    } else {
      f16x8 a;
#pragma unroll
      for (int i = 0; i < 8; ++i) a[i] = (f16)v[i];
      *reinterpret_cast<f16x8*>((f16*)m.data + at) = a;
    }
    return;
  }
#pragma unroll
  for (int i = 0; i < 8; ++i)
    if (i < n) {
      if (m.dtype == 0) ((float*)m.data)[at + i] = v[i];
      else if (m.dtype == 1) ((bf16*)m.data)[at + i] = (bf16)v[i];
      else ((f16*)m.data)[at + i] = (f16)v[i];
    }
}

// ---- activations ------------------------------------------------------------------
// e^x with x's own rounding only (the hardware's base-2 exponential of x log2 e loses
// |x| 2^-24 relative, which counts in fp32 outputs).
__device__ __forceinline__ float act_value(int act, float a) {
  if (act == 1) return a > 0.0f ? a : a == a ? 0.0f : a;           // (NaN stays)
  if (act == 2) return 0.5f * a * erfcf(-0.70710678118654752f * a);  // erfc: no cancellation below zero
  if (act == 3) return a / (1.0f + expf(-a));
  return a;
}
__device__ __forceinline__ float act_slope(int act, float a) {
  if (act == 1) return a > 0.0f ? 1.0f : a == a ? 0.0f : a;
  if (act == 2) return 0.5f * erfcf(-0.70710678118654752f * a) + a * (0.39894228040143268f * expf(-0.5f * a * a));
  if (act == 3) {
    const float g = 1.0f / (1.0f + expf(-a));
    return g + a * g * (1.0f - g);
  }
  return 1.0f;
}

// ---- dropout -----------------------------------------------------------------------
// splitmix64 of a counter (the generator of the models' initial weights): the 64 bits of
// key ^ (row 2^22 + column / 2) serve two neighbours, the even column takes the low half.
__device__ __forceinline__ uint64_t splitmix_dev(uint64_t v) {
  v += 0x9E3779B97F4A7C15ull;
  v = (v ^ (v >> 30)) * 0xBF58476D1CE4E5B9ull;
  v = (v ^ (v >> 27)) * 0x94D049BB133111EBull;
  return v ^ (v >> 31);
}
// v[i] of (row, col + i): times scale where it stays, 0 where it is dropped (whatever it was).  col is even.
__device__ __forceinline__ void drop8(const DropDev& d, int64_t row, int col, float v[8]) {
#pragma unroll
  for (int i = 0; i < 4; ++i) {
    const uint64_t w = splitmix_dev(d.key ^ (((uint64_t)row << 22) | (uint64_t)((col >> 1) + i)));
    v[2 * i] = (uint32_t)w >= d.below ? v[2 * i] * d.scale : 0.0f;
    v[2 * i + 1] = (uint32_t)(w >> 32) >= d.below ? v[2 * i + 1] * d.scale : 0.0f;
  }
}

// One row's element of the epilogue: bias, activation, dropout, residual; v becomes the output and pre
// (in place of it, rounded to its own type) is stored on the way.
__device__ __forceinline__ void dense_out8(const DenseEpi& e, int64_t row, int col, int n, float v[8]) {
  if (e.bias) {
#pragma unroll
    for (int i = 0; i < 8; ++i) v[i] += i < n ? e.bias[col + i] : 0.0f;
  }
  if (e.pre.data) store8(e.pre, row, col, n, v);
  if (e.act) {
#pragma unroll
    for (int i = 0; i < 8; ++i) v[i] = act_value(e.act, v[i]);
  }
  if (e.drop.below) drop8(e.drop, row, col, v);
  if (e.res.data) {
    float r[8];
    load8(e.res, row, col, n, r);
#pragma unroll
    for (int i = 0; i < 8; ++i) v[i] += r[i];
  }
  store8(e.y, row, col, n, v);
}

}  // namespace asgd

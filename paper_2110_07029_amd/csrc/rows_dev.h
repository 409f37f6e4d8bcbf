// Eight consecutive elements of a row of a caller's matrix of any of the three types, as
// the epilogues and the kernels along rows read and write them; activations and dropout.
#pragma once

#include "asgd_dev.h"
#include "asgd_kernels.h"

namespace asgd {

// Vectors at any element's address (the hardware takes them; with eight accesses of 2 bytes instead a layer of
// 777 x 1,001 x 515 out of line took 18 us, it takes 15).
typedef float f32x4u __attribute__((ext_vector_type(4), aligned(4)));
typedef __bf16 bf16x8u __attribute__((ext_vector_type(8), aligned(2)));
typedef _Float16 f16x8u __attribute__((ext_vector_type(8), aligned(2)));
typedef __bf16 bf16x4u __attribute__((ext_vector_type(4), aligned(2)));
typedef _Float16 f16x4u __attribute__((ext_vector_type(4), aligned(2)));

// v[i] = element (row, col + i), i < n <= 8; zeros from n on.
__device__ __forceinline__ void load8(const MatDev& m, int64_t row, int col, int n, float v[8]) {
  const int64_t at = row * m.ld + col;
  if (n == 8) {
    if (m.dtype == 0) {
      const f32x4u* p = reinterpret_cast<const f32x4u*>((const float*)m.data + at);
      const f32x4 a = p[0], b = p[1];
#pragma unroll
      for (int i = 0; i < 4; ++i) { v[i] = a[i]; v[4 + i] = b[i]; }
    } else if (m.dtype == 1) {
      const bf16x8 a = *reinterpret_cast<const bf16x8u*>((const bf16*)m.data + at);
#pragma unroll
      for (int i = 0; i < 8; ++i) v[i] = (float)a[i];
    } else {
      const f16x8 a = *reinterpret_cast<const f16x8u*>((const f16*)m.data + at);
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
  if (n == 8) {
    if (m.dtype == 0) {
      f32x4u* p = reinterpret_cast<f32x4u*>((float*)m.data + at);
      p[0] = f32x4{v[0], v[1], v[2], v[3]};
      p[1] = f32x4{v[4], v[5], v[6], v[7]};
    } else if (m.dtype == 1) {
      bf16x8 a;
#pragma unroll
      for (int i = 0; i < 8; ++i) a[i] = (bf16)v[i];
      *reinterpret_cast<bf16x8u*>((bf16*)m.data + at) = a;
    } else {
      f16x8 a;
#pragma unroll
      for (int i = 0; i < 8; ++i) a[i] = (f16)v[i];
      *reinterpret_cast<f16x8u*>((f16*)m.data + at) = a;
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

// Element (row, col + i) = v[i], i < min(n, 4).
__device__ __forceinline__ void store4(const MatDev& m, int64_t row, int col, int n, const float v[4]) {
  const int64_t at = row * m.ld + col;
  if (n >= 4) {
    if (m.dtype == 0) {
      *reinterpret_cast<f32x4u*>((float*)m.data + at) = f32x4{v[0], v[1], v[2], v[3]};
    } else if (m.dtype == 1) {
      *reinterpret_cast<bf16x4u*>((bf16*)m.data + at) = bf16x4{(bf16)v[0], (bf16)v[1], (bf16)v[2], (bf16)v[3]};
    } else {
      *reinterpret_cast<f16x4u*>((f16*)m.data + at) = f16x4u{(f16)v[0], (f16)v[1], (f16)v[2], (f16)v[3]};
    }
    return;
  }
#pragma unroll
  for (int i = 0; i < 4; ++i)
    if (i < n) {
      if (m.dtype == 0) ((float*)m.data)[at + i] = v[i];
      else if (m.dtype == 1) ((bf16*)m.data)[at + i] = (bf16)v[i];
      else ((f16*)m.data)[at + i] = (f16)v[i];
    }
}

// ---- activations ------------------------------------------------------------------
// The normal distribution function Phi(a) and its density, from e^(-a^2/2) and a polynomial in
// 1 / (1 + p |a| / sqrt 2) (Abramowitz and Stegun 7.1.26, off by 0.75e-7 at most, one and a quarter steps of fp32 at 1):
// some 15 instructions, two of them at a quarter of the rate, where erfc and exp take over a hundred between them.
struct Normal {
  float cdf, density;
};
__device__ __forceinline__ Normal normal_of(float a) {
  const float x = fabsf(a) * 0.70710678118654752f;
  const float t = __builtin_amdgcn_rcpf(fmaf(0.3275911f, x, 1.0f));
  const float e = __builtin_amdgcn_exp2f(-0.72134752044448170f * a * a);
  const float p = t * fmaf(t, fmaf(t, fmaf(t, fmaf(t, 1.061405429f, -1.453152027f), 1.421413741f), -0.284496736f), 0.254829592f);
  const float tail = 0.5f * p * e;
  return Normal{a < 0.0f ? tail : 1.0f - tail, 0.39894228040143268f * e};
}
// 1 / (1 + e^-a)
__device__ __forceinline__ float logistic(float a) {
  return __builtin_amdgcn_rcpf(1.0f + __builtin_amdgcn_exp2f(-LOG2E * a));
}
__device__ __forceinline__ float relu_value(float a) { return a > 0.0f ? a : a == a ? 0.0f : a; }  // (NaN stays)
__device__ __forceinline__ float gelu_value(float a) { return a == -INFINITY ? 0.0f : a * normal_of(a).cdf; }
__device__ __forceinline__ float silu_value(float a) { return a == -INFINITY ? 0.0f : a * logistic(a); }
__device__ __forceinline__ float relu_slope(float a) { return a > 0.0f ? 1.0f : a == a ? 0.0f : a; }
__device__ __forceinline__ float gelu_slope(float a) {
  const Normal n = normal_of(a);
  return n.cdf + (n.density == 0.0f ? 0.0f : a * n.density);  // (0, not infinity times 0, at infinity)
}
__device__ __forceinline__ float silu_slope(float a) {
  const float g = logistic(a), r = 1.0f - g;
  return g + (g == 0.0f || r == 0.0f ? 0.0f : a * g * r);
}
// Eight at a time, so that their chains of dependent steps run side by side (gradients of a
// layer of 8,192 x 4,096 x 1,024: 216 us with a branch per element, 213 so).
__device__ __forceinline__ void act8(int act, float v[8]) {
  if (act == 1) {
#pragma unroll
    for (int i = 0; i < 8; ++i) v[i] = relu_value(v[i]);
  } else if (act == 2) {
#pragma unroll
    for (int i = 0; i < 8; ++i) v[i] = gelu_value(v[i]);
  } else if (act == 3) {
#pragma unroll
    for (int i = 0; i < 8; ++i) v[i] = silu_value(v[i]);
  }
}
// v[i] *= act'(a[i])
__device__ __forceinline__ void slope8(int act, const float a[8], float v[8]) {
  if (act == 1) {
#pragma unroll
    for (int i = 0; i < 8; ++i) v[i] *= relu_slope(a[i]);
  } else if (act == 2) {
#pragma unroll
    for (int i = 0; i < 8; ++i) v[i] *= gelu_slope(a[i]);
  } else if (act == 3) {
#pragma unroll
    for (int i = 0; i < 8; ++i) v[i] *= silu_slope(a[i]);
  }
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

// Biases of columns col .. col + 7 (zeros without, and from n on).
__device__ __forceinline__ void bias8(const float* bias, int col, int n, float b[8]) {
#pragma unroll
  for (int i = 0; i < 8; ++i) b[i] = bias && i < n ? bias[col + i] : 0.0f;
}
// Eight elements of the epilogue: bias, activation, dropout, residual; v becomes the output, and the pre-activation
// is stored on the way.
__device__ __forceinline__ void dense_out8(const DenseEpi& e, const float b[8], int64_t row, int col, int n, float v[8]) {
#pragma unroll
  for (int i = 0; i < 8; ++i) v[i] += b[i];
  if (e.pre.data) store8(e.pre, row, col, n, v);
  act8(e.act, v);
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

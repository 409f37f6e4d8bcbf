// Rows of a caller's matrix, shared by the kernels over label logits.
//
// A row may start anywhere (odd label counts put every row at another
// alignment), so it is walked in the 16-byte vectors that memory is divided
// into: `phase` elements of the first vector lie before the row, vector i holds
// columns V i - phase .. + V - 1, and the elements before the first and after the
// last whole vector are accessed one by one.
#pragma once

#include "asgd_dev.h"

namespace asgd {

typedef _Float16 f16;
typedef unsigned long long u64;

template <typename T>
struct Row {
  static constexpr int V = 16 / (int)sizeof(T);
  typedef T vec __attribute__((ext_vector_type(V)));
  T* base;  // 16-byte aligned; element (i, e) of vector i is column V i - phase + e
  int phase, n_cols;

  __device__ Row(T* p, int64_t ld, int row, int cols) {
    T* const first = p + (int64_t)row * ld;
    phase = (int)(((uintptr_t)first & 15) / sizeof(T));
    base = first - phase;
    n_cols = cols;
  }
  __device__ int col(int i) const { return V * i - phase; }
};

// v of lane ^ X, without a trip through LDS.
template <int CTRL>
__device__ __forceinline__ unsigned dpp(unsigned v) {
  return (unsigned)__builtin_amdgcn_update_dpp(0, (int)v, CTRL, 0xf, 0xf, true);
}
template <int X>
__device__ __forceinline__ unsigned lane_xor(unsigned v, int) {
  if constexpr (X == 1) return dpp<0xb1>(v);         // quad_perm [1, 0, 3, 2]
  else if constexpr (X == 2) return dpp<0x4e>(v);    // quad_perm [2, 3, 0, 1]
  else if constexpr (X == 4) return dpp<0x1b>(dpp<0x141>(v));  // half row mirrored (xor 7), then xor 3
  else if constexpr (X == 8) return dpp<0x128>(v);   // row rotated by 8
  else if constexpr (X == 16) {
    const auto s = __builtin_amdgcn_permlane16_swap(v, v, false, false);
    const unsigned a = s[0], b = s[1];
    return __builtin_amdgcn_inverse_ballot_w64(0xffff0000ffff0000ull) ? a : b;
  } else {
    const auto s = __builtin_amdgcn_permlane32_swap(v, v, false, false);
    const unsigned a = s[0], b = s[1];
    return __builtin_amdgcn_inverse_ballot_w64(0xffffffff00000000ull) ? a : b;
  }
}
template <int X>
__device__ __forceinline__ u64 lane_xor(u64 v, int lane) {
  return ((u64)lane_xor<X>((unsigned)(v >> 32), lane) << 32) | lane_xor<X>((unsigned)v, lane);
}

// Entries [*q0, *q1) of row i of a list, kept inside [*first, *first + nnz) whatever
// indptr holds.
__device__ __forceinline__ void list_range(const IdLists& a, int i, int* q0, int* q1) {
  const int64_t lo = *a.first, hi = lo + a.nnz;
  const int64_t s = max((int64_t)a.indptr[i], lo), e = min((int64_t)a.indptr[i + 1], hi);
  *q0 = (int)s;
  *q1 = (int)(e < s ? s : e);
}

// (m, s) of a softmax: the maximum so far and the sum of e^(c (z - m)), c = ce / log2(e).  m = -inf: nothing yet.
__device__ __forceinline__ void soft_merge(float& m, float& s, float m2, float s2, float ce) {
  const float mm = fmaxf(m, m2);
  if (mm == -INFINITY) return;
  // (a side that holds the maximum is not rescaled: inf - inf of a row with +inf stays out)
  const float a = m == mm ? s : m == -INFINITY ? 0.0f : s * __builtin_amdgcn_exp2f((m - mm) * ce);
  const float b = m2 == mm ? s2 : m2 == -INFINITY ? 0.0f : s2 * __builtin_amdgcn_exp2f((m2 - mm) * ce);
  s = a + b;
  m = mm;
}

}  // namespace asgd

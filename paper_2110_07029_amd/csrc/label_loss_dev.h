// What the kernels of the label loss share (k_label_loss.hip, k_label_narrow.hip).
#pragma once

#include "logits_dev.h"
#include "tile_plan.h"

namespace asgd {

// Entries of row i: the first 65,535 of them (counts of a label in a row then fit 16 bits).
__device__ __forceinline__ void label_range(const IdLists& y, int i, int* q0, int* q1) {
  list_range(y, i, q0, q1);
  if (*q1 - *q0 > 65535) *q1 = *q0 + 65535;
}

// Calls take(id) for every `step`-th entry of row i from `first` on that is not negative, eight loads at a time (one at a
// time, lists of 75 ids cost more than a tile's products).
template <class F>
__device__ __forceinline__ void each_label(const IdLists& y, int i, int first, int step, F take) {
  int q0, q1;
  label_range(y, i, &q0, &q1);
  const int32_t* const list = y.indices + q0;
  const int n = q1 - q0;
  for (int q = first; q < n; q += 8 * step) {
    int id[8];
#pragma unroll
    for (int k = 0; k < 8; ++k) id[k] = q + k * step < n ? list[q + k * step] : -1;
#pragma unroll
    for (int k = 0; k < 8; ++k)
      if (id[k] >= 0) take(id[k]);
  }
}

// How dz is formed from z.
struct DzArgs {
  const float* bias;   // of the piece's first label
  // p_ij = e^(z_ij - top_i) inv_i: the rounding of a log-sum-exp would be in all of a row's probabilities alike
  const float *top, *inv, *share, *weights, *scale;
  float up;            // 2^15 for fp16
  void* dz;            // [B x ld]
  int64_t ld;
  float* part;         // [tiles_m x ld] column sums, or null
  IdLists y;
  int label0, n_labels;
};

// ---- rows of at most 128 columns of 16 bits (k_label_narrow.hip) -------------------------
struct NarrowPlan {
  int row_blocks, tiles, per, ranges;
};
bool narrow_takes(int dtype, int d);
bool narrow_grad_takes(int dtype, int n_rows, int d);
bool narrow_sides_take(int dtype, int n_rows, int n_labels, int d);
bool narrow_sides_worth(int n_rows, int n_labels, int nnz);
NarrowPlan narrow_rows_plan(int n_rows, int n_labels);
NarrowPlan narrow_lse_plan(int n_rows, int n_labels);
NarrowPlan narrow_grad_plan(int n_labels);
size_t narrow_slab_bytes(const NarrowPlan& p, int n_rows);
// part [n_rows][ranges]: maximum and sum of exponentials of a row's labels in a range.
hipError_t launch_narrow_lse(int dtype, const NarrowPlan& p, const TpOperand& h, const TpOperand& w, const float* bias,
                             int n_rows, int n_labels, int d, float2* part, hipStream_t st);
// dw, db complete (scaled by alpha *a.scale); slabs [ranges][n_rows][128]: sums for dh, not scaled.
hipError_t launch_narrow_grad(int dtype, const NarrowPlan& p, const TpOperand& h, const TpOperand& w, const DzArgs& a,
                              int n_rows, int d, float alpha, const MatDev& dw, float* db, float* slabs, hipStream_t st);
// The same, for any number of rows.
hipError_t launch_narrow_sides(int dtype, const NarrowPlan& p, const TpOperand& h, const TpOperand& w, const DzArgs& a,
                               int n_rows, int d, float alpha, const MatDev& dw, float* db, float* slabs, hipStream_t st);

}  // namespace asgd

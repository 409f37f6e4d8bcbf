// Distillation from a teacher's top logits (asgd_distill).
//
// With p the softmax of a row of z over the temperature T and q that of the teacher's
// k logits, loss = T^2 sum q (ln q - ln p) and dz = w T (p - q).  Two passes over z:
// k_distill_sums gives (max, sum of exponentials) per piece of a row and
// takes the student's logits of the teacher's labels; k_distill_grad joins the pieces,
// and writes w T p for its piece and then, apart, the entries that the teacher names.
#include <math.h>

#include "asgd_dev.h"
#include "asgd_kernels.h"
#include "logits_dev.h"

namespace asgd {

namespace {

constexpr int KD_THREADS = 256;
constexpr int KD_WAVES = KD_THREADS / 64;
constexpr int KD_MAX_K = 512;

__device__ __forceinline__ bool finite(float v) { return (__float_as_uint(v) & 0x7f800000u) != 0x7f800000u; }

// One piece's maximum m and sum of e^((z - m) / T); ce = log2(e) / T.
template <typename T>
__global__ __launch_bounds__(KD_THREADS) void k_distill_sums(const T* __restrict__ z, int64_t ld, int L, int n_labels,
                                                             const int32_t* __restrict__ t_ids, int k, float ce,
                                                             int splits, int vec_split, float2* __restrict__ part,
                                                             float* __restrict__ z_t) {
  using R = Row<T>;
  constexpr int V = R::V, U = 4;
  __shared__ float2 red[KD_WAVES];
  const int row = blockIdx.x / splits, split = blockIdx.x % splits;
  const R zr(const_cast<T*>(z), ld, row, L);
  const int v0 = split * vec_split, v1 = min(zr.n_vec, v0 + vec_split);
  if (split == 0)
    for (int e = threadIdx.x; e < k; e += KD_THREADS) {
      const int id = t_ids[(int64_t)row * k + e];
      z_t[(int64_t)row * k + e] = id >= 0 && id < n_labels ? (float)z[(int64_t)row * ld + id] : 0.0f;
    }
  float m = -INFINITY, s = 0.0f;
  for (int base = v0; base < v1; base += KD_THREADS * U) {
    float x[U][V];
    unsigned ok[U];
    float mx = -INFINITY;
    bool nan = false;
#pragma unroll
    for (int u = 0; u < U; ++u) {
      const int i = base + u * KD_THREADS + (int)threadIdx.x;
      ok[u] = i < v1 ? zr.in_row(i) : 0;
      if (ok[u]) zr.load(i, ok[u], x[u]);
#pragma unroll
      for (int e = 0; e < V; ++e) {
        x[u][e] = (ok[u] >> e) & 1 ? x[u][e] : -INFINITY;
        nan |= x[u][e] != x[u][e];
        mx = fmaxf(mx, x[u][e]);
      }
    }
    if (mx > m) {
      s = m == -INFINITY ? 0.0f : s * __builtin_amdgcn_exp2f((m - mx) * ce);
      m = mx;
    }
    if (m != -INFINITY) {
      float a = 0.0f;
#pragma unroll
      for (int u = 0; u < U; ++u)
#pragma unroll
        for (int e = 0; e < V; ++e) a += __builtin_amdgcn_exp2f((x[u][e] - m) * ce);
      s += a;
    }
    if (nan) m = INFINITY;  // a NaN ends like an infinity: (inf, NaN)
    if (m == INFINITY) s = NAN;
  }
#pragma unroll
  for (int o = 32; o >= 1; o >>= 1) soft_merge(m, s, __shfl_xor(m, o), __shfl_xor(s, o), ce);
  const int lane = threadIdx.x & 63, w = threadIdx.x >> 6;
  if (lane == 0) red[w] = make_float2(m, s);
  __syncthreads();
  if (threadIdx.x == 0) {
    for (int i = 1; i < KD_WAVES; ++i) soft_merge(m, s, red[i].x, red[i].y, ce);
    part[blockIdx.x] = make_float2(m, s);
  }
}

// Sum / maximum over the workgroup, the same on every thread.
__device__ __forceinline__ float wg_sum(float v, float* red) {
  v = wave_sum(v);
  __syncthreads();
  if ((threadIdx.x & 63) == 0) red[threadIdx.x >> 6] = v;
  __syncthreads();
  float t = red[0];
  for (int i = 1; i < KD_WAVES; ++i) t += red[i];
  return t;
}
__device__ __forceinline__ float wg_max(float v, float* red) {
  v = wave_max(v);
  __syncthreads();
  if ((threadIdx.x & 63) == 0) red[threadIdx.x >> 6] = v;
  __syncthreads();
  float t = red[0];
  for (int i = 1; i < KD_WAVES; ++i) t = fmaxf(t, red[i]);
  return t;
}

// The row's loss, and with GRAD the gradient of one piece of it.
template <typename T, bool GRAD>
__global__ __launch_bounds__(KD_THREADS) void k_distill_grad(const T* z, int64_t ld, int L, int n_labels,
                                                             const int32_t* __restrict__ t_ids,
                                                             const float* __restrict__ t_logits, int k, float temp,
                                                             float ce, float ce_lo, const float* __restrict__ weights,
                                                             float mean_weight, int n_part, int splits, int vec_split,
                                                             const float2* __restrict__ part,
                                                             const float* __restrict__ z_t,
                                                             float* __restrict__ loss_rows, T* grad, int64_t ld_g) {
  using R = Row<T>;
  constexpr int V = R::V;
  __shared__ float red[KD_WAVES];
  __shared__ float2 red2[KD_WAVES];
  __shared__ float q[KD_MAX_K];
  __shared__ int q_id[KD_MAX_K];
  const int row = blockIdx.x / splits, split = blockIdx.x % splits;
  const int tid = threadIdx.x, lane = tid & 63, wave = tid >> 6;

  // the row's maximum and sum from its pieces
  float m = -INFINITY, s = 0.0f;
  for (int i = tid; i < n_part; i += KD_THREADS) {
    const float2 ms = part[(int64_t)row * n_part + i];
    soft_merge(m, s, ms.x, ms.y, ce);
  }
#pragma unroll
  for (int o = 32; o >= 1; o >>= 1) soft_merge(m, s, __shfl_xor(m, o), __shfl_xor(s, o), ce);
  if (lane == 0) red2[wave] = make_float2(m, s);
  __syncthreads();
  m = red2[0].x;
  s = red2[0].y;
  for (int i = 1; i < KD_WAVES; ++i) soft_merge(m, s, red2[i].x, red2[i].y, ce);

  // q: the softmax of the teacher's counted logits
  float t_max = -INFINITY;
  for (int e = tid; e < k; e += KD_THREADS) {
    const int id = t_ids[(int64_t)row * k + e];
    const float t = t_logits[(int64_t)row * k + e];
    const bool on = id >= 0 && id < n_labels && finite(t);
    q_id[e] = on ? id : -1;
    q[e] = t;
    if (on) t_max = fmaxf(t_max, t);
  }
  t_max = wg_max(t_max, red);
  float t_sum = 0.0f;
  for (int e = tid; e < k; e += KD_THREADS) {
    q[e] = q_id[e] >= 0 ? expf((q[e] - t_max) / temp) : 0.0f;
    t_sum += q[e];
  }
  t_sum = wg_sum(t_sum, red);
  const bool some = t_max != -INFINITY;
  const float inv_t = some ? 1.0f / t_sum : 0.0f;
  const float log_s = logf(s);
  float part_loss = 0.0f;
  for (int e = tid; e < k; e += KD_THREADS) {
    const float w = q[e] * inv_t;
    q[e] = w;
    if (split == 0 && w > 0.0f)
      part_loss += w * (logf(w) - ((z_t[(int64_t)row * k + e] - m) / temp - log_s));
  }
  if (split == 0) {
    part_loss = wg_sum(part_loss, red);
    // (a row of -inf gives no label any probability)
    if (tid == 0) loss_rows[row] = !some ? 0.0f : m == -INFINITY ? INFINITY : temp * temp * part_loss;
  }
  if constexpr (!GRAD) return;
  const float scale = (weights ? weights[row] : mean_weight) * temp;
  const float f = s == 0.0f ? 0.0f : scale / s;
  const R zr(const_cast<T*>(z), ld, row, L);
  const R gr(grad, ld_g, row, L);
  const int v0 = split * vec_split, v1 = min(zr.n_vec, v0 + vec_split);
  auto softmax = [&](float x) {
    // e^((x - m) / T) / s: the exponent's product in two parts, for fp32's sake
    const float d = x - m;
    if (x == -INFINITY && m != INFINITY) return 0.0f;
    if constexpr (sizeof(T) == 4) {
      const float t = d * ce;
      const float r = fmaf(d, ce, -t) + d * ce_lo;
      const float p = __builtin_amdgcn_exp2f(t);
      return fmaf(p, r * LN2, p);
    } else {
      return __builtin_amdgcn_exp2f(d * ce);
    }
  };
  for (int i = v0 + tid; i < v1; i += KD_THREADS) {
    const unsigned in = zr.in_row(i);
    float x[V];
    zr.load(i, in, x);
#pragma unroll
    for (int e = 0; e < V; ++e) x[e] = some ? f * softmax(x[e]) : 0.0f;
    if (gr.phase == zr.phase) {
      gr.store(i, x);
    } else {
      const int c = zr.col(i);
#pragma unroll
      for (int e = 0; e < V; ++e)
        if ((in >> e) & 1) grad[(int64_t)row * ld_g + c + e] = (T)x[e];
    }
  }
  if (!some) return;
  // the labels that the teacher names, after the others' stores: the first of equal ids writes
  __syncthreads();
  const int c0 = zr.col(v0), c1 = zr.col(v1);
  for (int e = tid; e < k; e += KD_THREADS) {
    const int id = q_id[e];
    if (id < 0 || id < c0 || id >= c1) continue;
    float sum = 0.0f;
    bool first = true;
    for (int j = 0; j < k; ++j)
      if (q_id[j] == id) {
        first = first && j >= e;
        sum += q[j];
      }
    if (first) grad[(int64_t)row * ld_g + id] = (T)(f * softmax(z_t[(int64_t)row * k + e]) - scale * sum);
  }
}

}  // namespace

DistillShape distill_shape(int rows, int cols) {
  DistillShape sh;
  const int want = (2048 + rows - 1) / rows, most = (cols + 8191) / 8192;
  sh.splits = want < most ? want : most;
  return sh;
}

static size_t part_bytes(const DistillShape& sh, int rows) {
  return ((size_t)rows * sh.splits * sizeof(float2) + 255) / 256 * 256;
}

size_t distill_ws_bytes(const DistillShape& sh, int rows, int k) {
  return part_bytes(sh, rows) + (size_t)rows * k * sizeof(float);
}

template <typename T>
static hipError_t distill_as(const DistillJob& j, const DistillShape& sh, void* ws, hipStream_t st) {
  const int n_vec = (j.n_cols + 2 * Row<T>::V - 2) / Row<T>::V;
  const int vps = (n_vec + sh.splits - 1) / sh.splits;
  float2* part = (float2*)ws;
  float* z_t = (float*)((char*)ws + part_bytes(sh, j.n_rows));
  const double c = 1.4426950408889634 / (double)j.temperature;
  const float ce = (float)c, ce_lo = (float)(c - (double)ce);
  const unsigned n = (unsigned)j.n_rows * sh.splits;
  hipLaunchKernelGGL(k_distill_sums<T>, dim3(n), dim3(KD_THREADS), 0, st, (const T*)j.z, j.ld, j.n_cols, j.n_labels, j.t_ids, j.k,
                     ce, sh.splits, vps, part, z_t);
  const float mean = 1.0f / (float)j.n_rows;
  if (j.grad)
    hipLaunchKernelGGL((k_distill_grad<T, true>), dim3(n), dim3(KD_THREADS), 0, st, (const T*)j.z, j.ld, j.n_cols,
                       j.n_labels, j.t_ids, j.t_logits, j.k, j.temperature, ce, ce_lo, j.weights, mean, sh.splits, sh.splits, vps,
                       part, z_t, j.loss_rows, (T*)j.grad, j.ld_grad);
  else
    hipLaunchKernelGGL((k_distill_grad<T, false>), dim3(j.n_rows), dim3(KD_THREADS), 0, st, (const T*)j.z, j.ld,
                       j.n_cols, j.n_labels, j.t_ids, j.t_logits, j.k, j.temperature, ce, ce_lo, j.weights, mean, sh.splits, 1, vps,
                       part, z_t, j.loss_rows, (T*)nullptr, (int64_t)0);
  return hipGetLastError();
}

hipError_t launch_distill(int dtype, const DistillJob& j, const DistillShape& sh, void* ws, hipStream_t st) {
  if (dtype == 0) return distill_as<float>(j, sh, ws, st);
  if (dtype == 1) return distill_as<bf16>(j, sh, ws, st);
  return distill_as<f16>(j, sh, ws, st);
}

}  // namespace asgd

// Distillation from a teacher's top logits (asgd_distill).
//
// With p the softmax of a row of z over the temperature T and q that of the teacher's
// k logits, loss = T^2 sum q (ln q - ln p) and dz = w T (p - q).  The gradient needs the row's
// sum, so a row is read twice unless something holds it meanwhile:
//   k_distill_row    a row that a workgroup's registers hold (128 KB, many rows: 256 KB): one read, one write;
//   k_distill_sums   longer rows, first pass: (max, sum of exponentials) per piece of a row, and
//                    the student's logits of the teacher's labels (the gradient may take z's place);
//   k_distill_grad   second pass: joins the pieces' sums and writes the piece's gradient.
// The gradient is w T p everywhere and then, after the workgroup's other stores, once more
// at the labels that the teacher names: the first of the entries that name a label writes it,
// with the sum of q over all of them.
#include <math.h>

#include "asgd_dev.h"
#include "asgd_kernels.h"
#include "logits_dev.h"

namespace asgd {

namespace {

constexpr int KD_THREADS = 256;
constexpr int KD_WAVES = KD_THREADS / 64;
constexpr int KD_WGS = 2048;  // workgroups wanted per pass of a slab
constexpr int KD_ROWS = 512;
constexpr int64_t KD_SLAB = 192 << 20;

__device__ __forceinline__ bool finite(float v) { return (__float_as_uint(v) & 0x7f800000u) != 0x7f800000u; }

// A row as whole vectors [va, vb) and the labels before and after them, at most 14: edge e is
// column e < head ? e : tail + e - head.
template <typename T>
struct Parts {
  static constexpr int V = Row<T>::V;
  int va, vb, head, tail, edges;
  __device__ explicit Parts(const Row<T>& r) {
    va = r.phase ? 1 : 0;
    vb = max(va, (r.phase + r.n_cols) / V);
    head = min(r.n_cols, r.col(va));
    tail = min(r.n_cols, max(head, r.col(vb)));
    edges = head + r.n_cols - tail;
  }
  __device__ int edge(int e) const { return e < head ? e : tail + e - head; }
};

template <int WAVES>
__device__ __forceinline__ float wg_sum(float v, float* red) {
  v = wave_sum(v);
  __syncthreads();
  if ((threadIdx.x & 63) == 0) red[threadIdx.x >> 6] = v;
  __syncthreads();
  float t = red[0];
#pragma unroll
  for (int i = 1; i < WAVES; ++i) t += red[i];
  return t;
}
template <int WAVES>
__device__ __forceinline__ float wg_max(float v, float* red) {
  v = wave_max(v);
  __syncthreads();
  if ((threadIdx.x & 63) == 0) red[threadIdx.x >> 6] = v;
  __syncthreads();
  float t = red[0];
#pragma unroll
  for (int i = 1; i < WAVES; ++i) t = fmaxf(t, red[i]);
  return t;
}

// The softmax of a logit: e^((x - m) / T) / s, given f = 1 / s times what the caller wants.  For
// fp32 gradients the exponent's product is carried in two parts (the error of one fp32 product,
// 2^-24 of an exponent of tens, would show in the gradient).
template <typename T>
__device__ __forceinline__ float soft(float x, float m, float f, float ce, float ce_lo) {
  const float d = x - m;
  if constexpr (sizeof(T) == 4) {
    const float t = d * ce;
    const float r = fmaf(d, ce, -t) + d * ce_lo;
    const float p = __builtin_amdgcn_exp2f(t);
    // (far below the maximum, or -inf: p = 0 and r is none; a row whose f is NaN stays NaN)
    return f * (t == -INFINITY ? 0.0f : fmaf(p, r * LN2, p));
  } else {
    return f * __builtin_amdgcn_exp2f(d * ce);
  }
}

// The teacher of a row: q and ids of the entries that count (id -1 where one does not), in LDS.
// Returns whether any does.
template <int THREADS>
__device__ __forceinline__ bool teacher(const int32_t* t_ids, const float* t_logits, int k, int n_labels, float temp,
                                        float* q, int* q_id, float* red) {
  float t_max = -INFINITY;
  for (int e = threadIdx.x; e < k; e += THREADS) {
    const int id = t_ids[e];
    const float t = t_logits[e];
    const bool on = id >= 0 && id < n_labels && finite(t);
    q_id[e] = on ? id : -1;
    q[e] = t;
    if (on) t_max = fmaxf(t_max, t);
  }
  t_max = wg_max<THREADS / 64>(t_max, red);
  float sum = 0.0f;
  for (int e = threadIdx.x; e < k; e += THREADS) {
    q[e] = q_id[e] >= 0 ? expf((q[e] - t_max) / temp) : 0.0f;
    sum += q[e];
  }
  sum = wg_sum<THREADS / 64>(sum, red);
  const bool some = t_max != -INFINITY;
  const float inv = some ? 1.0f / sum : 0.0f;
  for (int e = threadIdx.x; e < k; e += THREADS) q[e] *= inv;
  return some;
}

// T^2 sum q (ln q - ln p) from the student's logits of the entries (the thread's own entries' q).
template <int THREADS>
__device__ __forceinline__ float row_loss(const float* q, const float* z_t, int k, float m, float s, float temp, bool some,
                                          float* red) {
  const float log_s = logf(s);
  float part = 0.0f;
  for (int e = threadIdx.x; e < k; e += THREADS)
    if (q[e] > 0.0f) part += q[e] * (logf(q[e]) - ((z_t[e] - m) / temp - log_s));
  part = wg_sum<THREADS / 64>(part, red);
  // (a row of -inf gives no label any probability)
  return !some ? 0.0f : m == -INFINITY ? INFINITY : temp * temp * part;
}

// The gradient at the teacher's labels in [c0, c1), after the workgroup's other stores.
template <typename T, int THREADS>
__device__ __forceinline__ void put_teacher(T* grow, const float* q, const int* q_id, const float* z_t, int k, int c0,
                                            int c1, float m, float f, float scale, float ce, float ce_lo) {
  __syncthreads();
  for (int e = threadIdx.x; e < k; e += THREADS) {
    const int id = q_id[e];
    if (id < 0 || id < c0 || id >= c1) continue;
    float sum = 0.0f;
    bool first = true;
    for (int j = 0; j < k; ++j)
      if (q_id[j] == id) {
        first = first && j >= e;
        sum += q[j];
      }
    if (first) grow[id] = (T)((m == -INFINITY ? 0.0f : soft<T>(z_t[e], m, f, ce, ce_lo)) - scale * sum);
  }
}

template <typename T>
__device__ __forceinline__ void store_vec(const Row<T>& g, bool same_phase, int i, int c, const float (&x)[Row<T>::V]) {
  constexpr int V = Row<T>::V;
  typename Row<T>::vec v;
#pragma unroll
  for (int e = 0; e < V; ++e) v[e] = (T)x[e];
  if (same_phase) {
    // (past the caches: they hold logits that are read again)
    __builtin_nontemporal_store(v, reinterpret_cast<typename Row<T>::vec*>(g.base + (int64_t)V * i));
  } else {
    T* const to = g.base + g.phase + c;
#pragma unroll
    for (int e = 0; e < V; ++e) to[e] = v[e];
  }
}

// Everything about one row, its logits in registers, NV vectors a thread.
template <typename T, int THREADS, int NV, bool GRAD>
__global__ __launch_bounds__(THREADS) void k_distill_row(DistillJob job, float ce, float ce_lo, float mean_weight) {
  using R = Row<T>;
  constexpr int V = R::V, WAVES = THREADS / 64;
  __shared__ float red[WAVES];
  __shared__ float q[DISTILL_MAX_K], z_t[DISTILL_MAX_K];
  __shared__ int q_id[DISTILL_MAX_K];
  const int row = blockIdx.x, tid = threadIdx.x, k = job.k;
  const R zr((T*)const_cast<void*>(job.z), job.ld, row, job.n_cols);
  const Parts<T> at(zr);
  typename R::vec x[NV];
#pragma unroll
  for (int j = 0; j < NV; ++j) {
    const int i = at.va + j * THREADS + tid;
    if (i < at.vb) x[j] = *reinterpret_cast<const typename R::vec*>(zr.base + (int64_t)V * i);
  }
  const bool has_edge = tid < at.edges;
  const float edge = has_edge ? (float)zr.base[zr.phase + at.edge(tid)] : -INFINITY;
  const int32_t* t_ids = job.t_ids + (int64_t)row * k;
  for (int e = tid; e < k; e += THREADS) {
    const int id = t_ids[e];
    z_t[e] = id >= 0 && id < job.n_labels ? (float)zr.base[zr.phase + id] : 0.0f;
  }
  const bool some = teacher<THREADS>(t_ids, job.t_logits + (int64_t)row * k, k, job.n_labels, job.temperature, q, q_id, red);
  float m = edge;
  bool nan = edge != edge;
#pragma unroll
  for (int j = 0; j < NV; ++j)
    if (at.va + j * THREADS + tid < at.vb)
#pragma unroll
      for (int e = 0; e < V; ++e) {
        m = fmaxf(m, (float)x[j][e]);
        nan |= (float)x[j][e] != (float)x[j][e];
      }
  m = wg_max<WAVES>(nan ? INFINITY : m, red);  // (NaN ends like +inf: a sum that is NaN)
  float s = 0.0f;
  if (m != -INFINITY) {
    if (has_edge) s = __builtin_amdgcn_exp2f((edge - m) * ce);
#pragma unroll
    for (int j = 0; j < NV; ++j)
      if (at.va + j * THREADS + tid < at.vb)
#pragma unroll
        for (int e = 0; e < V; ++e) s += __builtin_amdgcn_exp2f(((float)x[j][e] - m) * ce);
  }
  s = wg_sum<WAVES>(s, red);
  if (m == INFINITY) s = NAN;
  const float loss = row_loss<THREADS>(q, z_t, k, m, s, job.temperature, some, red);
  if (tid == 0) job.loss_rows[row] = loss;
  if constexpr (!GRAD) return;
  const float scale = (job.weights ? job.weights[row] : mean_weight) * job.temperature;
  const float f = some && s != 0.0f ? scale / s : 0.0f;
  const R gr((T*)job.grad, job.ld_grad, row, job.n_cols);
  const bool same = gr.phase == zr.phase;
  auto value = [&](float v) { return m == -INFINITY || !some ? 0.0f : soft<T>(v, m, f, ce, ce_lo); };
  if (has_edge) gr.base[gr.phase + at.edge(tid)] = (T)value(edge);
#pragma unroll
  for (int j = 0; j < NV; ++j) {
    const int i = at.va + j * THREADS + tid;
    if (i < at.vb) {
      float y[V];
#pragma unroll
      for (int e = 0; e < V; ++e) y[e] = value((float)x[j][e]);
      store_vec<T>(gr, same, i, zr.col(i), y);
    }
  }
  if (some) put_teacher<T, THREADS>(gr.base + gr.phase, q, q_id, z_t, k, 0, job.n_cols, m, f, scale, ce, ce_lo);
}

// First pass over one piece of a row.
template <typename T>
__device__ __forceinline__ void piece_sums(const DistillJob& job, int row, int split, float ce, int splits, int vec_split,
                                           float2* part, float* z_t, float2* red) {
  using R = Row<T>;
  constexpr int V = R::V, U = 16 / V;
  const int tid = threadIdx.x, k = job.k;
  const R zr((T*)const_cast<void*>(job.z), job.ld, row, job.n_cols);
  const Parts<T> at(zr);
  const int v0 = at.va + split * vec_split, v1 = min(at.vb, v0 + vec_split);
  float m = -INFINITY, s = 0.0f;
  if (split == 0) {
    for (int e = tid; e < k; e += KD_THREADS) {
      const int id = job.t_ids[(int64_t)row * k + e];
      z_t[(int64_t)row * k + e] = id >= 0 && id < job.n_labels ? (float)zr.base[zr.phase + id] : 0.0f;
    }
    if (tid < at.edges) {
      m = (float)zr.base[zr.phase + at.edge(tid)];
      if (m != m) m = INFINITY;
      s = m == -INFINITY ? 0.0f : m == INFINITY ? NAN : 1.0f;
    }
  }
  typename R::vec x[U];
  auto load = [&](int base) {
#pragma unroll
    for (int u = 0; u < U; ++u)
      x[u] = *reinterpret_cast<const typename R::vec*>(zr.base + (int64_t)V * min(base + u * KD_THREADS + tid, v1 - 1));
  };
  if (v0 < v1) load(v0);
  for (int base = v0; base < v1; base += KD_THREADS * U) {
    float y[U][V];
    float mx = -INFINITY;
    bool nan = false;
#pragma unroll
    for (int u = 0; u < U; ++u) {
      const bool on = base + u * KD_THREADS + tid < v1;
#pragma unroll
      for (int e = 0; e < V; ++e) {
        y[u][e] = on ? (float)x[u][e] : -INFINITY;
        mx = fmaxf(mx, y[u][e]);
      }
    }
    if (base + KD_THREADS * U < v1) load(base + KD_THREADS * U);
    if (mx > m) {
      s = m == -INFINITY ? 0.0f : s * __builtin_amdgcn_exp2f((m - mx) * ce);
      m = mx;
    }
    if (m != -INFINITY) {
      float a = 0.0f;
#pragma unroll
      for (int u = 0; u < U; ++u)
#pragma unroll
        for (int e = 0; e < V; ++e) a += __builtin_amdgcn_exp2f((y[u][e] - m) * ce);
      s += a;  // (NaN from a NaN or from +inf - +inf)
    } else {
#pragma unroll
      for (int u = 0; u < U; ++u)
#pragma unroll
        for (int e = 0; e < V; ++e) nan |= y[u][e] != y[u][e];
    }
    if (nan || s != s) {  // ends like +inf
      m = INFINITY;
      s = NAN;
    }
  }
#pragma unroll
  for (int o = 32; o >= 1; o >>= 1) soft_merge(m, s, __shfl_xor(m, o), __shfl_xor(s, o), ce);
  const int lane = tid & 63, w = tid >> 6;
  if (lane == 0) red[w] = make_float2(m, s);
  __syncthreads();
  if (tid == 0) {
    for (int i = 1; i < KD_WAVES; ++i) soft_merge(m, s, red[i].x, red[i].y, ce);
    part[(int64_t)row * splits + split] = make_float2(m, s);
  }
}

// Second pass: the row's loss, and with GRAD the gradient of one piece of it.
template <typename T, bool GRAD>
__device__ __forceinline__ void piece_grad(const DistillJob& job, int row, int split, float ce, float ce_lo,
                                           float mean_weight, int n_part, int vec_split, const float2* part,
                                           const float* z_t, float2* red2) {
  using R = Row<T>;
  constexpr int V = R::V, U = 2;
  __shared__ float red[KD_WAVES];
  __shared__ float q[DISTILL_MAX_K];
  __shared__ int q_id[DISTILL_MAX_K];
  const int tid = threadIdx.x, lane = tid & 63, wave = tid >> 6, k = job.k;
  const R zr((T*)const_cast<void*>(job.z), job.ld, row, job.n_cols);
  const Parts<T> at(zr);
  const int v0 = at.va + split * vec_split, v1 = max(v0, min(at.vb, v0 + vec_split));
  typename R::vec x[U];
  auto load = [&](int base) {
#pragma unroll
    for (int u = 0; u < U; ++u)
      x[u] = *reinterpret_cast<const typename R::vec*>(zr.base + (int64_t)V * min(base + u * KD_THREADS + tid, v1 - 1));
  };
  if (GRAD && v0 < v1) load(v0);

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

  z_t += (int64_t)row * k;
  const bool some = teacher<KD_THREADS>(job.t_ids + (int64_t)row * k, job.t_logits + (int64_t)row * k, k, job.n_labels,
                                        job.temperature, q, q_id, red);
  if (split == 0) {
    const float loss = row_loss<KD_THREADS>(q, z_t, k, m, s, job.temperature, some, red);
    if (tid == 0) job.loss_rows[row] = loss;
  }
  if constexpr (!GRAD) return;
  const float scale = (job.weights ? job.weights[row] : mean_weight) * job.temperature;
  const float f = some && s != 0.0f ? scale / s : 0.0f;
  const R gr((T*)job.grad, job.ld_grad, row, job.n_cols);
  const bool same = gr.phase == zr.phase, zero = m == -INFINITY || !some;
  auto value = [&](float v) { return zero ? 0.0f : soft<T>(v, m, f, ce, ce_lo); };
  if (split == 0 && tid < at.edges) {
    const int c = at.edge(tid);
    gr.base[gr.phase + c] = (T)value((float)zr.base[zr.phase + c]);
  }
  for (int base = v0; base < v1; base += KD_THREADS * U) {
    float y[U][V];
#pragma unroll
    for (int u = 0; u < U; ++u)
#pragma unroll
      for (int e = 0; e < V; ++e) y[u][e] = (float)x[u][e];
    if (base + KD_THREADS * U < v1) load(base + KD_THREADS * U);
#pragma unroll
    for (int u = 0; u < U; ++u) {
      const int i = base + u * KD_THREADS + tid;
      if (i < v1) {
#pragma unroll
        for (int e = 0; e < V; ++e) y[u][e] = value(y[u][e]);
        store_vec<T>(gr, same, i, zr.col(i), y[u]);
      }
    }
  }
  if (!some) return;
  // the piece's labels; the first one's edges too (its own stores, like the others of the piece)
  const int c0 = split == 0 ? 0 : zr.col(v0), c1 = zr.col(v1);
  T* const grow = gr.base + gr.phase;
  put_teacher<T, KD_THREADS>(grow, q, q_id, z_t, k, c0, c1, m, f, scale, ce, ce_lo);
  if (split == 0) put_teacher<T, KD_THREADS>(grow, q, q_id, z_t, k, max(c1, at.tail), job.n_cols, m, f, scale, ce, ce_lo);
}

// The passes over `rows` rows from row0 on.  The second one takes the rows last first: those
// that the first pass read last are the ones that the memory's cache still holds.
template <typename T>
__global__ __launch_bounds__(KD_THREADS) void k_distill_sums(DistillJob job, int row0, float ce, int splits, int vec_split,
                                                             float2* part, float* z_t) {
  __shared__ float2 red[KD_WAVES];
  piece_sums<T>(job, row0 + blockIdx.x / splits, blockIdx.x % splits, ce, splits, vec_split, part, z_t, red);
}
template <typename T>
__global__ __launch_bounds__(KD_THREADS) void k_distill_grad(DistillJob job, int row0, int rows, float ce, float ce_lo,
                                                             float mean_weight, int splits, int vec_split,
                                                             const float2* part, const float* z_t) {
  __shared__ float2 red[KD_WAVES];
  piece_grad<T, true>(job, row0 + rows - 1 - blockIdx.x / splits, blockIdx.x % splits, ce, ce_lo, mean_weight, splits,
                      vec_split, part, z_t, red);
}

// The loss alone, after the first pass.
template <typename T>
__global__ __launch_bounds__(KD_THREADS) void k_distill_loss(DistillJob job, float ce, int n_part, const float2* part,
                                                             const float* z_t) {
  __shared__ float2 red[KD_WAVES];
  piece_grad<T, false>(job, blockIdx.x, 0, ce, 0.0f, 0.0f, n_part, 0, part, z_t, red);
}

}  // namespace

// Slabs of rows whose logits the memory's cache (256 MB) holds between the two passes, and
// pieces per row so that a slab's fill the GPU.  Measured, one slab | slabs of 192 MB (16-bit logits): 256 x
// 670,091 bf16 202 | 196 us (first pass 70, second 127, which is what a copy of z takes; rows in the same order in
// both passes, one slab: 219), 512 x 205,443 fp32 243 | 226; slabs of 64 MB, the first pass of one beside the
// second of another in a launch: 226 and 257.
DistillShape distill_shape(int rows, int cols) {
  DistillShape sh;
  const int64_t n = ((int64_t)rows * cols * 2 + KD_SLAB - 1) / KD_SLAB;
  sh.slabs = (int)(n < rows ? n : rows);
  const int per = (rows + sh.slabs - 1) / sh.slabs;
  const int want = (KD_WGS + per - 1) / per, most = (cols + 8191) / 8192;
  sh.splits = want < most ? want : most;
  return sh;
}

static size_t part_bytes(const DistillShape& sh, int rows) {
  return ((size_t)rows * sh.splits * sizeof(float2) + 255) / 256 * 256;
}

size_t distill_ws_bytes(const DistillShape& sh, int rows, int k) {
  return part_bytes(sh, rows) + (size_t)rows * k * sizeof(float);
}

template <typename T, int THREADS, int NV>
static hipError_t distill_rows(const DistillJob& j, float ce, float ce_lo, hipStream_t st) {
  const float mean = 1.0f / (float)j.n_rows;
  if (j.grad)
    hipLaunchKernelGGL((k_distill_row<T, THREADS, NV, true>), dim3(j.n_rows), dim3(THREADS), 0, st, j, ce, ce_lo, mean);
  else
    hipLaunchKernelGGL((k_distill_row<T, THREADS, NV, false>), dim3(j.n_rows), dim3(THREADS), 0, st, j, ce, ce_lo, mean);
  return hipGetLastError();
}

template <typename T>
static hipError_t distill_as(const DistillJob& j, const DistillShape& sh, void* ws, hipStream_t st) {
  const double c = 1.4426950408889634 / (double)j.temperature;
  const float ce = (float)c, ce_lo = (float)(c - (double)ce);
  const int n_vec = j.n_cols / Row<T>::V;  // whole vectors of a row at most
  if (n_vec <= 2 * 256) return distill_rows<T, 256, 2>(j, ce, ce_lo, st);
  if (n_vec <= 8 * 256) return distill_rows<T, 256, 8>(j, ce, ce_lo, st);
  if (n_vec <= 8 * 1024) return distill_rows<T, 1024, 8>(j, ce, ce_lo, st);
  // 256 KB: half of a compute unit's registers, so one row at a time on each, and worth it from two rows for
  // each on (two passes | this: 512 x 60,000 fp32 65 | 51 us, 300 x 100,000 bf16 43 | 47 us; rows of 400 KB in the
  // same way no longer gain: 512 x 205,443 bf16 120 | 121 us)
  if (j.n_rows >= KD_ROWS && n_vec <= 16 * 1024) return distill_rows<T, 1024, 16>(j, ce, ce_lo, st);
  const int vps = (n_vec + sh.splits - 1) / sh.splits;
  float2* part = (float2*)ws;
  float* z_t = (float*)((char*)ws + part_bytes(sh, j.n_rows));
  const float mean = 1.0f / (float)j.n_rows;
  const int per = j.grad ? (j.n_rows + sh.slabs - 1) / sh.slabs : j.n_rows;
  for (int r0 = 0; r0 < j.n_rows; r0 += per) {
    const int rows = per < j.n_rows - r0 ? per : j.n_rows - r0;
    const dim3 grid((unsigned)rows * sh.splits), block(KD_THREADS);
    hipLaunchKernelGGL(k_distill_sums<T>, grid, block, 0, st, j, r0, ce, sh.splits, vps, part, z_t);
    if (j.grad)
      hipLaunchKernelGGL(k_distill_grad<T>, grid, block, 0, st, j, r0, rows, ce, ce_lo, mean, sh.splits, vps, part, z_t);
  }
  if (!j.grad)
    hipLaunchKernelGGL(k_distill_loss<T>, dim3(j.n_rows), dim3(KD_THREADS), 0, st, j, ce, sh.splits, part, z_t);
  return hipGetLastError();
}

hipError_t launch_distill(int dtype, const DistillJob& j, const DistillShape& sh, void* ws, hipStream_t st) {
  if (dtype == 0) return distill_as<float>(j, sh, ws, st);
  if (dtype == 1) return distill_as<bf16>(j, sh, ws, st);
  return distill_as<f16>(j, sh, ws, st);
}

}  // namespace asgd

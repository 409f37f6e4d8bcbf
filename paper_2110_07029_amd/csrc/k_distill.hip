// Distillation from a teacher's top logits (asgd_distill).
//
// With p the softmax of a row of z over the temperature T and q that of the teacher's
// k logits, loss = T^2 sum q (ln q - ln p) and dz = w T (p - q).  The gradient needs the row's
// sum, so a row is read twice unless something holds it meanwhile:
//   k_distill_row    a row that a workgroup's registers hold (128 KB, many rows: 256 KB): one read, one write;
//   k_distill_sums   longer rows, first pass: (max, sum of exponentials) per piece of a row, and q and
//                    the student's logits at the teacher's labels (the gradient may take z's place);
//   k_distill_grad   second pass: joins the pieces' sums and writes the gradient.
// The gradient is w T p everywhere and then, after the workgroup's other stores, once more
// at the labels that the teacher names: the first of the entries that name a label writes it,
// with the sum of q over all of them.
//
// Measured: 128 x 1,000 fp32 10 us (a launch and three dependent reductions); 256 x 30,000 fp32 16 us (61 MB, 3.8
// TB/s: one workgroup per compute unit holds its row between reading and writing); 256 x 670,091 bf16 163 to 170 us, a
// first pass of 57 (6.0 TB/s) and a second of 107 (343 MB read and as many written, 6.4 TB/s; both passes ask the
// memory for the whole of z).
#include <math.h>

#include <type_traits>

#include "asgd_dev.h"
#include "asgd_kernels.h"
#include "logits_dev.h"

namespace asgd {

namespace {

constexpr int KD_THREADS = 256;
constexpr int KD_WAVES = KD_THREADS / 64;
constexpr int KD_WGS = 1024;  // workgroups wanted for the first pass
// Vectors a thread of the second pass, 12 KB a workgroup; 2 | 3 | 4 of them: 256 x 670,091 bf16 184 | 171 | 170 us,
// 512 x 205,443 fp32 207 | 199 | 216.
constexpr int KD_U = 3;
constexpr int KD_ROWS = 512;
constexpr int KD_GRID = 1 << 20;  // workgroups along x at most (a dimension has below 2^32 threads)

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

// An entry's part of the loss, T^2 q (ln q - ln p) with ln p = (z - m) / T - ln s.  (z - m) / T may pass the type's
// range where T times it does not (z of the lowest value as a mask, T below 1), and z - m itself may: so the
// distance is taken at half its size and meets q first, then 2 T.
__device__ __forceinline__ float entry_loss(float q, float z, float m, float log_s, float temp) {
  return fmaf(2.0f * temp, q * (0.5f * m - 0.5f * z), temp * temp * (q * (logf(q) + log_s)));
}
// (a row of -inf gives no label any probability)
__device__ __forceinline__ float whole_loss(float sum, float m, bool some) {
  return !some ? 0.0f : m == -INFINITY ? INFINITY : sum;
}

// The loss from the student's logits of the entries (the thread's own entries' q).
template <int THREADS>
__device__ __forceinline__ float row_loss(const float* q, const float* z_t, int k, float m, float s, float temp, bool some,
                                          float* red) {
  const float log_s = logf(s);
  float part = 0.0f;
  for (int e = threadIdx.x; e < k; e += THREADS)
    if (q[e] > 0.0f) part += entry_loss(q[e], z_t[e], m, log_s, temp);
  return whole_loss(wg_sum<THREADS / 64>(part, red), m, some);
}

// Whether entry e is the first of those that name its label; *sum: q over all of them.
__device__ __forceinline__ bool teacher_sum(const float* q, const int* q_id, int k, int e, float* sum) {
  const int id = q_id[e];
  if (id < 0) return false;
  bool first = true;
  float t = 0.0f;
  for (int j = 0; j < k; ++j)
    if (q_id[j] == id) {
      first = first && j >= e;
      t += q[j];
    }
  *sum = t;
  return first;
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
  if (!some) return;
  __syncthreads();  // (the workgroup's other stores come first)
  for (int e = tid; e < k; e += THREADS) {
    float sum = 0.0f;
    if (teacher_sum(q, q_id, k, e, &sum))
      gr.base[gr.phase + q_id[e]] = (T)((m == -INFINITY ? 0.0f : soft<T>(z_t[e], m, f, ce, ce_lo)) - scale * sum);
  }
}

// First pass over one piece of a row.
template <typename T>
__device__ __forceinline__ void piece_sums(const DistillJob& job, int row, int split, float ce, int splits, int vec_split,
                                           float2* part, float2* red) {
  using R = Row<T>;
  constexpr int V = R::V, U = 16 / V;
  const int tid = threadIdx.x;
  const R zr((T*)const_cast<void*>(job.z), job.ld, row, job.n_cols);
  const Parts<T> at(zr);
  const int v0 = at.va + split * vec_split, v1 = min(at.vb, v0 + vec_split);
  float m = -INFINITY, s = 0.0f;
  if (split == 0 && tid < at.edges) {
    m = (float)zr.base[zr.phase + at.edge(tid)];
    if (m != m) m = INFINITY;
    s = m == -INFINITY ? 0.0f : m == INFINITY ? NAN : 1.0f;
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
    part[(int64_t)row * (splits + 1) + split] = make_float2(m, s);
  }
}

// An entry of a teacher's list: its q, the student's logit of its label, and if it is the
// first that names this label the label and the sum of q over all that do (otherwise id -1).
struct __align__(16) Entry {
  int id;
  float q, sum, z;
};

// First pass.  The first workgroups make the rows' entries, beside the others' reading.
template <typename T>
__global__ __launch_bounds__(KD_THREADS) void k_distill_sums(DistillJob job, float ce, int splits,
                                                             int vec_split, float2* __restrict__ part,
                                                             Entry* __restrict__ entries) {
  __shared__ float2 red2[KD_WAVES];
  __shared__ float red[KD_WAVES];
  __shared__ float q[DISTILL_MAX_K];
  __shared__ int q_id[DISTILL_MAX_K];
  const int block = (int)blockIdx.x - job.n_rows;
  if (block >= 0) {
    piece_sums<T>(job, block / splits, block % splits, ce, splits, vec_split, part, red2);
    return;
  }
  const int row = blockIdx.x, tid = threadIdx.x, k = job.k;
  const Row<T> zr((T*)const_cast<void*>(job.z), job.ld, row, job.n_cols);
  const bool some = teacher<KD_THREADS>(job.t_ids + (int64_t)row * k, job.t_logits + (int64_t)row * k, k, job.n_labels,
                                        job.temperature, q, q_id, red);
  __syncthreads();
  for (int e = tid; e < k; e += KD_THREADS) {
    Entry t{-1, q[e], 0.0f, q_id[e] >= 0 ? (float)zr.base[zr.phase + q_id[e]] : 0.0f};
    if (teacher_sum(q, q_id, k, e, &t.sum)) t.id = q_id[e];
    entries[(int64_t)row * k + e] = t;
  }
  // (behind the row's pieces: whether any entry counts)
  if (tid == 0) part[(int64_t)row * (splits + 1) + splits] = make_float2(some ? 1.0f : 0.0f, 0.0f);
}

// Second pass: a workgroup writes KD_U vectors a thread of a row, then the teacher's entries among
// them; the first of a row's also finds its loss (without GRAD the only one).  Workgroups go through the rows from
// the last one back, beginning with what the first pass read last (from the first row on | from the last one back:
// 256 x 670,091 bf16 167 | 163 us; 512 x 205,443 fp32 202 | 201, bf16 99 | 100).
template <typename T, bool GRAD>
__global__ __launch_bounds__(KD_THREADS) void k_distill_grad(DistillJob job, int chunks, float ce,
                                                             float ce_lo, float mean_weight, int splits,
                                                             const float2* __restrict__ part,
                                                             const Entry* __restrict__ entries) {
  using R = Row<T>;
  constexpr int V = R::V;
  __shared__ float red[KD_WAVES];
  const int tid = threadIdx.x, lane = tid & 63, k = job.k;
  const unsigned block = blockIdx.y * gridDim.x + blockIdx.x;
  const int row = job.n_rows - 1 - (int)(block / (unsigned)chunks), chunk = chunks - 1 - (int)(block % (unsigned)chunks);
  if (row < 0) return;
  const R zr((T*)const_cast<void*>(job.z), job.ld, row, job.n_cols);
  const Parts<T> at(zr);
  const int v0 = at.va + chunk * (KD_THREADS * KD_U), v1 = max(v0, min(at.vb, v0 + KD_THREADS * KD_U));
  typename R::vec x[KD_U];
  float edge = 0.0f;
  const bool has_edge = chunk == 0 && tid < at.edges;
  if constexpr (GRAD) {
#pragma unroll
    for (int u = 0; u < KD_U; ++u) {
      const int i = v0 + u * KD_THREADS + tid;
      if (i < v1) x[u] = *reinterpret_cast<const typename R::vec*>(zr.base + (int64_t)V * i);
    }
    if (has_edge) edge = (float)zr.base[zr.phase + at.edge(tid)];
  }
  constexpr int E = DISTILL_MAX_K / KD_THREADS;
  Entry t[E];
#pragma unroll
  for (int j = 0; j < E; ++j) {
    t[j] = Entry{-1, 0.0f, 0.0f, 0.0f};
    if (tid + j * KD_THREADS < k) t[j] = entries[(int64_t)row * k + tid + j * KD_THREADS];
  }
  // The pieces' sums as one, in every wave for itself.
  part += (int64_t)row * (splits + 1);
  const bool some = part[splits].x != 0.0f;
  float m = -INFINITY, s = 0.0f;
  for (int i = lane; i < splits; i += 64) {
    const float2 ms = part[i];
    soft_merge(m, s, ms.x, ms.y, ce);
  }
  auto merge = [&](auto x) {
    const float m2 = __uint_as_float(lane_xor<decltype(x)::value>(__float_as_uint(m), lane));
    const float s2 = __uint_as_float(lane_xor<decltype(x)::value>(__float_as_uint(s), lane));
    soft_merge(m, s, m2, s2, ce);
  };
  merge(std::integral_constant<int, 1>());
  merge(std::integral_constant<int, 2>());
  merge(std::integral_constant<int, 4>());
  merge(std::integral_constant<int, 8>());
  merge(std::integral_constant<int, 16>());
  merge(std::integral_constant<int, 32>());
  if (chunk == 0) {
    const float log_s = logf(s);
    float sum = 0.0f;
#pragma unroll
    for (int j = 0; j < E; ++j)
      if (t[j].q > 0.0f) sum += entry_loss(t[j].q, t[j].z, m, log_s, job.temperature);
    sum = wg_sum<KD_WAVES>(sum, red);
    if (tid == 0) job.loss_rows[row] = whole_loss(sum, m, some);
  }
  if constexpr (GRAD) {
    const R gr((T*)job.grad, job.ld_grad, row, job.n_cols);
    const float scale = (job.weights ? job.weights[row] : mean_weight) * job.temperature;
    const float f = some && s != 0.0f ? scale / s : 0.0f;
    const bool zero = !some || m == -INFINITY, same = gr.phase == zr.phase;
    if (zero)  // (the products below are none, or not 0 for a logit that is none)
#pragma unroll
      for (int u = 0; u < KD_U; ++u) x[u] = (typename R::vec)(T)0.0f;
#pragma unroll
    for (int u = 0; u < KD_U; ++u) {
      const int i = v0 + u * KD_THREADS + tid;
      if (i >= v1) continue;
      float y[V];
#pragma unroll
      for (int e = 0; e < V; ++e) y[e] = soft<T>((float)x[u][e], zero ? 0.0f : m, f, ce, ce_lo);
      store_vec<T>(gr, same, i, zr.col(i), y);
    }
    T* const grow = gr.base + gr.phase;
    if (has_edge) grow[at.edge(tid)] = (T)(zero ? 0.0f : soft<T>(edge, m, f, ce, ce_lo));
    __syncthreads();  // (the workgroup's other stores come first)
    const int c0 = zr.col(v0), c1 = zr.col(v1);
#pragma unroll
    for (int j = 0; j < E; ++j) {
      const int id = t[j].id;
      if (id >= 0 && ((id >= c0 && id < c1) || (chunk == 0 && (id < at.head || id >= at.tail))))
        grow[id] = (T)((zero ? 0.0f : soft<T>(t[j].z, m, f, ce, ce_lo)) - scale * t[j].sum);
    }
  }
}

}  // namespace

// Pieces per row so that the first pass fills the GPU: 512 | 1,024 | 2,048 workgroups wanted take 180 | 171 | 172 us
// for 256 x 670,091 bf16, and differ by at most 2 us elsewhere.  Both passes of 192 MB of rows before the next such
// slab were slower than each pass in one launch (180 | 173; 512 x 205,443 fp32 205 | 200, bf16 109 | 100).
int distill_splits(int rows, int cols) {
  const int want = (KD_WGS + rows - 1) / rows, most = (cols + 8191) / 8192;
  return want < most ? want : most;
}

// Scratch memory: per row the pieces' sums and whether its teacher counts, then the teachers' entries.
static size_t part_bytes(int splits, int rows) {
  return ((size_t)rows * (splits + 1) * sizeof(float2) + 255) / 256 * 256;
}
size_t distill_ws_bytes(int splits, int rows, int k) { return part_bytes(splits, rows) + (size_t)rows * k * sizeof(Entry); }

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
static hipError_t distill_as(const DistillJob& j, int splits, void* ws, hipStream_t st) {
  const double c = 1.4426950408889634 / (double)j.temperature;
  const float ce = (float)c, ce_lo = (float)(c - (double)ce);
  const int n_vec = j.n_cols / Row<T>::V;  // whole vectors of a row at most
  if (n_vec <= 2 * 256) return distill_rows<T, 256, 2>(j, ce, ce_lo, st);
  if (n_vec <= 8 * 256) return distill_rows<T, 256, 8>(j, ce, ce_lo, st);
  if (n_vec <= 8 * 1024) return distill_rows<T, 1024, 8>(j, ce, ce_lo, st);
  // 256 KB: half of a compute unit's registers, so one row at a time on each, and worth it from two rows for
  // each on (two passes | this, with gradient: 512 x 60,000 fp32 61 | 51 us, 512 x 100,000 bf16 53 | 52, 300 of these
  // 36 | 47; the loss alone 25 | 29 and 23 | 32.  Rows of 400 KB in the same way: 512 x 205,443 bf16 100 | 121)
  if (j.n_rows >= KD_ROWS && n_vec <= 16 * 1024) return distill_rows<T, 1024, 16>(j, ce, ce_lo, st);
  const int vps = (n_vec + splits - 1) / splits;
  float2* part = (float2*)ws;
  Entry* entries = (Entry*)((char*)ws + part_bytes(splits, j.n_rows));
  const float mean = 1.0f / (float)j.n_rows;
  const dim3 block(KD_THREADS);
  hipLaunchKernelGGL(k_distill_sums<T>, dim3((unsigned)j.n_rows * (splits + 1)), block, 0, st, j, ce, splits, vps, part,
                     entries);
  if (j.grad) {
    const int chunks = (n_vec + KD_THREADS * KD_U - 1) / (KD_THREADS * KD_U);
    const int64_t n = (int64_t)j.n_rows * chunks, y = (n + KD_GRID - 1) / KD_GRID;
    hipLaunchKernelGGL((k_distill_grad<T, true>), dim3((unsigned)((n + y - 1) / y), (unsigned)y), block, 0, st, j, chunks,
                       ce, ce_lo, mean, splits, part, entries);
  } else {
    hipLaunchKernelGGL((k_distill_grad<T, false>), dim3(j.n_rows), block, 0, st, j, 1, ce, ce_lo, mean, splits, part,
                       entries);
  }
  return hipGetLastError();
}

hipError_t launch_distill(int dtype, const DistillJob& j, int splits, void* ws, hipStream_t st) {
  if (dtype == 0) return distill_as<float>(j, splits, ws, st);
  if (dtype == 1) return distill_as<bf16>(j, splits, ws, st);
  return distill_as<f16>(j, splits, ws, st);
}

}  // namespace asgd

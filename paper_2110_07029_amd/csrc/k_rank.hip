// The k best labels of logit rows under rules (asgd_logits_topk).
//
// One pass over the logits.  A workgroup takes one piece of one row; each of
// its waves keeps the 64 best (score, label) pairs that it has met, one per
// lane in descending order, as 64-bit keys: the score's bits in an order that
// integers share, above the label's complement, so that one comparison ranks by
// score and then by smaller label, and 0 is below every label.  A label passes
// if its key is above the wave's k-th; those that pass gather in LDS, and 64 of
// them at a time are sorted across the lanes and merged into the list.  The lists of
// the waves are merged in LDS, those of a row's pieces by k_rank_join.
//
// Penalties touch few labels: the occurrences of a row's `seen` ids are counted
// in LDS (integers: any order gives the same count) for SUB columns at a time, as are the last entries of row_bias,
// and labels that neither list names take none of that arithmetic.
#include <math.h>

#include "asgd_dev.h"
#include "asgd_kernels.h"
#include "logits_dev.h"

namespace asgd {

namespace {

constexpr int RK_THREADS = 256;
constexpr int RK_WAVES = RK_THREADS / 64;
constexpr int RK_U = 2;       // vectors per lane and round
constexpr int RK_SUB = 4096;  // columns whose penalties are in LDS at a time
constexpr int RK_NONE = 0x7fffffff;

// Bits of a float in an order that unsigned integers share; every number's is above 0.
__device__ __forceinline__ unsigned order_of(float v) {
  const unsigned u = __float_as_uint(v);
  return (int)u < 0 ? ~u : u | 0x80000000u;
}
__device__ __forceinline__ float of_order(unsigned o) {
  return __uint_as_float((int)o < 0 ? o & 0x7fffffffu : ~o);
}
__device__ __forceinline__ u64 key_of(float v, int label) { return ((u64)order_of(v) << 32) | (unsigned)~label; }

__device__ __forceinline__ u64 swap_lanes(u64 v, int x) { return __shfl_xor(v, x); }

// Sorts the lanes' keys in descending order.
__device__ __forceinline__ u64 sort64(u64 v, int lane) {
#pragma unroll
  for (int size = 2; size <= 64; size *= 2)
#pragma unroll
    for (int d = size / 2; d >= 1; d /= 2) {
      const u64 o = swap_lanes(v, d);
      const bool big = ((lane & d) == 0) == ((lane & size) == 0);
      v = (o > v) == big ? o : v;
    }
  return v;
}

// The 64 best of two lists in descending order.
__device__ __forceinline__ u64 merge64(u64 a, u64 b, int lane) {
  const u64 r = __shfl(b, 63 - lane);
  u64 v = a > r ? a : r;
#pragma unroll
  for (int d = 32; d >= 1; d /= 2) {
    const u64 o = swap_lanes(v, d);
    v = (o > v) == ((lane & d) == 0) ? o : v;
  }
  return v;
}

struct Best {
  u64 list;  // lane i: the i-th best
  u64 least;  // the k-th best
  int n;     // keys waiting in buf
  u64* buf;  // LDS, 128 keys of this wave

  __device__ void flush(int lane, int k, int count) {
    __builtin_amdgcn_fence(__ATOMIC_SEQ_CST, "wavefront");
    const u64 v = lane < count ? buf[n - count + lane] : 0;
    __builtin_amdgcn_fence(__ATOMIC_SEQ_CST, "wavefront");
    n -= count;
    list = merge64(list, sort64(v, lane), lane);
    least = __shfl(list, k - 1);
  }
  // All lanes call it; key 0 never passes.
  __device__ void offer(u64 key, int lane, int k) {
    const bool in = key > least;
    const u64 who = __ballot(in);
    if (!who) return;
    if (in) buf[n + __builtin_amdgcn_mbcnt_hi((unsigned)(who >> 32), __builtin_amdgcn_mbcnt_lo((unsigned)who, 0))] = key;
    n += __popcll(who);
    if (n >= 64) flush(lane, k, 64);
  }
};

// Bits of the columns c .. c + v - 1 in a row's mask of `words` words.
__device__ __forceinline__ unsigned mask_bits(const uint32_t* m, int words, int c, int v) {
  if (c < 0) return m[0] << -c;
  const int w = c >> 5, sh = c & 31;
  if (w >= words) return 0;
  u64 b = m[w];
  if (sh + v > 32 && w + 1 < words) b |= (u64)m[w + 1] << 32;
  return (unsigned)(b >> sh);
}

// Writes the first k of a wave's list as ids and scores, or as keys.
__device__ __forceinline__ void put_best(u64 key, int lane, int k, int64_t row, int32_t* ids, float* scores) {
  if (lane >= k) return;
  ids[row * k + lane] = key ? (int)~(unsigned)key : RK_NONE;
  if (scores) scores[row * k + lane] = key ? of_order((unsigned)(key >> 32)) : -INFINITY;
}

__device__ __forceinline__ float lse_of(float m, float s) {
  if (m == -INFINITY || m == INFINITY) return m;
  return m + __builtin_amdgcn_logf(s) * LN2;
}

template <typename T>
__global__ __launch_bounds__(RK_THREADS) void k_rank(const T* __restrict__ z, int64_t ld, int L, RankRules ru, int k,
                                                     int splits, int vec_split, u64* __restrict__ part,
                                                     float2* __restrict__ part_ms, int32_t* __restrict__ ids,
                                                     float* __restrict__ scores, float* __restrict__ lse) {
  using R = Row<T>;
  constexpr int V = R::V;
  constexpr int SUBV = RK_SUB / V;
  __shared__ u64 buf[RK_WAVES][128];
  __shared__ float2 red[RK_WAVES];
  extern __shared__ int touched[];  // counts [RK_SUB], then last row_bias entries [RK_SUB]
  int* const count = touched;
  int* const last = touched + RK_SUB;
  const int lane = threadIdx.x & 63;
  const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  const int row = blockIdx.x / splits, split = blockIdx.x % splits;
  const R zr(const_cast<T*>(z), ld, row, L);
  const int v0 = split * vec_split, v1 = min(zr.n_vec, v0 + vec_split);
  const uint32_t* mask = ru.allowed ? ru.allowed + (int64_t)row * ru.allowed_ld : nullptr;
  const int words = (L + 31) >> 5;
  int s0 = 0, s1 = 0, b0 = 0, b1 = 0;
  if (ru.seen.indptr) list_range(ru.seen, row, &s0, &s1);
  if (ru.row_bias.indptr) list_range(ru.row_bias, row, &b0, &b1);
  const bool lists = s1 > s0 || b1 > b0;

  Best best{0, 0, 0, buf[wave]};
  float m = -INFINITY, s = 0.0f;
  for (int w0 = v0; w0 < v1; w0 += SUBV) {
    const int w1 = min(v1, w0 + SUBV), c0 = zr.col(w0);
    if (lists) {
      __syncthreads();
      for (int i = threadIdx.x; i < 2 * RK_SUB; i += RK_THREADS) touched[i] = 0;
      __syncthreads();
      for (int q = s0 + (int)threadIdx.x; q < s1; q += RK_THREADS) {
        const int id = ru.seen.indices[q];
        if (id >= 0 && id < L && (unsigned)(id - c0) < (unsigned)RK_SUB) atomicAdd(&count[id - c0], 1);
      }
      for (int q = b0 + (int)threadIdx.x; q < b1; q += RK_THREADS) {
        const int id = ru.row_bias.indices[q];
        if (id >= 0 && id < L && (unsigned)(id - c0) < (unsigned)RK_SUB) atomicMax(&last[id - c0], q - b0 + 1);
      }
      __syncthreads();
    }
    for (int base = w0; base < w1; base += RK_THREADS * RK_U) {
      float x[RK_U][V];
      unsigned ok[RK_U];
#pragma unroll
      for (int u = 0; u < RK_U; ++u) {
        const int i = base + u * RK_THREADS + (int)threadIdx.x;
        ok[u] = i < w1 ? zr.in_row(i) : 0;
        if (mask && ok[u]) ok[u] &= mask_bits(mask, words, zr.col(i), V);
        if (ok[u]) zr.load(i, ok[u], x[u]);
      }
      float mx = -INFINITY;
#pragma unroll
      for (int u = 0; u < RK_U; ++u) {
        const int c = zr.col(base + u * RK_THREADS + (int)threadIdx.x);
#pragma unroll
        for (int e = 0; e < V; ++e) {
          const bool on = (ok[u] >> e) & 1;
          float v = on ? x[u][e] : 0.0f;
          // (+ 0: a negative zero ties with zero)
          const float b = ru.bias && on ? ru.bias[c + e] : 0.0f;
          int n = 0, l = 0;
          if (lists && on) {
            n = count[c + e - c0];
            l = last[c + e - c0];
          }
          if (n | l) {
            double t = v;
            if (n) t = (t > 0.0 ? t / ru.repetition : t * ru.repetition) - ru.frequency * (double)n - ru.presence;
            t += (double)b;
            if (l) t += (double)ru.row_bias.values[b0 + l - 1];
            v = (float)t + 0.0f;
          } else {
            v += b;
          }
          if (!on || v != v) {
            ok[u] &= ~(1u << e);
            v = -INFINITY;
          }
          x[u][e] = v;
          mx = fmaxf(mx, v);
          best.offer((ok[u] >> e) & 1 ? key_of(v, c + e) : 0, lane, k);
        }
      }
      if (lse) {
        if (mx > m) {
          s = m == -INFINITY ? 0.0f : s * __builtin_amdgcn_exp2f((m - mx) * LOG2E);
          m = mx;
        }
        if (m != -INFINITY) {
#pragma unroll
          for (int u = 0; u < RK_U; ++u)
#pragma unroll
            for (int e = 0; e < V; ++e)
              s += x[u][e] == -INFINITY ? 0.0f : __builtin_amdgcn_exp2f((x[u][e] - m) * LOG2E);
        }
      }
    }
  }
  if (best.n) best.flush(lane, k, best.n);
  if (lse) {
#pragma unroll
    for (int o = 32; o >= 1; o >>= 1) soft_merge(m, s, __shfl_xor(m, o), __shfl_xor(s, o), LOG2E);
    if (lane == 0) red[wave] = make_float2(m, s);
  }
  buf[wave][lane] = best.list;
  __syncthreads();
  if (wave) return;
  for (int w = 1; w < RK_WAVES; ++w) {
    best.list = merge64(best.list, buf[w][lane], lane);
    if (lse) soft_merge(m, s, red[w].x, red[w].y, LOG2E);
  }
  if (splits == 1) {
    put_best(best.list, lane, k, row, ids, scores);
    if (lse && lane == 0) lse[row] = lse_of(m, s);
  } else {
    if (lane < k) part[(int64_t)blockIdx.x * k + lane] = best.list;
    if (lse && lane == 0) part_ms[blockIdx.x] = make_float2(m, s);
  }
}

// Per row: the k best of its pieces' lists, and lse of their sums, in a fixed order.
__global__ __launch_bounds__(RK_THREADS) void k_rank_join(int splits, int k, const u64* __restrict__ part,
                                                          const float2* __restrict__ part_ms,
                                                          int32_t* __restrict__ ids, float* __restrict__ scores,
                                                          float* __restrict__ lse) {
  __shared__ u64 buf[RK_WAVES][64];
  __shared__ float2 red[RK_WAVES];
  const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
  const int64_t row = blockIdx.x;
  const int n = splits * k;
  const u64* p = part + row * n;
  u64 list = 0, least = 0;
  for (int i = wave * 64; i < n; i += RK_THREADS) {
    const u64 v = i + lane < n ? p[i + lane] : 0;
    if (!__ballot(v > least)) continue;
    list = merge64(list, sort64(v, lane), lane);
    least = __shfl(list, k - 1);
  }
  float m = -INFINITY, s = 0.0f;
  if (lse) {
    for (int i = threadIdx.x; i < splits; i += RK_THREADS) {
      const float2 ms = part_ms[row * splits + i];
      soft_merge(m, s, ms.x, ms.y, LOG2E);
    }
#pragma unroll
    for (int o = 32; o >= 1; o >>= 1) soft_merge(m, s, __shfl_xor(m, o), __shfl_xor(s, o), LOG2E);
    if (lane == 0) red[wave] = make_float2(m, s);
  }
  buf[wave][lane] = list;
  __syncthreads();
  if (wave) return;
  for (int w = 1; w < RK_WAVES; ++w) {
    list = merge64(list, buf[w][lane], lane);
    if (lse) soft_merge(m, s, red[w].x, red[w].y, LOG2E);
  }
  put_best(list, lane, k, row, ids, scores);
  if (lse && lane == 0) lse[row] = lse_of(m, s);
}

// Pieces per row: enough workgroups to fill the GPU, each with at least one full round.
RankShape shape_of(int rows, int cols) {
  RankShape sh;
  const int want = (2048 + rows - 1) / rows;
  const int most = (cols + RK_SUB - 1) / RK_SUB;
  sh.splits = want < most ? want : most;
  if (sh.splits < 1) sh.splits = 1;
  return sh;
}

}  // namespace

RankShape rank_shape(int rows, int cols) { return shape_of(rows, cols); }

size_t rank_ws_bytes(const RankShape& sh, int rows, int k) {
  if (sh.splits == 1) return 0;
  const size_t keys = ((size_t)rows * sh.splits * k * sizeof(u64) + 255) / 256 * 256;
  return keys + (size_t)rows * sh.splits * sizeof(float2);
}

template <typename T>
static hipError_t rank_as(const void* z, int64_t ld, int rows, int L, const RankRules& ru, int k, const RankShape& sh,
                          int32_t* ids, float* scores, float* lse, void* ws, hipStream_t st) {
  // vectors of a row of any phase, and per piece
  const int n_vec = (L + 2 * Row<T>::V - 2) / Row<T>::V;
  const int vps = (n_vec + sh.splits - 1) / sh.splits;
  u64* part = (u64*)ws;
  float2* ms = (float2*)((char*)ws + ((size_t)rows * sh.splits * k * sizeof(u64) + 255) / 256 * 256);
  const int lds = ru.seen.indptr || ru.row_bias.indptr ? 2 * RK_SUB * (int)sizeof(int) : 0;
  hipLaunchKernelGGL(k_rank<T>, dim3((unsigned)rows * sh.splits), dim3(RK_THREADS), lds, st, (const T*)z, ld, L, ru,
                     k, sh.splits, vps, part, ms, ids, scores, lse);
  if (sh.splits > 1)
    hipLaunchKernelGGL(k_rank_join, dim3(rows), dim3(RK_THREADS), 0, st, sh.splits, k, part, ms, ids, scores, lse);
  return hipGetLastError();
}

hipError_t launch_rank(int dtype, const void* z, int64_t ld, int rows, int L, const RankRules& ru, int k,
                       const RankShape& sh, int32_t* ids, float* scores, float* lse, void* ws, hipStream_t st) {
  if (dtype == 0) return rank_as<float>(z, ld, rows, L, ru, k, sh, ids, scores, lse, ws, st);
  if (dtype == 1) return rank_as<bf16>(z, ld, rows, L, ru, k, sh, ids, scores, lse, ws, st);
  return rank_as<f16>(z, ld, rows, L, ru, k, sh, ids, scores, lse, ws, st);
}

}  // namespace asgd

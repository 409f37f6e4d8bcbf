// The k best labels of logit rows under rules (asgd_logits_topk).
//
// One pass over the logits.  A workgroup takes one piece of one row; each of
// its waves keeps the 64 best (score, label) pairs that it has met, one per
// lane in descending order, as 64-bit keys: the score's bits in an order that
// integers share, above the label's complement, so that one comparison ranks by
// score and then by smaller label, and 0 is below every label.  A lane's largest score of
// a round of loads is compared with the k-th best so far (of any wave of the
// workgroup); only a round that has something above it looks at its labels one by
// one.  Those gather in LDS, are sorted across the lanes 64 at a time, and merge into the list.
// The first round starts from the k-th largest of its lanes' maxima, so that few of its labels
// pass.  The lists of the waves are merged in LDS, those of a row's pieces by k_rank_join.
// A label that is not ranked (not allowed, NaN) carries a NaN through the arithmetic, which
// maxima and comparisons leave out.
//
// Penalties touch few labels.  The pieces skip every label that `seen` or `row_bias`
// name (one bit per column in LDS), and more workgroups per row, each with a range of labels, look only at those: a
// hash table in LDS counts occurrences (integers: any order gives the same count), keeps
// the last row_bias entry and the first entry that names a label, and that entry's thread
// forms the label's score in float64, so sums follow the lists' order.  A range with more
// labels than the table holds is counted 1,024 columns at a time.
//
// Measured: 1,024 x 670,091 fp32, k = 5, all rules, 551 us for 2.83 GB (5.1 TB/s: memory; the biases of rows that
// start at odd places are not aligned: without biases 430, with aligned rows 478; aligned loads whose elements
// neighbouring lanes pass on took 747, their branches end the loads' overlap); 256 x 205,443 bf16, k = 32, all
// rules, 48 us, of which k_rank_join 4 (112 MB at 2.4 TB/s: vector units busy 68 % of k_rank; without rules 41, without lse too 33, with
// k = 1 besides 24); one row of 670,091 13 to 15 us in two launches of 8.6 and 4.8 (no rules 7.2 and 4.9: listed labels
// add 1.0, biases nothing; without lse 6.3 and 4.4, with k = 1 7.7 and 3.9).  Many distinct listed labels in one range
// are slow: 256 x 670,091 fp32 with 40 in every row 122 us, with 900 | 3,000 in one of the rows 1,260 | 2,310.
#include <math.h>

#include <algorithm>

#include "asgd_dev.h"
#include "asgd_kernels.h"
#include "logits_dev.h"

namespace asgd {

namespace {

constexpr int RK_THREADS = 256;
constexpr int RK_WAVES = RK_THREADS / 64;
constexpr int RK_BITS = 1 << 17;   // columns of a piece at most where lists are given (as many bits as the table takes)
constexpr int RK_SLOTS = 1024;     // the table of listed labels
constexpr int RK_PROBES = 32;
constexpr int RK_RANGES = 32;     // ranges of listed labels per row at most
constexpr int RK_WGS = 1024;      // workgroups wanted
constexpr int RK_NONE = 0x7fffffff;

// Bits of a float in an order that unsigned integers share; every number's is above 0.
__device__ __forceinline__ unsigned order_of(float v) {
  const unsigned u = __float_as_uint(v);
  return (int)u < 0 ? ~u : u | 0x80000000u;
}
__device__ __forceinline__ float of_order(unsigned o) {
  return __uint_as_float((int)o < 0 ? o & 0x7fffffffu : ~o);
}
// (+ 0: a negative zero ties with zero)
__device__ __forceinline__ u64 key_of(float v, int label) {
  return ((u64)order_of(v + 0.0f) << 32) | (unsigned)~label;
}

__device__ __forceinline__ unsigned lane_of(unsigned v, int l) { return (unsigned)__builtin_amdgcn_readlane((int)v, l); }
__device__ __forceinline__ u64 lane_of(u64 v, int l) {
  return ((u64)lane_of((unsigned)(v >> 32), l) << 32) | lane_of((unsigned)v, l);
}

// Bit l: of lanes l and l ^ D, l keeps the larger key, in runs of SIZE that alternate between
// descending and ascending.
constexpr u64 keeps_larger(int D, int SIZE) {
  u64 b = 0;
  for (int l = 0; l < 64; ++l) b |= (u64)(((l & D) == 0) == ((l & SIZE) == 0)) << l;
  return b;
}
// One step of a bitonic network over the lanes, D apart.  (The lanes' roles as a constant: as
// comparisons of the lane they would take a scalar register pair each through the whole kernel.)
template <int D, int SIZE, typename K>
__device__ __forceinline__ K bitonic_step(K v, int lane) {
  const K o = lane_xor<D>(v, lane);
  constexpr u64 KEEPS = keeps_larger(D, SIZE);
  const bool big = __builtin_amdgcn_inverse_ballot_w64(KEEPS);
  return (o > v) == big ? o : v;
}
template <int D, int SIZE, typename K>
__device__ __forceinline__ K bitonic_merge(K v, int lane) {
  v = bitonic_step<D, SIZE>(v, lane);
  if constexpr (D > 1) v = bitonic_merge<D / 2, SIZE>(v, lane);
  return v;
}
// Sorts the lanes' keys in descending order.
template <typename K>
__device__ __forceinline__ K sort64(K v, int lane) {
  v = bitonic_merge<1, 2>(v, lane);
  v = bitonic_merge<2, 4>(v, lane);
  v = bitonic_merge<4, 8>(v, lane);
  v = bitonic_merge<8, 16>(v, lane);
  v = bitonic_merge<16, 32>(v, lane);
  return bitonic_merge<32, 64>(v, lane);
}

// The 64 best of two lists, the second one in ascending order.
__device__ __forceinline__ u64 merge64(u64 a, u64 r, int lane) {
  return bitonic_merge<32, 64>(a > r ? a : r, lane);
}
__device__ __forceinline__ u64 reverse64(u64 v, int lane) { return __shfl(v, 63 - lane); }

// What the waves of a workgroup have found, in LDS: k labels of a wave are as good as `kth`,
// ceil(k / waves) as good as `part`.  So the workgroup's k-th best is at least the largest
// kth and the smallest part, and labels below that need not be looked at by any wave: `bound`.
template <int WAVES>
struct Found {
  u64 bound, part[WAVES];
};

struct Best {
  u64 list;   // lane i: the i-th best
  u64 least;  // keys up to it need not be looked at
  u64 part;   // what this wave published
  int n;      // keys waiting in buf
  u64* buf;   // LDS, 128 keys of this wave

  // Appends the lanes' keys that are above the bound (0 never is): at most 64 to at most 63.
  __device__ void append(u64 key) {
    const bool in = key > least;
    const u64 who = __ballot(in);
    if (in) buf[n + __builtin_amdgcn_mbcnt_hi((unsigned)(who >> 32), __builtin_amdgcn_mbcnt_lo((unsigned)who, 0))] = key;
    n += __popcll(who);
  }
  // Takes up to 64 waiting keys into the list.
  __device__ void flush(int lane) {
    const int count = min(n, 64);
    __builtin_amdgcn_fence(__ATOMIC_SEQ_CST, "wavefront");
    const u64 v = lane < count ? buf[n - count + lane] : 0;
    __builtin_amdgcn_fence(__ATOMIC_SEQ_CST, "wavefront");
    n -= count;
    list = merge64(list, reverse64(sort64(v, lane), lane), lane);
  }
  template <int WAVES>
  __device__ void publish(Found<WAVES>& f, u64 kth, u64 p, int lane, int wave) {
    static_assert(WAVES == 4);
    part = p > part ? p : part;
    if (lane == 0) *(volatile u64*)&f.part[wave] = part;
    u64 b = *(const volatile u64*)&f.part[lane & 3];
    u64 o = lane_xor<1>(b, lane);
    b = o < b ? o : b;
    o = lane_xor<2>(b, lane);
    b = o < b ? o : b;
    b = b ? b - 1 : 0;  // (a key equal to it passes: it may be the k-th)
    b = b > kth ? b : kth;
    if (lane == 0) atomicMax(&f.bound, b);
    b = lane_of(b, 0);
    least = b > least ? b : least;
  }
  template <int WAVES>
  __device__ void publish_list(Found<WAVES>& f, int lane, int wave, int k) {
    publish(f, lane_of(list, k - 1), lane_of(list, (k + WAVES - 1) / WAVES - 1), lane, wave);
  }
  template <int WAVES>
  __device__ void look(const Found<WAVES>& f) {
    const u64 t = lane_of(*(const volatile u64*)&f.bound, 0);
    least = t > least ? t : least;
  }
  // Scores below it do not pass.
  __device__ float bound() const {
    const unsigned o = (unsigned)(least >> 32);
    return o > 0x007fffffu ? of_order(o) : -INFINITY;  // (0x007fffff: -inf)
  }
};

// Writes the first k of a wave's list as ids and scores, or as keys.
__device__ __forceinline__ void put_best(u64 key, int lane, int k, int64_t row, int32_t* ids, float* scores) {
  if (lane >= k) return;
  ids[row * k + lane] = key ? (int)~(unsigned)key : RK_NONE;
  if (scores) scores[row * k + lane] = key ? of_order((unsigned)(key >> 32)) : -INFINITY;
}

// A row's sum of e^score as (m, s): the sum is s 2^m.  m is a whole number (or infinite), so a
// term 2^(score log2 e - m) takes one fused product and one exponential, and is at most
// 1: its clamp to [0, 1] turns the NaN of a label that is not ranked into 0.
__device__ __forceinline__ float term2(float v, float m) {
  return __builtin_amdgcn_fmed3f(__builtin_amdgcn_exp2f(fmaf(v, LOG2E, -m)), 0.0f, 1.0f);
}
__device__ __forceinline__ void raise2(float v, float& m, float& s) {
  const float c = ceilf(v * LOG2E);
  if (c > m) {
    s = m == -INFINITY ? 0.0f : s * __builtin_amdgcn_exp2f(m - c);
    m = c;
  }
}
__device__ __forceinline__ void merge2(float& m, float& s, float m2, float s2) { soft_merge(m, s, m2, s2, 1.0f); }
// The row's log-sum-exp; best: its best key.  From 2^28 on the sum's logarithm, at most ln 2^22 = 15.3, is below
// half a step (16; a step above -2^28 itself) of the best score, which is then the answer.  Below that the product that m is
// taken from is below 2^29 and its rounding at most 16, so the best label's term neither vanishes nor
// loses more to its clamp than a step of the score; far above it that rounding passes the exponents of floats.
__device__ __forceinline__ float lse_of(u64 best, float m, float s) {
  if (!best) return -INFINITY;
  const float top = of_order((unsigned)(best >> 32));
  return fabsf(top) < 268435456.0f ? (m + __builtin_amdgcn_logf(s)) * LN2 : top;
}

// (m, s) of all lanes as one, on all of them: the largest m, and the sums under it.
template <int X>
__device__ __forceinline__ float float_xor(float v, int lane) {
  return __uint_as_float(lane_xor<X>(__float_as_uint(v), lane));
}
__device__ __forceinline__ void merge2_wave(float& m, float& s, int lane) {
  float t = m;
  t = fmaxf(t, float_xor<1>(t, lane));
  t = fmaxf(t, float_xor<2>(t, lane));
  t = fmaxf(t, float_xor<4>(t, lane));
  t = fmaxf(t, float_xor<8>(t, lane));
  t = fmaxf(t, float_xor<16>(t, lane));
  t = fmaxf(t, float_xor<32>(t, lane));
  s = m == -INFINITY ? 0.0f : s * __builtin_amdgcn_exp2f(m - t);
  m = t;
  s += float_xor<1>(s, lane);
  s += float_xor<2>(s, lane);
  s += float_xor<4>(s, lane);
  s += float_xor<8>(s, lane);
  s += float_xor<16>(s, lane);
  s += float_xor<32>(s, lane);
}
// The lists of the waves of a workgroup as one, on wave 0; likewise (m, s) on its lanes.
template <int WAVES, int STRIDE>
__device__ __forceinline__ void gather_waves(u64& list, float& m, float& s, bool sums, u64 (*lists)[STRIDE], float2* red,
                                             int lane, int wave) {
  if (sums) {
    merge2_wave(m, s, lane);
    if (lane == 0) red[wave] = make_float2(m, s);
  }
#pragma unroll 1
  for (int d = 1; d < WAVES; d *= 2) {
    if ((wave & (2 * d - 1)) == d) lists[wave][63 - lane] = list;
    __syncthreads();
    if ((wave & (2 * d - 1)) == 0) list = merge64(list, lists[wave + d][lane], lane);
  }
  if (sums && wave == 0) {
    const float2 r = lane < WAVES ? red[lane] : make_float2(-INFINITY, 0.0f);
    m = r.x;
    s = r.y;
    merge2_wave(m, s, lane);
  }
}

struct Table {
  int id[RK_SLOTS], count[RK_SLOTS], last[RK_SLOTS], first[RK_SLOTS];
};

__device__ __forceinline__ unsigned slot_of(int id) { return ((unsigned)id * 2654435761u) >> 22; }
// The slot that holds id (put there if absent), or -1 after RK_PROBES others.
__device__ __forceinline__ int table_put(Table& t, int id) {
  unsigned h = slot_of(id);
  for (int p = 0; p < RK_PROBES; ++p, h = (h + 1) & (RK_SLOTS - 1)) {
    const int was = atomicCAS(&t.id[h], -1, id);
    if (was == -1 || was == id) return (int)h;
  }
  return -1;
}

// A listed label's logit and bias, and whether it is allowed.
struct Listed {
  float z, bias;
  bool allowed;
};
template <typename T>
__device__ __forceinline__ Listed listed_load(const T* zrow, const RankRules& ru, const uint32_t* mask, int id) {
  return {(float)zrow[id], ru.bias ? ru.bias[id] : 0.0f, !mask || ((mask[id >> 5] >> (id & 31)) & 1)};
}
// Its score: n occurrences in seen, and the last of the row_bias entries from b0 on (1-based, 0:
// none).  NaN if it is not ranked.
__device__ __forceinline__ float listed_score(const Listed& l, const RankRules& ru, int n, int last, int b0) {
  if (!l.allowed) return NAN;
  double t = (double)l.z;
  if (n) t = (t > 0.0 ? t / ru.repetition : t * ru.repetition) - ru.frequency * (double)n - ru.presence;
  t += (double)l.bias;
  if (last) t += (double)ru.row_bias.values[b0 + last - 1];
  return (float)t;
}

// The listed labels in [lo, hi).
template <typename T>
__device__ void rank_listed(const T* zrow, const RankRules& ru, const uint32_t* mask, int lo, int hi, int s0, int s1,
                            int b0, int b1, Table& t, int* overflow, Best& best, float& m, float& s, int lane) {
  const int tid = threadIdx.x, ns = s1 - s0, n = ns + (b1 - b0);
  auto entry = [&](int i) {
    const int id = i < ns ? ru.seen.indices[s0 + i] : ru.row_bias.indices[b0 + i - ns];
    return id >= lo && id < hi ? id : -1;
  };
  auto take = [&](float v, int id) {
    best.append(v == v ? key_of(v, id) : 0);
    if (best.n >= 64) best.flush(lane);
    if (v == v) {
      raise2(v, m, s);
      if (m != -INFINITY) s += term2(v, m);
    }
  };
  // (a thread's first entry and what it leads to are on their way while the table is made)
  const int id0 = tid < n ? entry(tid) : -1;
  Listed l0{};
  if (id0 >= 0) l0 = listed_load(zrow, ru, mask, id0);
  for (int i = tid; i < RK_SLOTS; i += RK_THREADS) {
    t.id[i] = -1;
    t.count[i] = t.last[i] = 0;
    t.first[i] = n;
  }
  if (tid == 0) *overflow = 0;
  __syncthreads();
  for (int i = tid; i < n; i += RK_THREADS) {
    const int id = i == tid ? id0 : entry(i);
    if (id < 0) continue;
    const int h = table_put(t, id);
    if (h < 0) {
      *overflow = 1;
      break;
    }
    atomicMin(&t.first[h], i);
    if (i < ns)
      atomicAdd(&t.count[h], 1);
    else
      atomicMax(&t.last[h], i - ns + 1);
  }
  __syncthreads();
  if (!*overflow) {
    for (int i0 = 0; i0 < n; i0 += RK_THREADS) {
      const int i = i0 + tid, id = i0 == 0 ? id0 : i < n ? entry(i) : -1;
      float v = NAN;
      if (id >= 0) {
        unsigned h = slot_of(id);
        while (t.id[h] != id) h = (h + 1) & (RK_SLOTS - 1);  // (it is there)
        if (t.first[h] == i)
          v = listed_score(i0 == 0 ? l0 : listed_load(zrow, ru, mask, id), ru, t.count[h], t.last[h], b0);
      }
      take(v, id);
    }
    return;
  }
  for (int c0 = lo; c0 < hi; c0 += RK_SLOTS) {
    __syncthreads();
    for (int i = tid; i < RK_SLOTS; i += RK_THREADS) t.count[i] = t.last[i] = 0;
    __syncthreads();
    for (int i = tid; i < n; i += RK_THREADS) {
      const int id = entry(i);
      if (id < 0 || (unsigned)(id - c0) >= (unsigned)RK_SLOTS) continue;
      if (i < ns)
        atomicAdd(&t.count[id - c0], 1);
      else
        atomicMax(&t.last[id - c0], i - ns + 1);
    }
    __syncthreads();
    for (int i = tid; i < RK_SLOTS; i += RK_THREADS) {
      const int c = t.count[i], l = t.last[i];
      take(c | l ? listed_score(listed_load(zrow, ru, mask, c0 + i), ru, c, l, b0) : NAN, c0 + i);
    }
  }
}

template <int N>
struct __attribute__((packed, aligned(4))) Floats {
  float v[N];
};

// Workgroup = (piece, row): `splits` pieces of columns and, with LISTS, `ranges` ranges of
// listed labels; no ranges: one piece, whose workgroup looks at the listed labels first.
template <typename T, bool LISTS>
__global__ __launch_bounds__(RK_THREADS) void k_rank(const T* __restrict__ z, int64_t ld, int L, RankRules ru, int k,
                                                     int splits, int ranges, int vec_split, u64* __restrict__ part,
                                                     float2* __restrict__ part_ms, int32_t* __restrict__ ids,
                                                     float* __restrict__ scores, float* __restrict__ lse) {
  using R = Row<T>;
  constexpr int V = R::V, RK_U = 2, ROUND = RK_THREADS * RK_U;
  constexpr unsigned ALL = (1u << V) - 1;
  __shared__ u64 buf[RK_WAVES][128];
  __shared__ float2 red[RK_WAVES];
  __shared__ Found<RK_WAVES> found;
  __shared__ union Lists {
    unsigned bits[LISTS ? RK_BITS / 32 : 1];
    char table[LISTS ? sizeof(Table) : 1];
  } in;
  __shared__ int overflow;
  __shared__ unsigned edge_bits;
  const int lane = threadIdx.x & 63;
  const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  const int parts = splits + ranges;
  // (rows side by side: workgroups that run together read the same columns' biases)
  const int n_rows = (int)(gridDim.x / (unsigned)parts), row = blockIdx.x % n_rows, piece = blockIdx.x / n_rows;
  const R zr(const_cast<T*>(z), ld, row, L);
  const uint32_t* mask = ru.allowed ? ru.allowed + (int64_t)row * ru.allowed_ld : nullptr;
  const int words = (L + 31) >> 5;
  Best best{0, 0, 0, 0, buf[wave]};
  float m = -INFINITY, s = 0.0f;
  if (threadIdx.x <= RK_WAVES) (&found.bound)[threadIdx.x] = 0;

  int s0 = 0, s1 = 0, b0 = 0, b1 = 0;
  bool lists = false;
  if constexpr (LISTS) {
    if (ru.seen.indptr) list_range(ru.seen, row, &s0, &s1);
    if (ru.row_bias.indptr) list_range(ru.row_bias, row, &b0, &b1);
    lists = s1 > s0 || b1 > b0;
  }
  if (LISTS && (piece >= splits || ranges == 0)) {
    const int width = ranges ? (L + ranges - 1) / ranges : L, lo = ranges ? (piece - splits) * width : 0;
    __syncthreads();
    if (lists)
      rank_listed(zr.base + zr.phase, ru, mask, lo, min(L, lo + width), s0, s1, b0, b1,
                  *reinterpret_cast<Table*>(in.table), &overflow, best, m, s, lane);
    if (ranges == 0) __syncthreads();  // (the table's memory holds bits next)
  }
  if (!LISTS || piece < splits) {
    // whole vectors [va, vb) are shared out; the first piece's first wave takes the labels before and after them
    const int va = zr.phase ? 1 : 0, vb = max(va, (zr.phase + L) / V);
    const int v0 = va + piece * vec_split, v1 = max(v0, min(vb, v0 + vec_split)), c0 = zr.col(v0);
    const int head = min(L, zr.col(va)), tail = min(L, max(head, zr.col(vb)));
    // Rounds of loads: a round's logits and biases are on their way while the one before it is
    // worked on, and its words of the mask while the one before that is.  Lanes past the
    // piece's end load its last vector again.
    typename R::vec x[RK_U];
    Floats<V> bias[RK_U];
    unsigned ok[RK_U], m0[RK_U], m1[RK_U];
    const int rounds = (v1 - v0 + ROUND - 1) / ROUND;
    const int first = v0 + (int)threadIdx.x;
    auto load_mask = [&](int r) {
#pragma unroll
      for (int u = 0; u < RK_U; ++u) {
        const int w = zr.col(min(first + r * ROUND + u * RK_THREADS, v1 - 1)) >> 5;
        m0[u] = mask[(unsigned)w];
        m1[u] = mask[(unsigned)min(w + 1, words - 1)];
      }
    };
    auto load = [&](int r) {
#pragma unroll
      for (int u = 0; u < RK_U; ++u) {
        const int i = first + r * ROUND + u * RK_THREADS, j = min(i, v1 - 1), c = zr.col(j);
        unsigned o = i == j ? ALL : 0;
        if (mask) o &= __builtin_amdgcn_alignbit(m1[u], m0[u], c & 31);
        ok[u] = o;
        if (!__ballot(o != 0)) continue;
        x[u] = __builtin_nontemporal_load(
            reinterpret_cast<const typename R::vec*>(reinterpret_cast<const char*>(zr.base) + (unsigned)(16 * j)));
        if (ru.bias)
          bias[u] = *reinterpret_cast<const Floats<V>*>(reinterpret_cast<const char*>(ru.bias) + (unsigned)(4 * c));
      }
    };
    if (rounds) {
      if (mask) load_mask(0);
      load(0);
      if (mask && rounds > 1) load_mask(1);
    }
    if (lists) {
      for (int i = threadIdx.x; i < ((v1 - v0) * V + 31) / 32; i += RK_THREADS) in.bits[i] = 0;
      if (threadIdx.x == 0) edge_bits = 0;
      __syncthreads();
      const unsigned width = (unsigned)(v1 - v0) * V;
      auto skip = [&](int id) {
        const unsigned c = (unsigned)(id - c0);
        if (c < width) atomicOr(&in.bits[c >> 5], 1u << (c & 31));
        if (id >= 0 && id < L && (id < head || id >= tail)) atomicOr(&edge_bits, 1u << (id < head ? id : head + id - tail));
      };
      for (int q = s0 + (int)threadIdx.x; q < s1; q += RK_THREADS) skip(ru.seen.indices[q]);
      for (int q = b0 + (int)threadIdx.x; q < b1; q += RK_THREADS) skip(ru.row_bias.indices[q]);
    }
    __syncthreads();
    if (piece == 0 && wave == 0 && head + (L - tail) > 0) {
      float v = NAN;
      const int c = lane < head ? lane : tail + lane - head;
      if (c < L && !(mask && !((mask[c >> 5] >> (c & 31)) & 1)) && !(lists && ((edge_bits >> lane) & 1)))
        v = (float)zr.base[zr.phase + c] + (ru.bias ? ru.bias[c] : 0.0f);
      best.append(v == v ? key_of(v, c) : 0);
      if (best.n >= 64) best.flush(lane);  // (listed labels may wait too)
      raise2(v, m, s);
      if (m != -INFINITY) s += term2(v, m);
    }
    for (int r = 0; r < rounds; ++r) {
      const int base = v0 + r * ROUND;
      if (r) best.look(found);
      float w[RK_U][V];
      float mx = -INFINITY;
#pragma unroll
      for (int u = 0; u < RK_U; ++u) {
        if (ru.bias) {
#pragma unroll
          for (int e = 0; e < V; ++e) w[u][e] = (float)x[u][e] + bias[u].v[e];
        } else {
#pragma unroll
          for (int e = 0; e < V; ++e) w[u][e] = (float)x[u][e];
        }
        if (LISTS && lists) {
          const int at = (min(first + r * ROUND + u * RK_THREADS, v1 - 1) - v0) * V;
          ok[u] &= ~(in.bits[at >> 5] >> (at & 31));
        }
        if (__ballot(ok[u] != ALL)) {
          const int off = (int)~ok[u];
#pragma unroll
          for (int e = 0; e < V; ++e)
            w[u][e] = __int_as_float(__float_as_int(w[u][e]) | (off << (31 - e) >> 31));  // a NaN
        }
#pragma unroll
        for (int e = 0; e < V; ++e) mx = fmaxf(mx, w[u][e]);
      }
      if (r + 1 < rounds) {
        load(r + 1);
        if (mask && r + 2 < rounds) load_mask(r + 2);
      }
      if (r == 0) {
        // (keys of the k-th largest maximum's score are above the bound)
        const unsigned tops = sort64(order_of(mx), lane);
        best.publish(found, ((u64)lane_of(tops, k - 1) << 32) - 1,
                     (u64)lane_of(tops, (k + RK_WAVES - 1) / RK_WAVES - 1) << 32, lane, wave);
      }
      const float bound = best.bound();
      if (__ballot(mx >= bound)) {
        unsigned pass = 0;
#pragma unroll
        for (int u = 0; u < RK_U; ++u)
#pragma unroll
          for (int e = 0; e < V; ++e) pass |= w[u][e] >= bound ? 1u << (u * V + e) : 0u;
        // one label of each lane at a time; the list takes them 64 at a time (as soon as k of them
        // wait: 62 us instead of 54 for 256 x 205,443 bf16 and k = 32, no difference for k = 5)
        do {
          const int at = pass ? __builtin_ctz(pass) : 0;
          float v = w[0][0];
#pragma unroll
          for (int j = 1; j < RK_U * V; ++j) v = at == j ? w[j / V][j % V] : v;
          const int c = zr.col(base + at / V * RK_THREADS + (int)threadIdx.x) + at % V;
          best.append(pass ? key_of(v, c) : 0);
          pass &= pass - 1;
          if (best.n >= 64) {
            best.flush(lane);
            best.publish_list(found, lane, wave, k);
          }
        } while (__ballot(pass != 0));
      }
      if (lse) {
        raise2(mx, m, s);
        if (m != -INFINITY) {
#pragma unroll
          for (int u = 0; u < RK_U; ++u)
#pragma unroll
            for (int e = 0; e < V; ++e) s += term2(w[u][e], m);
        }
      }
    }
  }
  if (best.n) best.flush(lane);
  gather_waves<RK_WAVES>(best.list, m, s, lse != nullptr, buf, red, lane, wave);
  if (wave) return;
  if (parts == 1) {
    put_best(best.list, lane, k, row, ids, scores);
    if (lse && lane == 0) lse[row] = lse_of(best.list, m, s);
  } else {
    if (lane < k) part[((int64_t)row * parts + piece) * k + lane] = best.list;
    if (lse && lane == 0) part_ms[(int64_t)row * parts + piece] = make_float2(m, s);
  }
}

// Per row: the k best of its pieces' lists, and lse of their sums, in a fixed order.
template <int WAVES>
__global__ __launch_bounds__(64 * WAVES) void k_rank_join(int parts, int k, const u64* __restrict__ part,
                                                          const float2* __restrict__ part_ms,
                                                          int32_t* __restrict__ ids, float* __restrict__ scores,
                                                          float* __restrict__ lse) {
  __shared__ u64 buf[WAVES][64];
  __shared__ float2 red[WAVES];
  const int lane = threadIdx.x & 63;
  const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  const int64_t row = blockIdx.x;
  const int n = parts * k;
  const u64* p = part + row * n;
  float m = -INFINITY, s = 0.0f;
  if (lse)
    for (int i = threadIdx.x; i < parts; i += 64 * WAVES) {
      const float2 ms = part_ms[row * parts + i];
      merge2(m, s, ms.x, ms.y);
    }
  u64 list = 0, least = 0;
  int i = wave * 64 + lane;
  u64 next = i < n ? p[i] : 0;
  for (; i - lane < n; i += 64 * WAVES) {
    const u64 v = next;
    if (i + 64 * WAVES < n) next = p[i + 64 * WAVES];
    else next = 0;
    if (!__ballot(v > least)) continue;
    list = merge64(list, reverse64(sort64(v, lane), lane), lane);
    least = lane_of(list, k - 1);
  }
  gather_waves<WAVES>(list, m, s, lse != nullptr, buf, red, lane, wave);
  if (wave) return;
  put_best(list, lane, k, row, ids, scores);
  if (lse && lane == 0) lse[row] = lse_of(list, m, s);
}

}  // namespace

// Pieces per row: enough workgroups to fill the GPU, each with two rounds of loads or more (one row of
// 670,091 under rules, at least 2,048 | 4,096 | 8,192 columns: 14.9 | 14.0 | 15.7 us); where lists are given, no more columns than a workgroup has bits for.
static int row_pieces(int rows, int cols, bool lists) {
  const int want = (RK_WGS + rows - 1) / rows, most = (cols + 4095) / 4096;
  const int least = lists ? (cols + RK_BITS - 1) / RK_BITS : 1;
  return std::max(std::min(want, most), least);
}

RankShape rank_shape(int rows, int cols) {
  return RankShape{row_pieces(rows, cols, true), std::max(1, std::min(RK_RANGES, 2048 / rows))};
}

// Ranges of listed labels per row: about 256 entries each.  (The scratch memory has room for
// the most, whatever the lists.)
static int rank_ranges(const RankShape& sh, const RankRules& ru, int rows) {
  const int64_t n = (ru.seen.indptr ? ru.seen.nnz : 0) + (int64_t)(ru.row_bias.indptr ? ru.row_bias.nnz : 0);
  if (!n) return 0;
  return (int)std::min<int64_t>(sh.ranges, (n + 256 * (int64_t)rows - 1) / (256 * (int64_t)rows));
}

static size_t key_bytes(const RankShape& sh, int rows, int k) {
  return ((size_t)rows * (sh.splits + sh.ranges) * k * sizeof(u64) + 255) / 256 * 256;
}

size_t rank_ws_bytes(const RankShape& sh, int rows, int k) {
  return key_bytes(sh, rows, k) + (size_t)rows * (sh.splits + sh.ranges) * sizeof(float2);
}

template <typename T>
static hipError_t rank_as(const void* z, int64_t ld, int rows, int L, const RankRules& ru, int k, const RankShape& sh,
                          int32_t* ids, float* scores, float* lse, void* ws, hipStream_t st) {
  int ranges = rank_ranges(sh, ru, rows);
  const bool lists = ranges > 0;
  const int splits = std::min(sh.splits, row_pieces(rows, L, lists));
  // (a row of one piece takes its lists along, which saves the join and a workgroup: 1,024 x
  // 40,000 fp32 with 10 listed labels a row 77 -> 47 us)
  if (splits == 1) ranges = 0;
  const int parts = splits + ranges;
  // whole vectors of a row at most, and per piece
  const int n_vec = L / Row<T>::V;
  const int vps = (n_vec + splits - 1) / splits;
  if (lists && (int64_t)vps * Row<T>::V > RK_BITS) return hipErrorInvalidValue;
  u64* part = (u64*)ws;
  float2* ms = (float2*)((char*)ws + key_bytes(sh, rows, k));
  const dim3 grid((unsigned)rows * parts), block(RK_THREADS);
  if (lists)
    hipLaunchKernelGGL((k_rank<T, true>), grid, block, 0, st, (const T*)z, ld, L, ru, k, splits, ranges, vps, part, ms,
                       ids, scores, lse);
  else
    hipLaunchKernelGGL((k_rank<T, false>), grid, block, 0, st, (const T*)z, ld, L, ru, k, splits, 0, vps, part, ms, ids,
                       scores, lse);
  // (4 | 16 waves: 1 x 670,091, k = 64, 55 | 27 us, 16 x 205,443, k = 32, 18.4 | 14.8; from 256 rows on, where
  // the rows fill the GPU, 43.2 | 44.0)
  if (parts > 1 && parts * k > 512 && rows <= 256)
    hipLaunchKernelGGL(k_rank_join<16>, dim3(rows), dim3(1024), 0, st, parts, k, part, ms, ids, scores, lse);
  else if (parts > 1)
    hipLaunchKernelGGL(k_rank_join<4>, dim3(rows), dim3(256), 0, st, parts, k, part, ms, ids, scores, lse);
  return hipGetLastError();
}

hipError_t launch_rank(int dtype, const void* z, int64_t ld, int rows, int L, const RankRules& ru, int k,
                       const RankShape& sh, int32_t* ids, float* scores, float* lse, void* ws, hipStream_t st) {
  if (dtype == 0) return rank_as<float>(z, ld, rows, L, ru, k, sh, ids, scores, lse, ws, st);
  if (dtype == 1) return rank_as<bf16>(z, ld, rows, L, ru, k, sh, ids, scores, lse, ws, st);
  return rank_as<f16>(z, ld, rows, L, ru, k, sh, ids, scores, lse, ws, st);
}

}  // namespace asgd

// The label loss over rows of at most 128 columns of 16 bits: a tile of labels then needs no loop over k, and
// what bounds the general kernels (k_label_loss.hip) is what surrounds it: an epilogue per two steps of k,
// and dz, which is larger than the label matrix itself at such widths, written to memory and read twice.
//
//   k_narrow_lse   256 rows in registers (a wave has 64), labels pass by in tiles of 64 through LDS; maximum and
//                  sum of exponentials per lane until the end
//   k_narrow_side  more rows: one kernel for dh and one for dw and db, each of which forms dz again
//   k_narrow_grad  up to 256 rows.  Per tile of 64 labels: z, dz in registers; dz W onto the rows' gradient, which stays in
//                  registers (dz is fed to the matrix cores as the accumulators hold it, the tile of W read with the k order
//                  that this gives); dz through LDS, turned around, times h: the tile's rows of dw
//
// 256 rows, 670,091 labels, width 128 in bf16, loss and gradients: 245 to 260 us; the general kernels took 638.  W is read
// twice and dw written once, 515 MB (101 us at a copy's rate); four products of 44 GFLOP.
//
// LDS rows of W and h are 256 bytes; chunk c (16 bytes) of row r lies at place c ^ (4 (r % 4) + r / 4 % 4), which makes both
// row reads (16 lanes of consecutive rows, the same c) and transposing reads (four rows, 64 bytes each) free of
// conflicts.  dz rows are 128 bytes (64 labels), in slots of 8: slot s of row r at s ^ (8 (r / 2 % 2) + r / 4 % 8), for
// transposing reads of four rows and writes of 32.
#include "label_loss_dev.h"

namespace asgd {

namespace {

typedef unsigned u32x2 __attribute__((ext_vector_type(2)));
typedef unsigned u32x4 __attribute__((ext_vector_type(4)));
typedef int i32x4u __attribute__((ext_vector_type(4), aligned(4)));
typedef unsigned u32x4u __attribute__((ext_vector_type(4), aligned(2)));
constexpr int NW_THREADS = 512, NW_ROWS = 256, NW_TILE = 64, NW_COLS = 128;
constexpr int NW_WBUF = NW_TILE * 256, NW_BIAS = 8 * 256;  // bytes of a tile; of its biases, a copy per wave

__device__ __forceinline__ int nw_turn(int r) { return 4 * (r & 3) + ((r >> 2) & 3); }

// The copies of tiles of W and their biases by a workgroup of THREADS.
template <int THREADS>
struct NwLoad {
  static constexpr int ITS = 1024 / THREADS, COPIES = ITS + 1;
  const char* base;
  int64_t ld, end;
  const float* bias;
  int n;
  unsigned voff[ITS];
  __device__ NwLoad(const TpOperand& w, const float* b, int n_labels, int d_bytes, int tid)
      : base(w.base), ld(w.ld), end(w.end), bias(b), n(n_labels) {
#pragma unroll
    for (int i = 0; i < ITS; ++i) {
      const int r = (tid >> 4) + THREADS / 16 * i, c = (tid & 15) ^ nw_turn(r);
      voff[i] = 16 * c < d_bytes ? (unsigned)(r * ld) + 16 * c : 0x80000000u;
    }
  }
  // tile t into LDS byte `to` (the buffer) and `to_bias` (this wave's copy)
  __device__ __forceinline__ void copy(int t, unsigned to, unsigned to_bias, int wave, int lane) const {
    const int64_t l0 = (int64_t)t * NW_TILE;
    const i32x4 rs = tp_rsrc(base + l0 * ld, end - l0 * ld);
#pragma unroll
    for (int i = 0; i < ITS; ++i) tp_copy16(rs, voff[i], to + 16 * THREADS * i + 1024 * wave);
    const i32x4 rb = tp_rsrc((const char*)(bias + (bias ? l0 : 0)), bias ? (n - l0) * 4 : 0);  // (zeros without)
    tp_copy4(rb, 4u * lane, to_bias);
  }
};

// Row r's chunk pair kk (32 bytes of k) of a tile in LDS.
template <typename T>
__device__ __forceinline__ typename TpMma<T>::frag8 nw_row_frag(const char* p, int r, int kk, int g) {
  return *reinterpret_cast<const typename TpMma<T>::frag8*>(p + 256 * r + 16 * ((2 * kk + g) ^ nw_turn(r)));
}
// Byte of a transposing read's source lane: row r (of this lane), columns 32 u + 16 (G % 2) + 4 a .. + 3.
__device__ __forceinline__ int nw_turned_at(int r, int u, int G, int a) {
  return 256 * r + 16 * ((4 * u + 2 * (G & 1) + (a >> 1)) ^ nw_turn(r)) + 8 * (a & 1);
}
template <typename T>
__device__ __forceinline__ typename TpMma<T>::frag8 nw_join(typename TpMma<T>::frag4 lo, typename TpMma<T>::frag4 hi) {
  return __builtin_shufflevector(lo, hi, 0, 1, 2, 3, 4, 5, 6, 7);
}

// A row of h as fragments (zeros past B and d).
template <typename T>
__device__ __forceinline__ void nw_rows(const TpOperand& h, int row, int B, int d_bytes, int g,
                                        typename TpMma<T>::frag8 (&f)[8]) {
#pragma unroll
  for (int kk = 0; kk < 8; ++kk) {
    f[kk] = typename TpMma<T>::frag8{};
    if (row < B && 32 * kk + 16 * g < d_bytes)
      f[kk] = *reinterpret_cast<const typename TpMma<T>::frag8*>(h.base + row * h.ld + 32 * kk + 16 * g);
  }
}

// z = bias for labels 32 b + 8 q + 4 g + i of a tile; then 32 bytes kk of k after the other.
__device__ __forceinline__ void nw_bias(const char* bias, int g, f32x16 (&z)[2]) {
#pragma unroll
  for (int b = 0; b < 2; ++b)
#pragma unroll
    for (int q = 0; q < 4; ++q) {
      const f32x4 t = *reinterpret_cast<const f32x4*>(bias + 4 * (32 * b + 8 * q + 4 * g));
#pragma unroll
      for (int i = 0; i < 4; ++i) z[b][4 * q + i] = t[i];
    }
}
template <typename T>
__device__ __forceinline__ void nw_logits(const char* w, const typename TpMma<T>::frag8 (&hf)[8], int lane, f32x16 (&z)[2]) {
  const int n = lane & 31, g = lane >> 5;
  // (what a product reads from LDS is on its way while the ones before run)
  typename TpMma<T>::frag8 f[3][2];
  auto read = [&](int kk) {
#pragma unroll
    for (int b = 0; b < 2; ++b) f[kk % 3][b] = nw_row_frag<T>(w, 32 * b + n, kk, g);
  };
  read(0);
  read(1);
#pragma unroll
  for (int kk = 0; kk < 8; ++kk) {
    if (kk + 2 < 8) read(kk + 2);
    __builtin_amdgcn_sched_barrier(0);
#pragma unroll
    for (int b = 0; b < 2; ++b) z[b] = tp_mma(f[kk % 3][b], hf[kk], z[b]);
    __builtin_amdgcn_sched_barrier(0);
  }
}

}  // namespace

// ---- log-sum-exp ---------------------------------------------------------------------------------
// Workgroup = (256 rows, a range of tiles); the row blocks of a range follow each other on one XCD, whose L2 then has its
// labels (and all 8 XCDs have work where there are fewer ranges: 65,536 rows, 5,000 labels 441 us on one, 202 on
// all).
// Four waves with 64 rows each: what a wave reads of a tile serves two products.  Two workgroups share a compute unit, so
// that one's exponentials meet the other's products.  Bound by issue: per tile and wave 32 products and 64 exponentials a
// lane with their sums and maxima, of which a part overlaps.  256 rows against 670,091 labels: 65 us (62 with a power of two
// as the base, one operation less for each exponential, which masks of large values do not allow; eight waves with 32 rows
// each 6 more).
constexpr int NWF_THREADS = 256, NWF_BUFS = 2;
constexpr int NWF_LDS = NWF_BUFS * (NW_WBUF + 4 * 256);

template <typename T>
__global__ __launch_bounds__(NWF_THREADS, 2) void k_narrow_lse(TpOperand h, TpOperand w, const float* bias, int B, int L,
                                                           int d_bytes, int row_blocks, int ranges, int per, int tiles,
                                                           float2* __restrict__ part) {
  extern __shared__ __attribute__((aligned(16))) char smem[];
  constexpr int BUF = NW_WBUF + 4 * 256;
  const int tid = threadIdx.x, lane = tid & 63, g = lane >> 5, n = lane & 31;
  const int wave = __builtin_amdgcn_readfirstlane(tid >> 6);
  const int all = ranges * row_blocks, share = (all + 7) >> 3, at = (int)(blockIdx.x & 7) * share + (int)(blockIdx.x >> 3);
  if (at >= all || (int)(blockIdx.x >> 3) >= share) return;
  const int range = at / row_blocks, row = at % row_blocks * NW_ROWS + 64 * wave + n;
  const int t0 = range * per, t1 = min(tiles, t0 + per);
  const NwLoad<NWF_THREADS> load(w, bias, L, d_bytes, tid);
  const unsigned lds0 = __builtin_amdgcn_readfirstlane((unsigned)(uintptr_t)(__attribute__((address_space(3))) char*)smem);
  auto issue = [&](int t) {
    const unsigned at = lds0 + (unsigned)((t - t0) % NWF_BUFS) * BUF;
    load.copy(t, at, at + NW_WBUF + 256 * wave, wave, lane);
  };
  typename TpMma<T>::frag8 hf[2][8];
  nw_rows<T>(h, row, B, d_bytes, g, hf[0]);
  nw_rows<T>(h, row + 32, B, d_bytes, g, hf[1]);
#pragma unroll
  for (int k = 0; k < NWF_BUFS - 1; ++k)
    if (t0 + k < t1) issue(t0 + k);
  float m[2] = {-INFINITY, -INFINITY}, s[2] = {0.0f, 0.0f};
  for (int t = t0; t < t1; ++t) {
    if (t + NWF_BUFS - 2 < t1) tp_wait<(NWF_BUFS - 2) * NwLoad<NWF_THREADS>::COPIES>();
    else tp_wait<0>();
    __builtin_amdgcn_s_barrier();  // the tile is here, and nobody reads the one before
    if (t + NWF_BUFS - 1 < t1) issue(t + NWF_BUFS - 1);
    const char* p = smem + (t - t0) % NWF_BUFS * BUF;
    f32x16 z[2][2];
    nw_bias(p + NW_WBUF + 256 * wave, g, z[0]);
    z[1][0] = z[0][0];
    z[1][1] = z[0][1];
#pragma unroll
    for (int kk = 0; kk < 8; ++kk)
#pragma unroll
      for (int b = 0; b < 2; ++b) {
        const auto f = nw_row_frag<T>(p, 32 * b + n, kk, g);
        z[0][b] = tp_mma(f, hf[0][kk], z[0][b]);
        z[1][b] = tp_mma(f, hf[1][kk], z[1][b]);
      }
    const bool edge = (t + 1) * NW_TILE > L;
#pragma unroll
    for (int i = 0; i < 2; ++i) {
      if (edge) {
#pragma unroll
        for (int b = 0; b < 2; ++b)
#pragma unroll
          for (int r = 0; r < 16; ++r)
            if (t * NW_TILE + 32 * b + 8 * (r >> 2) + 4 * g + (r & 3) >= L) z[i][b][r] = -INFINITY;
      }
      float top[2] = {m[i], m[i]};
#pragma unroll
      for (int b = 0; b < 2; ++b)
#pragma unroll
        for (int r = 0; r < 16; ++r) top[b] = fmaxf(top[b], z[i][b][r]);
      const float mm = fmaxf(top[0], top[1]);
      // Relative to the maximum, which is taken off first: masks may be of any size (the lowest value times log2 e is
      // -infinity, and from 10^10 on that product rounds by more than an exponent holds).
      const float base = mm == -INFINITY ? 0.0f : mm;
      float e[4] = {s[i] * exp_fast(m[i] - base), 0.0f, 0.0f, 0.0f};
#pragma unroll
      for (int b = 0; b < 2; ++b)
#pragma unroll
        for (int r = 0; r < 16; ++r) e[r & 3] += exp_fast(z[i][b][r] - base);
      s[i] = (e[0] + e[1]) + (e[2] + e[3]);
      m[i] = mm;
    }
  }
#pragma unroll
  for (int i = 0; i < 2; ++i) {
    const float m2 = __builtin_bit_cast(float, lane_xor<32>(__builtin_bit_cast(unsigned, m[i]), lane));
    const float s2 = __builtin_bit_cast(float, lane_xor<32>(__builtin_bit_cast(unsigned, s[i]), lane));
    const float mm = fmaxf(m[i], m2), base = mm == -INFINITY ? 0.0f : mm;
    if (row + 32 * i < B && g == 0)
      part[(int64_t)(row + 32 * i) * ranges + range] =
          make_float2(mm, s[i] * exp_fast(m[i] - base) + s2 * exp_fast(m2 - base));
  }
}

// ---- gradients ---------------------------------------------------------------------------------------
// Workgroup = a range of tiles with all the rows; one per compute unit (h, two tiles of W and dz fill its LDS).  Eight waves
// own 32 rows each for z, dz and dh, and one of the eight 32 x 32 blocks of dw.  256 rows, 670,091 labels: 170 to 185 us.
// Bound by latency: two barriers per tile, and what stands between them (LDS reads, dz's arithmetic, products) waits for
// each other in a wave while its SIMD has one more.  Four waves of 64 rows in 512 registers took 320 us, dz's exponentials
// between the products of dh 790 (spills).  All 256 registers of a lane are taken; two or four more, which rows whose targets
// do not fit the list need, lie in scratch.  Where dw has the operands' type it leaves in 16-byte stores.
constexpr int NWG_BUFS = 2, NWG_HITS = 1023;
constexpr int NWG_H = 0, NWG_DZ = NWG_H + NW_ROWS * 256, NWG_W = NWG_DZ + NW_ROWS * 128;
constexpr int NWG_HIT = NWG_W + NWG_BUFS * (NW_WBUF + NW_BIAS), NWG_SUM = NWG_HIT + 4 * (NWG_HITS + 1);
constexpr int NWG_LDS = NWG_SUM + 8 * NW_TILE * 4;
static_assert(NWG_LDS <= 160 * 1024, "LDS of a compute unit");

// LDS byte of labels 4 s .. + 3 of row r in the tile of dz.
__device__ __forceinline__ int nw_dz(int r, int s) { return 128 * r + 8 * (s ^ (8 * ((r >> 1) & 1) + ((r >> 2) & 7))); }

// v[k] summed over the 32 lanes of each half; lane i keeps label (k index) i.  Halves of the values change sides at every step.
__device__ __forceinline__ float nw_sum_lanes(float (&v)[32], int lane) {
#pragma unroll
  for (int k = 0; k < 16; ++k) {
    const auto s = __builtin_amdgcn_permlane16_swap(__builtin_bit_cast(unsigned, v[k]), __builtin_bit_cast(unsigned, v[k + 16]),
                                                    false, false);
    v[k] = __builtin_bit_cast(float, (unsigned)s[0]) + __builtin_bit_cast(float, (unsigned)s[1]);
  }
  auto halve = [&](int half, bool up, auto other) {
#pragma unroll
    for (int k = 0; k < half; ++k) {
      const float keep = up ? v[k + half] : v[k], give = up ? v[k] : v[k + half];
      v[k] = keep + __builtin_bit_cast(float, other(__builtin_bit_cast(unsigned, give)));
    }
  };
  halve(8, lane & 8, [&](unsigned x) { return lane_xor<8>(x, lane); });
  halve(4, lane & 4, [&](unsigned x) { return lane_xor<4>(x, lane); });
  halve(2, lane & 2, [&](unsigned x) { return lane_xor<2>(x, lane); });
  halve(1, lane & 1, [&](unsigned x) { return lane_xor<1>(x, lane); });
  return v[0];
}

// Columns col .. + 31 of a label's row of dw in two 16-byte stores: lanes n and n + 32 hold columns 8 q .. + 3 and + 4 .. + 7,
// and with a change of sides between q and q + 1 each has 8.
template <typename T>
__device__ __forceinline__ void nw_store32(const MatDev& dw, int label, int col, int g, const f32x16& acc, float out, bool in) {
  typedef typename TpMma<T>::frag4 Half;
#pragma unroll
  for (int q = 0; q < 4; q += 2) {
    u32x2 v[2];
#pragma unroll
    for (int i = 0; i < 2; ++i) {
      Half o;
#pragma unroll
      for (int k = 0; k < 4; ++k) o[k] = (T)(acc[4 * (q + i) + k] * out);
      v[i] = __builtin_bit_cast(u32x2, o);
    }
    const auto lo = __builtin_amdgcn_permlane32_swap(v[0][0], v[1][0], false, false);
    const auto hi = __builtin_amdgcn_permlane32_swap(v[0][1], v[1][1], false, false);
    const u32x4 o{(unsigned)lo[0], (unsigned)hi[0], (unsigned)lo[1], (unsigned)hi[1]};
    if (in) *reinterpret_cast<u32x4u*>((T*)dw.data + label * dw.ld + col + 8 * (q + g)) = o;
  }
}

template <typename T>
__global__ __launch_bounds__(NW_THREADS) void k_narrow_grad(TpOperand h, TpOperand w, DzArgs a, int B, int d, int ranges,
                                                           int per, int tiles, float alpha, MatDev dw, float* __restrict__ db,
                                                           float* __restrict__ slabs) {
  typedef typename TpMma<T>::frag8 Frag;
  typedef typename TpMma<T>::frag4 Half;
  extern __shared__ __attribute__((aligned(16))) char smem[];
  const int tid = threadIdx.x, lane = tid & 63, g = lane >> 5, n = lane & 31;
  const int wave = __builtin_amdgcn_readfirstlane(tid >> 6);
  const int G = lane >> 4, ti = (lane >> 2) & 3, ta = lane & 3;  // of a transposing read's address
  const int range = blockIdx.x, L = a.n_labels, d_bytes = d * 2;
  const int t0 = range * per, t1 = min(tiles, t0 + per);
  const NwLoad<NW_THREADS> load(w, a.bias, L, d_bytes, tid);
  const unsigned lds0 = __builtin_amdgcn_readfirstlane((unsigned)(uintptr_t)(__attribute__((address_space(3))) char*)smem);
  auto issue = [&](int t) {
    const unsigned at = lds0 + NWG_W + (unsigned)((t - t0) % NWG_BUFS) * (NW_WBUF + NW_BIAS);
    load.copy(t, at, at + NW_WBUF + 256 * wave, wave, lane);
  };
  // the rows: all of them in LDS, a wave's own in registers too
  {
    const i32x4 rs = tp_rsrc(h.base, h.end);
#pragma unroll
    for (int i = 0; i < 8; ++i) {
      const int r = (tid >> 4) + 32 * i, c = (tid & 15) ^ nw_turn(r);
      tp_copy16(rs, 16 * c < d_bytes && r < B ? (unsigned)(r * h.ld) + 16 * c : 0x80000000u, lds0 + NWG_H + 8192 * i + 1024 * wave);
    }
  }
  if (t0 < t1) issue(t0);
  const int row = 32 * wave + n;
  Frag hf[8];
  nw_rows<T>(h, row, B, d_bytes, g, hf);
  const float scale = *a.scale;
  float sh = 0.0f, top = 0.0f, f = 0.0f, fp = 0.0f;
  if (row < B) {
    sh = a.share[row];
    top = a.top[row];
    f = (a.weights ? scale > 0.0f ? a.weights[row] / scale : a.weights[row] : 1.0f) * a.up;
    fp = f * a.inv[row];
  }
  const bool live = sh > 0.0f;
  const float out = alpha * scale, fs = f * sh;
  // targets among this workgroup's labels, listed once (more than the list holds: every tile goes through the rows' lists, which
  // takes 256 rows x 670,091 labels of 75 targets a row from 304 us to 530 where all are among 2,000 labels; general kernels 638)
  int* const hits = reinterpret_cast<int*>(smem + NWG_HIT);
  if (tid == 0) hits[0] = 0;
  asm volatile("s_waitcnt lgkmcnt(0)" ::: "memory");
  __builtin_amdgcn_s_barrier();
  const int l0 = t0 * NW_TILE, l1 = min(L, t1 * NW_TILE);
  if ((tid >> 1) < B && a.y.indptr) {
    each_label(a.y, tid >> 1, tid & 1, 2, [&](int id) {
      if (id >= l0 && id < l1) {
        const int at = atomicAdd(hits, 1);
        if (at < NWG_HITS) hits[1 + at] = (tid >> 1) << 23 | (id - l0);
      }
    });
  }
  f32x16 dh[4];
#pragma unroll
  for (int u = 0; u < 4; ++u)
#pragma unroll
    for (int r = 0; r < 16; ++r) dh[u][r] = 0.0f;
  char* const dzt = smem + NWG_DZ;
  // addresses of the transposing reads: rows that differ by multiples of 16 differ by a constant
  int wat[2][4], hat[2], zat[2][2];
  const int lb = wave >> 2, wu = wave & 3;  // this wave's block of dw: labels 32 lb .., columns 32 wu ..
#pragma unroll
  for (int hi = 0; hi < 2; ++hi) {
#pragma unroll
    for (int u = 0; u < 4; ++u) wat[hi][u] = nw_turned_at(8 * hi + 4 * (G >> 1) + ti, u, G, ta);
    hat[hi] = nw_turned_at(8 * (G >> 1) + 4 * hi + ti, wu, G, ta);
#pragma unroll
    for (int c = 0; c < 2; ++c) zat[hi][c] = nw_dz(16 * c + 8 * (G >> 1) + 4 * hi + ti, 8 * lb + 4 * (G & 1) + ta);
  }
  // whole 16-byte pieces of dw in the operands' type
  const bool wide = dw.data && dw.dtype == (std::is_same<T, bf16>::value ? 1 : 2) && 32 * wu + 32 <= d;
  float* const sums = reinterpret_cast<float*>(smem + NWG_SUM);

  tp_wait<0>();
  for (int t = t0; t < t1; ++t) {
    // (the wait for this tile's copies stands before the last tile's stores of dw)
    asm volatile("s_waitcnt lgkmcnt(0)" ::: "memory");
    __builtin_amdgcn_s_barrier();  // the tile is here, and nobody reads dz or the other tile any more
    if (t + 1 < t1) issue(t + 1);
    const char* p = smem + NWG_W + (t - t0) % NWG_BUFS * (NW_WBUF + NW_BIAS);
    // how often this tile's labels stand in the wave's rows: 16-bit counts where dz will lie
    const int total = hits[0], c0 = (t - t0) * NW_TILE;
    bool any = total > NWG_HITS;
    if (total && !any) {
      bool mine = false;
      for (int k = lane; k < total; k += 64) {
        const int hit = hits[1 + k], c = (hit & 0x7fffff) - c0;
        mine |= (int)((unsigned)hit >> 28) == wave && c >= 0 && c < NW_TILE;
      }
      any = __ballot(mine) != 0;
    }
    if (any) {
      auto add = [&](int r, int c) {  // row of the wave, label of the tile
        const int at = nw_dz(32 * wave + r, c >> 2) + 2 * (c & 3);
        atomicAdd(reinterpret_cast<unsigned*>(dzt + (at & ~3)), at & 2 ? 0x10000u : 1u);
      };
#pragma unroll
      for (int k = 0; k < 8; ++k) *reinterpret_cast<uint64_t*>(dzt + 4096 * wave + 512 * k + 8 * lane) = 0;
      __builtin_amdgcn_fence(__ATOMIC_SEQ_CST, "wavefront");
      if (total <= NWG_HITS) {
        for (int k = lane; k < total; k += 64) {
          const int hit = hits[1 + k], c = (hit & 0x7fffff) - c0;
          if ((int)((unsigned)hit >> 28) == wave && c >= 0 && c < NW_TILE) add(((unsigned)hit >> 23) & 31, c);
        }
      } else if (32 * wave + (lane >> 1) < B) {
        each_label(a.y, 32 * wave + (lane >> 1), lane & 1, 2, [&](int id) {
          const int c = id - t * NW_TILE;
          if (c >= 0 && c < NW_TILE && id < L) add(lane >> 1, c);
        });
      }
      __builtin_amdgcn_fence(__ATOMIC_SEQ_CST, "wavefront");
    }
    f32x16 z[2];
    nw_bias(p + NW_WBUF + 256 * wave, g, z);
    nw_logits<T>(p, hf, lane, z);
    const bool edge = (t + 1) * NW_TILE > L;
    Frag df[2][2];
    // dz, to LDS and as fragments; checked: with targets, or past the last label
    auto form = [&](auto checked) {
#pragma unroll
      for (int b = 0; b < 2; ++b)
#pragma unroll
        for (int q = 0; q < 4; ++q) {
          char* const at = dzt + nw_dz(row, 8 * b + 2 * q + g);
          Half o;
          uint64_t times = 0;
          if (checked) times = any ? *reinterpret_cast<const uint64_t*>(at) : 0;
#pragma unroll
          for (int k = 0; k < 4; ++k) {
            float v = z[b][4 * q + k];
            v = exp_fast(v - top) * fp;  // (a row's best label gets 1 / sum exactly, so one that is certain 1)
            bool in = live;  // (rows without labels and labels past the last are zeros, whatever they hold)
            if (checked) {
              v -= (float)((times >> (16 * k)) & 0xffff) * fs;
              in = live && t * NW_TILE + 32 * b + 8 * q + 4 * g + k < L;
            }
            v = in ? v : 0.0f;
            z[b][4 * q + k] = v;
            o[k] = (T)v;
            df[b][q >> 1][4 * (q & 1) + k] = o[k];
          }
          *reinterpret_cast<Half*>(at) = o;
        }
    };
    if (any || edge) form(std::true_type());
    else form(std::false_type());
    if (db) {
      float v[32];
#pragma unroll
      for (int k = 0; k < 32; ++k) v[k] = z[k >> 4][k & 15];
      // lane i of half g keeps accumulator register i: label 32 (i / 16) + 8 (i / 4 % 4) + 4 g + i % 4
      sums[wave * NW_TILE + 32 * (n >> 4) + 8 * ((n >> 2) & 3) + 4 * g + (n & 3)] = nw_sum_lanes(v, lane);
    }
    // dz W: k are the labels in the accumulators' order, 16 c + 8 hi + 4 g + 0..3 of a block
    Frag uf[4];
    auto w_read = [&](int k) {  // k = 8 b + 4 c + u
      const char* const q = p + 256 * (16 * (k >> 2));
      uf[k & 3] = nw_join<T>(tp_turned<T>(q + wat[0][k & 3]), tp_turned<T>(q + wat[1][k & 3]));
    };
#pragma unroll
    for (int k = 0; k < 3; ++k) w_read(k);
#pragma unroll
    for (int k = 0; k < 16; ++k) {
      if (k + 3 < 16) w_read(k + 3);
      __builtin_amdgcn_sched_barrier(0);
      dh[k & 3] = tp_mma(uf[k & 3], df[k >> 3][(k >> 2) & 1], dh[k & 3]);
      __builtin_amdgcn_sched_barrier(0);
    }
    asm volatile("s_waitcnt lgkmcnt(0)" ::: "memory");
    __builtin_amdgcn_s_barrier();  // dz of all rows is here
    if (db && tid < NW_TILE && t * NW_TILE + tid < L) {
      float v = 0.0f;
#pragma unroll
      for (int k = 0; k < 8; ++k) v += sums[k * NW_TILE + tid];
      db[t * NW_TILE + tid] = v * out;
    }
    f32x16 acc;
    if (dw.data) {
#pragma unroll
      for (int r = 0; r < 16; ++r) acc[r] = 0.0f;
      // (what a product reads from LDS is on its way while the one before runs)
      Frag hd[2], zd[2];
      auto read = [&](int c) {
        const char *zp = dzt + 4096 * (c >> 1), *hp = smem + NWG_H + 4096 * c;
        hd[c & 1] = nw_join<T>(tp_turned<T>(hp + hat[0]), tp_turned<T>(hp + hat[1]));
        zd[c & 1] = nw_join<T>(tp_turned<T>(zp + zat[0][c & 1]), tp_turned<T>(zp + zat[1][c & 1]));
      };
      read(0);
#pragma unroll
      for (int c = 0; c < NW_ROWS / 16; ++c) {
        if (c + 1 < NW_ROWS / 16) read(c + 1);
        __builtin_amdgcn_sched_barrier(0);
        acc = tp_mma(hd[c & 1], zd[c & 1], acc);
        __builtin_amdgcn_sched_barrier(0);
      }
    }
    // The next tile's copies, of which the whole of this tile's work lies behind, before any store: nothing then goes by
    // how many stores follow them, or by the order in which loads and stores end.
    tp_wait<0>();
    if (dw.data) {
      const int label = t * NW_TILE + 32 * lb + n;
      if (wide) {
        nw_store32<T>(dw, label, 32 * wu, g, acc, out, label < L);
      } else if (label < L) {
#pragma unroll
        for (int q = 0; q < 4; ++q) {
          const int col = 32 * wu + 8 * q + 4 * g;
          const float v[4] = {acc[4 * q] * out, acc[4 * q + 1] * out, acc[4 * q + 2] * out, acc[4 * q + 3] * out};
          store4(dw, label, col, d - col, v);
        }
      }
    }
  }
  if (slabs && row < B) {
    float* o = slabs + ((int64_t)range * B + row) * NW_COLS + 4 * g;
#pragma unroll
    for (int u = 0; u < 4; ++u)
#pragma unroll
      for (int q = 0; q < 4; ++q)
        *reinterpret_cast<f32x4*>(o + 32 * u + 8 * q) = f32x4{dh[u][4 * q], dh[u][4 * q + 1], dh[u][4 * q + 2], dh[u][4 * q + 3]};
  }
}

// ---- gradients of more rows ----------------------------------------------------------------------------
// One side of the product in registers, 32 per wave, with the sums of its gradient; the other passes by in tiles of 64
// through LDS.  Rows in registers give dh, labels dw and db: z is formed once more for each (and its exponentials), but dz
// leaves its registers for neither.  Four waves, two workgroups per compute unit, one barrier per tile.  406 rows, 225,682
// labels, width 128 in bf16: dh 70 to 76 us, dw and db 94 to 104 (the general kernels' dz, 183 MB written and read twice, and
// its products 245); the whole call 304 -> 198 to 215.  For up to 256 rows k_narrow_grad, which forms z once for both, is
// faster.
constexpr int NWS_THREADS = 256, NWS_OWN = 128, NWS_HITS = 2047;
constexpr int NWS_BUF = NW_WBUF + 4 * 256, NWS_COUNT = 2 * NWS_BUF, NWS_ROW = NWS_COUNT + NWS_OWN * 128;
constexpr int NWS_HIT = NWS_ROW + 4 * 3 * 256, NWS_SORT = NWS_HIT + 4 * (NWS_HITS + 1), NWS_START = NWS_SORT + 4 * (NWS_HITS + 1);
constexpr int NWS_AT = NWS_START + 4 * 260, NWS_LDS = NWS_AT + 4 * 256;
static_assert(2 * NWS_LDS <= 160 * 1024, "two workgroups per compute unit");

// What turns a logit of row i into dz: v = e^(z - top) fp - times fs.  A row without labels gets zeros from
// any finite logit; one that is not (its h is zeros, but w or the bias of a label may hold anything) is made one before.
struct NwRow {
  float top, fp, fs;
};
__device__ __forceinline__ NwRow nw_row(const DzArgs& a, float top, float inv, float share, float weight, float scale) {
  if (!(share > 0.0f)) return NwRow{INFINITY, 0.0f, 0.0f};
  const float f = (a.weights ? scale > 0.0f ? weight / scale : weight : 1.0f) * a.up;
  return NwRow{top, f * inv, f * share};
}

// ROWS: own = rows of h, 128 of them, and tiles t0 .. of labels; else own = labels, `per` blocks of 128 after each other,
// and all tiles of rows.
template <typename T, bool ROWS>
__global__ __launch_bounds__(NWS_THREADS, 2) void k_narrow_side(TpOperand own, TpOperand other, DzArgs a, int n_own, int n_other,
                                                                int d, int blocks, int ranges, int per, int tiles, float alpha,
                                                                MatDev dw, float* __restrict__ db, float* __restrict__ slabs) {
  typedef typename TpMma<T>::frag8 Frag;
  typedef typename TpMma<T>::frag4 Half;
  extern __shared__ __attribute__((aligned(16))) char smem[];
  const int tid = threadIdx.x, lane = tid & 63, g = lane >> 5, n = lane & 31;
  const int wave = __builtin_amdgcn_readfirstlane(tid >> 6);
  const int G = lane >> 4, ti = (lane >> 2) & 3, ta = lane & 3;  // of a transposing read's address
  const int all = ROWS ? ranges * blocks : ranges, share = (all + 7) >> 3;
  const int at = (int)(blockIdx.x & 7) * share + (int)(blockIdx.x >> 3);
  if (at >= all || (int)(blockIdx.x >> 3) >= share) return;
  const int range = ROWS ? at / blocks : at;
  const int b0 = ROWS ? at % blocks : range * per, b1 = ROWS ? b0 + 1 : min(blocks, b0 + per);
  const int t0 = ROWS ? range * per : 0, t1 = ROWS ? min(tiles, t0 + per) : tiles;
  const int d_bytes = 2 * d, B = ROWS ? n_own : n_other;
  const NwLoad<NWS_THREADS> load(other, ROWS ? a.bias : nullptr, n_other, d_bytes, tid);
  const unsigned lds0 = __builtin_amdgcn_readfirstlane((unsigned)(uintptr_t)(__attribute__((address_space(3))) char*)smem);
  const float scale = *a.scale, out = alpha * scale;
  auto issue = [&](int t, int buf) {
    const unsigned to = lds0 + (unsigned)buf * NWS_BUF;
    load.copy(t, to, to + NW_WBUF + 256 * wave, wave, lane);
  };
  // (tiles of rows) this wave's copy of what belongs to the tile's rows, a lane per row, loaded a tile ahead
  float* const rows = reinterpret_cast<float*>(smem + NWS_ROW + 768 * wave);  // [3][64]
  float r_top = 0.0f, r_inv = 0.0f, r_share = 0.0f, r_weight = 0.0f;
  auto fetch_row = [&](int t) {
    const int r = t * NW_TILE + lane;
    const bool in = r < B;
    r_top = in ? a.top[r] : 0.0f;
    r_inv = in ? a.inv[r] : 0.0f;
    r_share = in ? a.share[r] : 0.0f;
    r_weight = in && a.weights ? a.weights[r] : 0.0f;
  };
  issue(t0, 0);
  if (!ROWS) fetch_row(t0);
  // Targets between own (first .. last of them) and tiles wa .. wb of what passes by, listed: own within the list's, other;
  // then in the order of the tiles (or of up to 256 groups of them), so that a tile looks at its own alone.  Returns how many
  // there are; more than NWS_HITS are not listed (nor all counted: then about how many).
  unsigned* const hits = reinterpret_cast<unsigned*>(smem + NWS_HIT);
  unsigned* const sorted = reinterpret_cast<unsigned*>(smem + NWS_SORT);
  int* const start = reinterpret_cast<int*>(smem + NWS_START);  // [257]
  int* const next = reinterpret_cast<int*>(smem + NWS_AT);
  constexpr int SHIFT = ROWS ? 24 : 18;
  int group = 0;  // tiles of one: 2^group
  auto list = [&](int first, int last, int wa, int wb) {
    __syncthreads();  // (nobody looks at the list before any more)
    for (group = 0; (wb - wa) >> group > 255;) ++group;
    start[tid] = 0;
    if (tid == 0) hits[0] = start[256] = 0;
    __syncthreads();
    int n_ids = 0;
    if constexpr (ROWS) {
      const int l0 = wa * NW_TILE, l1 = min(n_other, wb * NW_TILE);
      if (first + (tid >> 1) < last && a.y.indptr)
        each_label(a.y, first + (tid >> 1), tid & 1, 2, [&](int id) {
          if (id >= l0 && id < l1) {
            const unsigned k = atomicAdd(hits, 1u);
            if (k < NWS_HITS) hits[1 + k] = (unsigned)(tid >> 1) << SHIFT | (unsigned)id;
          }
        });
    } else if (a.y.indptr) {
      // the rows' lists as one: entries whose label is here, then their rows by bisection
      const int r0 = wa * NW_TILE, r1 = min(B, wb * NW_TILE);
      const int64_t begin = *a.y.first, end = begin + a.y.nnz;
      const int64_t q0 = min(max((int64_t)a.y.indptr[r0], begin), end), q1 = min(max((int64_t)a.y.indptr[r1], q0), end);
      const int32_t* const ids = a.y.indices + q0;
      n_ids = (int)(q1 - q0);
      auto take = [&](unsigned found, auto place) {  // bits: which of a thread's entries
        if (!found) return;
        for (unsigned h = atomicAdd(hits, (unsigned)__popc(found)); found && h < NWS_HITS; ++h, found &= found - 1)
          hits[1 + h] = (unsigned)place(__ffs(found) - 1);
      };
      const int whole = n_ids & ~(16 * NWS_THREADS - 1);  // (16 ids a thread on their way at once)
      int seen = 0;  // a list that is full already is not needed whole
      for (; seen < whole && __hip_atomic_load(hits, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_WORKGROUP) <= NWS_HITS;
           seen += 16 * NWS_THREADS) {
        const int q = seen + 4 * tid;
        i32x4 id[4];
#pragma unroll
        for (int k = 0; k < 4; ++k) id[k] = *reinterpret_cast<const i32x4u*>(ids + q + 4 * NWS_THREADS * k);
        unsigned found = 0;
#pragma unroll
        for (int k = 0; k < 16; ++k) found |= (unsigned)(id[k >> 2][k & 3] >= first && id[k >> 2][k & 3] < last) << k;
        take(found, [&](int k) { return q + 4 * NWS_THREADS * (k >> 2) + (k & 3); });
      }
      if (seen == whole) {
        for (int q = whole + tid; q < n_ids; q += 8 * NWS_THREADS) {
          int id[8];
          unsigned found = 0;
#pragma unroll
          for (int k = 0; k < 8; ++k) id[k] = q + k * NWS_THREADS < n_ids ? ids[q + k * NWS_THREADS] : -1;
#pragma unroll
          for (int k = 0; k < 8; ++k) found |= (unsigned)(id[k] >= first && id[k] < last) << k;
          take(found, [&](int k) { return q + k * NWS_THREADS; });
        }
        seen = n_ids;
      }
      if (tid == 0) next[0] = seen;
      // (of every row or every 2^skip-th where it begins, in LDS: from memory a step takes as long as a tile's products)
      int skip = 0;
      while ((r1 - r0 - 1) >> skip > NWS_HITS) ++skip;
      const int known = ((r1 - r0 - 1) >> skip) + 1;
      for (int i = tid; i < known; i += NWS_THREADS) sorted[i] = (unsigned)a.y.indptr[r0 + (i << skip)];
      __syncthreads();
      const int held = hits[0] <= NWS_HITS ? (int)hits[0] : 0;
      for (int h = tid; h < held; h += NWS_THREADS) {
        const int64_t q = q0 + hits[1 + h];
        int lo = 0, hi = known;  // the last row that does not begin behind q
        while (hi - lo > 1) {
          const int mid = (lo + hi) >> 1;
          if ((int)sorted[mid] <= q) lo = mid;
          else hi = mid;
        }
        lo = r0 + (lo << skip);
        hi = min(r1, lo + (1 << skip));
        while (hi - lo > 1) {
          const int mid = (lo + hi) >> 1;
          if (a.y.indptr[mid] <= q) lo = mid;
          else hi = mid;
        }
        int s0, s1;
        label_range(a.y, lo, &s0, &s1);
        hits[1 + h] = q >= s0 && q < s1 ? (unsigned)(a.y.indices[q] - first) << SHIFT | (unsigned)lo : ~0u;
      }
    }
    __syncthreads();
    const int total = (int)hits[0];
    if (total > NWS_HITS) return ROWS ? total : (int)((int64_t)total * n_ids / max(next[0], min(n_ids, 16 * NWS_THREADS)));
    if (total == 0) return 0;
    auto group_of = [&](unsigned hit) { return (int)((((hit & ((1u << SHIFT) - 1)) >> 6) - wa) >> group); };
    for (int h = tid; h < total; h += NWS_THREADS)
      if (hits[1 + h] != ~0u) atomicAdd(start + 1 + group_of(hits[1 + h]), 1);
    __syncthreads();
    for (int o = 1; o < 256; o <<= 1) {
      const int v = tid >= o ? start[1 + tid - o] : 0;
      __syncthreads();
      start[1 + tid] += v;
      __syncthreads();
    }
    next[tid] = start[tid];
    __syncthreads();
    for (int h = tid; h < total; h += NWS_THREADS)
      if (hits[1 + h] != ~0u) sorted[atomicAdd(next + group_of(hits[1 + h]), 1)] = hits[1 + h];
    __syncthreads();
    return total;
  };
  // One list for all of it where it fits; else one for each block of own; else as many as it takes, of as many tiles as
  // should fit if targets were spread evenly, or fewer.  (A tile that has too many by itself looks through its rows' lists.)
  const int own0 = b0 * NWS_OWN, own1 = min(n_own, b1 * NWS_OWN);
  int list0 = own0, list_n = own1 - own0, total = 0, wa = t0, wb = t0;  // the list's own, its tiles
  char* const counts = smem + NWS_COUNT;
  // LDS addresses, of which the parts of kk, u, hi, b and q flip bits: formed where they are used (as loop invariants they
  // would take the registers that the sums need)
  int row_at = 256 * n + 16 * (g ^ nw_turn(n)), turned_at = nw_turned_at(4 * (G >> 1) + ti, 0, G, ta);
  int count_at = nw_dz(32 * wave + n, g);
  int buf = 0;
  for (int blk = b0; blk < b1; ++blk) {
    const int me = blk * NWS_OWN + 32 * wave + n;
    Frag of[8];
    nw_rows<T>(own, me, n_own, d_bytes, g, of);
    const float own_bias = !ROWS && a.bias && me < n_own ? a.bias[me] : 0.0f;
    NwRow mine{INFINITY, 0.0f, 0.0f};
    if (ROWS && me < B) mine = nw_row(a, a.top[me], a.inv[me], a.share[me], a.weights ? a.weights[me] : 0.0f, scale);
    f32x16 acc[4];
#pragma unroll
    for (int u = 0; u < 4; ++u)
#pragma unroll
      for (int r = 0; r < 16; ++r) acc[u][r] = 0.0f;
    float sums = 0.0f;
    bool odd = false;  // some label of the wave holds a value that is not finite (0 times the others sum to 0)
    if constexpr (!ROWS) {
      float zero = own_bias * 0.0f;
#pragma unroll
      for (int kk = 0; kk < 8; ++kk)
#pragma unroll
        for (int i = 0; i < 8; ++i) zero = fmaf((float)of[kk][i], 0.0f, zero);
      odd = __ballot(!(zero == 0.0f)) != 0;
    }
    if (list_n <= NWS_OWN) {  // a list of each block's own
      list0 = blk * NWS_OWN;
      list_n = min(NWS_OWN, n_own - list0);
      if (blk > b0) wb = t0;
    }
    for (int t = t0; t < t1;) {
      if (t == wb) {
        wa = t;
        for (wb = t1;;) {
          total = list(list0, list0 + list_n, wa, wb);
          if (total <= NWS_HITS) break;
          if (list_n > NWS_OWN) {
            list0 = blk * NWS_OWN;
            list_n = NWS_OWN;
            continue;
          }
          if (wb - wa == 1) break;
          const int fit = (int)((int64_t)(wb - wa) * (NWS_HITS * 3 / 4) / total);
          wb = wa + (fit > 1 ? fit : 1);
        }
      }
      for (; t < wb; ++t) {
        tp_wait<0>();
        __builtin_amdgcn_s_barrier();  // the tile is here, and nobody reads the one before
        asm volatile("" : "+v"(row_at), "+v"(turned_at), "+v"(count_at));
        const char* const p = smem + buf * NWS_BUF;
        buf ^= 1;
        if (t + 1 < t1) issue(t + 1, buf);
        else if (blk + 1 < b1) issue(t0, buf);
        bool masked = false;  // labels past the last
        if constexpr (ROWS) {
          masked = (t + 1) * NW_TILE > n_other;
        } else {
          const NwRow r = nw_row(a, r_top, r_inv, r_share, r_weight, scale);
          rows[lane] = r.top;
          rows[64 + lane] = r.fp;
          rows[128 + lane] = r.fs;
          fetch_row(t + 1 < t1 ? t + 1 : t0);
        }
        // how often a label stands in a row's list: 16-bit counts per own
        bool any = total > NWS_HITS;
        const int first = t * NW_TILE, from = blk * NWS_OWN - list0 + 32 * wave;
        auto place = [&](unsigned hit, int* o, int* c) {
          *o = (int)(hit >> SHIFT) - from;
          *c = (int)(hit & ((1u << SHIFT) - 1)) - first;
          return *o >= 0 && *o < 32 && *c >= 0 && *c < NW_TILE;
        };
        int h0 = 0, h1 = 0;
        if (total && !any) {
          h0 = start[(t - wa) >> group];
          h1 = start[((t - wa) >> group) + 1];
          bool here = false;
          int o, c;
          for (int k = h0 + lane; k < h1; k += 64) here |= place(sorted[k], &o, &c);
          any = __ballot(here) != 0;
        }
        if (any) {
          auto add = [&](int o, int c) {
            const int to = nw_dz(32 * wave + o, c >> 2) + 2 * (c & 3);
            atomicAdd(reinterpret_cast<unsigned*>(counts + (to & ~3)), to & 2 ? 0x10000u : 1u);
          };
#pragma unroll
          for (int k = 0; k < 8; ++k) *reinterpret_cast<uint64_t*>(counts + 4096 * wave + 512 * k + 8 * lane) = 0;
          __builtin_amdgcn_fence(__ATOMIC_SEQ_CST, "wavefront");
          if (total <= NWS_HITS) {
            int o, c;
            for (int k = h0 + lane; k < h1; k += 64)
              if (place(sorted[k], &o, &c)) add(o, c);
          } else if constexpr (ROWS) {
            if (own0 + 32 * wave + (lane >> 1) < B)
              each_label(a.y, own0 + 32 * wave + (lane >> 1), lane & 1, 2, [&](int id) {
                const int c = id - first;
                if (c >= 0 && c < NW_TILE && id < n_other) add(lane >> 1, c);
              });
          } else if (first + lane < B) {
            each_label(a.y, first + lane, 0, 1, [&](int id) {
              const int o = id - list0 - from;
              if (o >= 0 && o < 32 && id < n_own) add(o, lane);
            });
          }
        }
        __builtin_amdgcn_fence(__ATOMIC_SEQ_CST, "wavefront");
        f32x16 z[2];
        if constexpr (ROWS) {
          nw_bias(p + NW_WBUF + 256 * wave, g, z);
        } else {
#pragma unroll
          for (int r = 0; r < 16; ++r) z[0][r] = z[1][r] = own_bias;
        }
        Frag f[2][2];
        auto read = [&](int kk) {
#pragma unroll
          for (int b = 0; b < 2; ++b) f[kk & 1][b] = *reinterpret_cast<const Frag*>(p + (row_at ^ (32 * kk)) + 8192 * b);
        };
        read(0);
#pragma unroll
        for (int kk = 0; kk < 8; ++kk) {
          if (kk + 1 < 8) read(kk + 1);
          __builtin_amdgcn_sched_barrier(0);
#pragma unroll
          for (int b = 0; b < 2; ++b) z[b] = tp_mma(f[kk & 1][b], of[kk], z[b]);
          __builtin_amdgcn_sched_barrier(0);
        }
        if constexpr (!ROWS) {
          if (odd) {  // (in dh such rows are made zeros when the slabs are joined)
#pragma unroll
            for (int b = 0; b < 2; ++b)
#pragma unroll
              for (int q = 0; q < 4; ++q) {
                const f32x4 top = *reinterpret_cast<const f32x4*>(rows + 32 * b + 8 * q + 4 * g);
#pragma unroll
                for (int k = 0; k < 4; ++k) z[b][4 * q + k] = top[k] == INFINITY ? 0.0f : z[b][4 * q + k];
              }
          }
        }
        Frag df[2][2];
        float part[4] = {};  // (one sum over thousands of rows would round as often)
        auto form = [&](auto checked) {
#pragma unroll
          for (int b = 0; b < 2; ++b)
#pragma unroll
            for (int q = 0; q < 4; ++q) {
              const int c = 32 * b + 8 * q + 4 * g;
              f32x4 top, fp, fs;
              if constexpr (!ROWS) {
                top = *reinterpret_cast<const f32x4*>(rows + c);
                fp = *reinterpret_cast<const f32x4*>(rows + 64 + c);
                if (checked) fs = *reinterpret_cast<const f32x4*>(rows + 128 + c);
              }
              uint64_t times = 0;
              if (checked) times = any ? *reinterpret_cast<const uint64_t*>(counts + (count_at ^ (64 * b) ^ (16 * q))) : 0;
#pragma unroll
              for (int k = 0; k < 4; ++k) {
                float v = exp_fast(z[b][4 * q + k] - (ROWS ? mine.top : top[k])) * (ROWS ? mine.fp : fp[k]);
                if (checked) {
                  v -= (float)((times >> (16 * k)) & 0xffff) * (ROWS ? mine.fs : fs[k]);
                  if (ROWS && first + c + k >= n_other) v = 0.0f;
                }
                if constexpr (!ROWS) part[k] += v;
                df[b][q >> 1][4 * (q & 1) + k] = (T)v;
              }
              __builtin_amdgcn_sched_barrier(0);
            }
        };
        if (any || masked) form(std::true_type());
        else form(std::false_type());
        if constexpr (!ROWS) sums += (part[0] + part[1]) + (part[2] + part[3]);
        // dz times what passes by: k in the accumulators' order, 16 c + 8 hi + 4 g + 0..3 of a block
        Frag uf[4];
        auto turned = [&](int k) {  // k = 8 b + 4 c + u
          const char* const q = p + 4096 * (k >> 2);
          const int to = turned_at ^ (64 * (k & 3));
          uf[k & 3] = nw_join<T>(tp_turned<T>(q + to), tp_turned<T>(q + (to ^ 32) + 2048));
        };
#pragma unroll
        for (int k = 0; k < 3; ++k) turned(k);
#pragma unroll
        for (int k = 0; k < 16; ++k) {
          if (k + 3 < 16) turned(k + 3);
          __builtin_amdgcn_sched_barrier(0);
          acc[k & 3] = tp_mma(uf[k & 3], df[k >> 3][(k >> 2) & 1], acc[k & 3]);
          __builtin_amdgcn_sched_barrier(0);
        }
      }
    }
    if constexpr (ROWS) {
      if (me < B) {
        float* o = slabs + ((int64_t)range * B + me) * NW_COLS + 4 * g;
#pragma unroll
        for (int u = 0; u < 4; ++u)
#pragma unroll
          for (int q = 0; q < 4; ++q)
            *reinterpret_cast<f32x4*>(o + 32 * u + 8 * q) =
                f32x4{acc[u][4 * q], acc[u][4 * q + 1], acc[u][4 * q + 2], acc[u][4 * q + 3]};
      }
    } else {
      sums += __builtin_bit_cast(float, lane_xor<32>(__builtin_bit_cast(unsigned, sums), lane));
      if (db && g == 0 && me < n_own) db[me] = sums * out;
      if (dw.data) {
        // 32 columns at a time through the wave's block of counts, chunk c of label r at place c ^ (r % 8)
        float* const block = reinterpret_cast<float*>(counts + 4096 * wave);
#pragma unroll
        for (int u = 0; u < 4; ++u) {
#pragma unroll
          for (int q = 0; q < 4; ++q)
            *reinterpret_cast<f32x4*>(block + 32 * n + 4 * ((2 * q + g) ^ (n & 7))) =
                f32x4{acc[u][4 * q] * out, acc[u][4 * q + 1] * out, acc[u][4 * q + 2] * out, acc[u][4 * q + 3] * out};
          __builtin_amdgcn_fence(__ATOMIC_SEQ_CST, "wavefront");
#pragma unroll 1
          for (int r = lane >> 2; r < 32; r += 16) {
            const int c = 2 * (lane & 3), label = me - n + r, col = 32 * u + 4 * c;
            const f32x4 lo = *reinterpret_cast<const f32x4*>(block + 32 * r + 4 * (c ^ (r & 7)));
            const f32x4 hi = *reinterpret_cast<const f32x4*>(block + 32 * r + 4 * ((c + 1) ^ (r & 7)));
            float v[8] = {lo[0], lo[1], lo[2], lo[3], hi[0], hi[1], hi[2], hi[3]};
            if (label < n_own && col < d) store8(dw, label, col, min(8, d - col), v);
          }
          __builtin_amdgcn_fence(__ATOMIC_SEQ_CST, "wavefront");
        }
      }
    }
  }
}

// ---- launches ----------------------------------------------------------------------------------------
bool narrow_takes(int dtype, int d) { return dtype != 0 && d <= NW_COLS; }
bool narrow_grad_takes(int dtype, int n_rows, int d) { return narrow_takes(dtype, d) && n_rows <= NW_ROWS; }

// Labels that give most of the chip's 512 places a block (loss and gradients in bf16, general kernels and these: 4,096 rows,
// 48,000 labels 503 and 384 us; 1,584 rows, 17,219 labels, 75 a row 140 and 205; 278 rows, 16,698 labels 58 and 83).
bool narrow_sides_take(int dtype, int n_rows, int n_labels, int d) {
  return narrow_takes(dtype, d) && n_rows > NW_ROWS && n_rows <= 1 << 18 && n_labels >= 40000;
}
// Whether the lists are short enough that most workgroups list the targets of their share of labels at once (evenly spread: three
// quarters of what a list holds).  More are right as well, in several lists, but then the general kernels are as fast or
// faster: 4,096 rows of 300 labels out of 40,001 918 us with them, 1,041 with these.  A few labels that fill lists of their own
// (ids by a Zipf law of exponent 1.1): 8,192 rows of 75 labels out of 205,443 5,400 and 3,867, 4,096 rows of 40 labels out of
// 40,001 518 and 590.
bool narrow_sides_worth(int n_rows, int n_labels, int nnz) {
  const int64_t labels = NWS_OWN * ceil_div(ceil_div(n_labels, NWS_OWN), 512);
  return (int64_t)nnz * labels <= (int64_t)(NWS_HITS * 3 / 4) * n_labels;
}
// Rows in registers: about 512 workgroups.
NarrowPlan narrow_rows_plan(int n_rows, int n_labels) {
  NarrowPlan p;
  p.row_blocks = (int)ceil_div(n_rows, NWS_OWN);
  p.tiles = (int)ceil_div(n_labels, NW_TILE);
  p.per = (int)ceil_div(p.tiles, p.row_blocks < 512 ? 512 / p.row_blocks : 1);
  p.ranges = (int)ceil_div(p.tiles, p.per);
  return p;
}
// Labels in registers: up to 512 workgroups.
static NarrowPlan narrow_labels_plan(int n_rows, int n_labels) {
  NarrowPlan p;
  p.row_blocks = (int)ceil_div(n_labels, NWS_OWN);
  p.tiles = (int)ceil_div(n_rows, NW_TILE);
  p.per = (int)ceil_div(p.row_blocks, 512);
  p.ranges = (int)ceil_div(p.row_blocks, p.per);
  return p;
}

NarrowPlan narrow_lse_plan(int n_rows, int n_labels) {
  NarrowPlan p;
  p.row_blocks = (int)ceil_div(n_rows, NW_ROWS);
  p.tiles = (int)ceil_div(n_labels, NW_TILE);
  // ranges: one round of the chip's 512 places, or up to 16 over several rounds where the last is then fuller (33,000 rows,
  // 30,000 labels: 483 us with 4 of them, 344 with 3, 324 with 11; 70,000 rows: 956 with 2, 898 with 1, 656 with 13)
  const auto rounds = [&](int64_t r) { return (double)ceil_div(p.row_blocks * r, 512) / (double)r; };
  int64_t want = p.row_blocks < 512 ? 512 / p.row_blocks : 1;
  for (int64_t r = want + 1; r <= 16; ++r)
    if (rounds(r) < 0.95 * rounds(want)) want = r;
  p.per = (int)ceil_div(p.tiles, want);
  p.ranges = (int)ceil_div(p.tiles, p.per);
  return p;
}
NarrowPlan narrow_grad_plan(int n_labels) {
  NarrowPlan p;
  p.row_blocks = 1;
  p.tiles = (int)ceil_div(n_labels, NW_TILE);
  p.per = (int)ceil_div(p.tiles, 256);
  p.ranges = (int)ceil_div(p.tiles, p.per);
  return p;
}
size_t narrow_slab_bytes(const NarrowPlan& p, int n_rows) { return round256((size_t)p.ranges * n_rows * NW_COLS * 4); }

hipError_t launch_narrow_lse(int dtype, const NarrowPlan& p, const TpOperand& h, const TpOperand& w, const float* bias,
                             int n_rows, int n_labels, int d, float2* part, hipStream_t st) {
  const unsigned blocks = (unsigned)(ceil_div((int64_t)p.ranges * p.row_blocks, 8) * 8);
  const auto fn = dtype == 1 ? k_narrow_lse<bf16> : k_narrow_lse<f16>;
  const hipError_t e = tp_allow_lds((const void*)fn, NWF_LDS);
  if (e != hipSuccess) return e;
  hipLaunchKernelGGL(fn, dim3(blocks), dim3(NWF_THREADS), NWF_LDS, st, h, w, bias, n_rows, n_labels, 2 * d, p.row_blocks,
                     p.ranges, p.per, p.tiles, part);
  return hipGetLastError();
}

hipError_t launch_narrow_grad(int dtype, const NarrowPlan& p, const TpOperand& h, const TpOperand& w, const DzArgs& a,
                              int n_rows, int d, float alpha, const MatDev& dw, float* db, float* slabs, hipStream_t st) {
  const auto fn = dtype == 1 ? k_narrow_grad<bf16> : k_narrow_grad<f16>;
  const hipError_t e = tp_allow_lds((const void*)fn, NWG_LDS);
  if (e != hipSuccess) return e;
  hipLaunchKernelGGL(fn, dim3(p.ranges), dim3(NW_THREADS), NWG_LDS, st, h, w, a, n_rows, d, p.ranges, p.per, p.tiles, alpha,
                     dw, db, slabs);
  return hipGetLastError();
}

template <typename T>
static hipError_t sides(const NarrowPlan& p, const TpOperand& h, const TpOperand& w, const DzArgs& a, int n_rows, int d,
                        float alpha, const MatDev& dw, float* db, float* slabs, hipStream_t st) {
  hipError_t e = hipSuccess;
  const int L = a.n_labels;
  if (slabs) {
    const auto fn = k_narrow_side<T, true>;
    if ((e = tp_allow_lds((const void*)fn, NWS_LDS)) != hipSuccess) return e;
    hipLaunchKernelGGL(fn, dim3((unsigned)(8 * ceil_div((int64_t)p.ranges * p.row_blocks, 8))), dim3(NWS_THREADS), NWS_LDS, st, h,
                       w, a, n_rows, L, d, p.row_blocks, p.ranges, p.per, p.tiles, alpha, MatDev{}, (float*)nullptr, slabs);
    if ((e = hipGetLastError()) != hipSuccess) return e;
  }
  if (dw.data || db) {
    const NarrowPlan q = narrow_labels_plan(n_rows, L);
    const auto fn = k_narrow_side<T, false>;
    if ((e = tp_allow_lds((const void*)fn, NWS_LDS)) != hipSuccess) return e;
    hipLaunchKernelGGL(fn, dim3((unsigned)(8 * ceil_div(q.ranges, 8))), dim3(NWS_THREADS), NWS_LDS, st, w, h, a, L, n_rows, d,
                       q.row_blocks, q.ranges, q.per, q.tiles, alpha, dw, db, (float*)nullptr);
    e = hipGetLastError();
  }
  return e;
}
hipError_t launch_narrow_sides(int dtype, const NarrowPlan& p, const TpOperand& h, const TpOperand& w, const DzArgs& a,
                               int n_rows, int d, float alpha, const MatDev& dw, float* db, float* slabs, hipStream_t st) {
  return dtype == 1 ? sides<bf16>(p, h, w, a, n_rows, d, alpha, dw, db, slabs, st)
                    : sides<f16>(p, h, w, a, n_rows, d, alpha, dw, db, slabs, st);
}

}  // namespace asgd

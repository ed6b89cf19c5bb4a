// Differential attention inside groups, forward and backward (diff_attn.h has the formulas of the forward).
//
// Backward, with lse_m, P_m = exp(s S_m - lse_m), O_m = P_m V and dP = dO V^T, which both maps share:
//   delta_m = rowsum(dO * O_m)
//   dS_1 = P_1 * (dP - delta_1), dS_2 = -lambda P_2 * (dP - delta_2), dQ_m = s dS_m K_m, dK_m = s dS_m^T Q_m
//   dV = (P_1 - lambda P_2)^T dO, dlambda = -sum P_2 * dP
// so that a backward has the matrix products of plain attention, and a forward one and a half times them (two weighted sums of V).
//
// bf16 calls of long groups are bound by the matrix and vector work of a SIMD (diff_steps.h, diff_keys.h), those of groups of some hundred rows by rounds of
// unequal blocks (matrix cores busy 0.33 to 0.37 of the cycles at 10,007 x 12, 20 groups), those of few queries by HBM, fp32 calls by products of 1 / 8
// of bf16's rate (8,192 x 12 heads of 128, one group: 120 TFLOP/s forward and dQ, 102 dK and dV, of 154) and, at the sizes of gradient
// checks, by launches and by the length of a group's sweep.
#include <algorithm>
#include <cmath>

#include "diff_keys.h"
#include "diff_steps.h"

namespace moga {
namespace {

constexpr float kLog2e = 1.4426950408889634f;

template <typename T> constexpr int kCols = sizeof(T) == 4 ? 1 : 2;   // columns of 16 rows of a wave
template <typename T> constexpr int kRows = 64 * kCols<T>;            // rows of a block of four waves
template <typename T> constexpr int kKeyRows = sizeof(T) == 4 ? 64 : 4 * DiffKeySweep::kKeys;   // the same of dK and dV

struct DiffFwd {
  const void *q, *k, *v;
  const float* lambda;
  const int32_t *cu_q, *cu_k, *tile_start;
  int64_t Nq, Nk;
  int H, G;
  float scale;
  void* o;
  float* parts;   // NULL, or O_1 and O_2 as they are, [2][H][Nq][D]
  float* lse;     // [2][H][Nq]
  // split: pieces of a tile's keys, [piece][H][Nq] rows of two maps' fp32 sums, and of their (maximum, sum)
  float *part, *stat;
};

// Running maximum of the exponents, sums of the weights, and sums of V: columns of a wave, both maps.
template <int D, int NC> struct DiffState {
  floatx4_t o[2][D / 16][NC];
  float m[2][NC], l[2][NC], thresh[2][NC];
  __device__ __forceinline__ void init() {
#pragma unroll
    for (int k = 0; k < 2; ++k)
#pragma unroll
      for (int q = 0; q < NC; ++q) {
        m[k][q] = l[k][q] = 0.f;
        thresh[k][q] = -INFINITY;
#pragma unroll
        for (int dt = 0; dt < D / 16; ++dt) o[k][dt][q] = floatx4_t{0.f, 0.f, 0.f, 0.f};
      }
  }
};

// One step: 32 keys, of which `left` exist (MASK).
template <bool MASK, typename T, int D, int NC, typename Tiles>
__device__ __forceinline__ void diff_fwd_step(const Tiles& tiles, const Frag<T> (&qf)[NC][D / 32], DiffState<D, NC>& st, float c, int left) {
  constexpr int KB = D / 64;   // k blocks of a map
  const int g = (threadIdx.x & 63) >> 4;
  float x[2][NC][8], mx[2][NC];
  bool up = false;
#pragma unroll
  for (int m = 0; m < 2; ++m) {
    floatx4_t s[2][NC];
#pragma unroll
    for (int t = 0; t < 2; ++t)
#pragma unroll
      for (int kb = 0; kb < KB; ++kb) {
        const Frag<T> a = tiles.nat(0, t, m * KB + kb);
#pragma unroll
        for (int q = 0; q < NC; ++q) s[t][q] = mma(a, qf[q][m * KB + kb], kb == 0 ? floatx4_t{0.f, 0.f, 0.f, 0.f} : s[t][q]);
      }
#pragma unroll
    for (int q = 0; q < NC; ++q) {
#pragma unroll
      for (int i = 0; i < 8; ++i) {
        x[m][q][i] = fmaf(s[i >> 2][q][i & 3], c, -st.m[m][q]);
        if (MASK && 8 * g + i >= left) x[m][q][i] = -INFINITY;
      }
      const float(&y)[8] = x[m][q];
      mx[m][q] = fmaxf(max3(max3(max3(y[0], y[1], y[2]), y[3], y[4]), y[5], y[6]), y[7]);
      up = up || mx[m][q] > st.thresh[m][q];
    }
  }
  // The maximum is raised when a weight would exceed 2^8 only: rare after the first step.
  if (__builtin_amdgcn_ballot_w64(up) != 0) {
#pragma unroll
    for (int m = 0; m < 2; ++m)
#pragma unroll
      for (int q = 0; q < NC; ++q) {
        float all = fmaxf(mx[m][q], __shfl_xor(mx[m][q], 16, kWave));
        all = fmaxf(all, __shfl_xor(all, 32, kWave));
        const bool first = st.thresh[m][q] == -INFINITY;
        const float by = first ? (all == -INFINITY ? 0.f : all) : fmaxf(all, 0.f);
        const float alpha = first ? 0.f : fast_exp2(-by);
        if (all != -INFINITY) st.thresh[m][q] = 8.f;
        st.m[m][q] += by;
        st.l[m][q] *= alpha;
#pragma unroll
        for (int i = 0; i < 8; ++i) x[m][q][i] -= by;
#pragma unroll
        for (int dt = 0; dt < D / 16; ++dt) st.o[m][dt][q] *= alpha;
      }
  }
  Frag<T> pf[2][NC];
#pragma unroll
  for (int m = 0; m < 2; ++m)
#pragma unroll
    for (int q = 0; q < NC; ++q) {
      float(&y)[8] = x[m][q];
#pragma unroll
      for (int i = 0; i < 8; ++i) y[i] = fast_exp2(y[i]);
      // sums of the weights in 32 bits, before they are rounded: the log-sum-exp is exact enough for the gradient of lambda
      st.l[m][q] += ((y[0] + y[1]) + (y[2] + y[3])) + ((y[4] + y[5]) + (y[6] + y[7]));
      make_frag(pf[m][q], y);
    }
#pragma unroll
  for (int dt = 0; dt < D / 16; ++dt) {
    const Frag<T> a = tiles.tr(1, dt);
#pragma unroll
    for (int m = 0; m < 2; ++m)
#pragma unroll
      for (int q = 0; q < NC; ++q) st.o[m][dt][q] = mma(a, pf[m][q], st.o[m][dt][q]);
  }
}

// fp32: step by step.  4,096 x 2 heads of 64, 8 groups: 33 us in pieces of the keys and 7 to join them.
template <typename T, int D>
struct DiffPlainSweep : DiffState<D, 1> {
  typedef DiffTiles<T, D> Tiles;
  Frag<T> qf[1][D / 32];
  float c;
  Tiles tiles;
  __device__ __forceinline__ void sweep(int n) {
    const int full = n >> 5;
    for (int s = 0; s < full; ++s) {
      if (s > 0) tiles.ready(s);
      diff_fwd_step<false, T, D, 1>(tiles, qf, *this, c, 32);
    }
    if (n & 31) {
      if (full > 0) tiles.ready(full);
      diff_fwd_step<true, T, D, 1>(tiles, qf, *this, c, n & 31);
    }
  }
};

// Piece `piece` of n rows from `first` on: whole steps of 32, as evenly as they go.
__device__ __forceinline__ void piece_range(int piece, int pieces, int& first, int& n) {
  const int64_t steps = (n + 31) >> 5;
  const int t0 = (int)(steps * piece / pieces), t1 = (int)(steps * (piece + 1) / pieces);
  const int end = min(n, 32 * t1);
  first += 32 * t0;
  n = end - 32 * t0;
}

// A tile of kRows queries, or (SPLIT) blockIdx.y's share of its keys.  32,760 x 12 heads, bf16, 8 groups 1.31 ms by itself; 10,007 x 12, 20 groups
// of unequal length 117 us.
template <typename T, int D, bool SPLIT>
__global__ __launch_bounds__(256, 2) void diff_fwd_kernel(DiffFwd a) {
  constexpr int NC = kCols<T>;
  typedef std::conditional_t<sizeof(T) == 4, DiffPlainSweep<float, D>, DiffFwdSweep> Sweep;
  __shared__ typename Sweep::Tiles::Lds lds;
  WorkTile w;
  if (!find_work<false>(a.cu_q, a.tile_start, a.G, a.H, kRows<T>, blockIdx.x, w)) return;
  const int head = w.head, ge = w.ti.row_end;
  int gs = a.cu_k[w.ti.group], n = a.cu_k[w.ti.group + 1] - gs;
  if constexpr (SPLIT) piece_range(blockIdx.y, gridDim.y, gs, n);
  gs = __builtin_amdgcn_readfirstlane(gs);
  n = __builtin_amdgcn_readfirstlane(n);
  const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), lane = threadIdx.x & 63, r = lane & 15, g = lane >> 4;
  const int row0 = w.ti.tile_row + 16 * NC * wave;
  const int64_t head_q = (int64_t)head * a.Nq, head_k = (int64_t)head * a.Nk;

  Sweep st;
  st.init();
  if (n > 0) {
    st.tiles.start(lds, (const T*)a.k + (head_k + gs) * D, (const T*)a.v + (head_k + gs) * D, n);
    if (row0 >= ge) {   // no queries: this wave moves its share of the tiles and keeps the barriers
      for (int s = 0; s < (n + 31) >> 5; ++s) st.tiles.ready(s);
      st.tiles.finish();
      return;
    }
    diff_columns<T, D, NC>(st.qf, (const T*)a.q, row0, ge, head_q);
    if constexpr (sizeof(T) == 2) settle(st.qf);
    st.c = uniform_float(a.scale * kLog2e);
    st.tiles.ready(0);
    st.sweep(n);
    st.tiles.finish();
  }
  if (row0 >= ge) return;
#pragma unroll
  for (int q = 0; q < NC; ++q) {
    const int row = row0 + 16 * q + r;
    float l[2];
#pragma unroll
    for (int m = 0; m < 2; ++m) {
      l[m] = st.l[m][q] + __shfl_xor(st.l[m][q], 16, kWave);
      l[m] += __shfl_xor(l[m], 32, kWave);
    }
    if (row >= ge) continue;
    if constexpr (SPLIT) {
      const int64_t at = ((int64_t)blockIdx.y * a.H * a.Nq + head_q + row) * 2;
#pragma unroll
      for (int m = 0; m < 2; ++m) {
#pragma unroll
        for (int dt = 0; dt < D / 16; ++dt) store4(a.part + (at + m) * D, dt, st.o[m][dt][q]);
        if (g == 0) *(floatx2_t*)(a.stat + (at + m) * 2) = floatx2_t{st.thresh[m][q] == -INFINITY ? -INFINITY : st.m[m][q], n > 0 ? l[m] : -1.f};
      }
    } else {
      const float inv1 = n > 0 ? 1.f / l[0] : 0.f, inv2 = n > 0 ? 1.f / l[1] : 0.f, lam = a.lambda[head];
#pragma unroll
      for (int dt = 0; dt < D / 16; ++dt) {
        const floatx4_t o1 = st.o[0][dt][q] * inv1, o2 = st.o[1][dt][q] * inv2;
        floatx4_t o;   // one rounding of the maps' own sums, written out: else the compiler chooses, and not alike with and without parts
#pragma unroll
        for (int i = 0; i < 4; ++i) o[i] = fmaf(-lam, o2[i], o1[i]);
        store4((T*)a.o + (head_q + row) * D, dt, o);
        if (a.parts) {
          store4(a.parts + (head_q + row) * D, dt, o1);
          store4(a.parts + ((int64_t)a.H * a.Nq + head_q + row) * D, dt, o2);
        }
      }
      if (g == 0)
#pragma unroll
        for (int m = 0; m < 2; ++m)
          a.lse[(int64_t)m * a.H * a.Nq + head_q + row] = n > 0 ? logf(l[m]) + st.m[m][q] * 0.6931471805599453f : -INFINITY;
    }
  }
}

// bf16 calls of few queries: the blocks go by the keys, `chunk` of a group each, and take all queries of the group, 16 at a time.  The
// four waves share the keys out, every fourth tile each from a ring of its own without a barrier, and add up what they have.  Bound by HBM:
// 4 x 32 KB are on their way to a CU.  4 queries, 65,536 keys, 12 heads: 78 us, 5.2 TB/s; a call, with the join, of four lists of equal length 92 us,
// by tiles of 128 queries with split keys 109.
// Sums and maxima go to part and stat, for piece (first key / chunk) of the group.
__global__ __launch_bounds__(256, 1) void diff_few_kernel(DiffFwd a, int chunk) {
  constexpr int D = kHeadDim;
  typedef unsigned short T;
  __shared__ union {
    DiffWaveTiles::Lds tiles[4];
    struct { float o[4][2][16][D], stat[4][2][16][2]; } sums;
  } lds;
  WorkTile w;
  if (!find_work<false>(a.cu_k, a.tile_start, a.G, a.H, chunk, blockIdx.x, w)) return;
  const int head = w.head, gs = __builtin_amdgcn_readfirstlane(w.ti.tile_row);
  const int n = __builtin_amdgcn_readfirstlane(min(w.ti.row_end, w.ti.tile_row + chunk)) - gs, piece = (gs - w.ti.row_begin) / chunk;
  const int q_first = a.cu_q[w.ti.group], q_end = a.cu_q[w.ti.group + 1];
  const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), lane = threadIdx.x & 63, r = lane & 15;
  const int64_t head_q = (int64_t)head * a.Nq, head_k = (int64_t)head * a.Nk;
  const int tiles_n = (n + 31) >> 5;
  const float c = a.scale * kLog2e;
  for (int row0 = q_first; row0 < q_end; row0 += 16) {
    DiffState<D, 1> st;
    st.init();
    bf16x8_t qf[1][4];
    diff_columns<T, D, 1>(qf, (const T*)a.q, row0, q_end, head_q);
    settle(qf);
    if (wave < tiles_n) {
      DiffWaveTiles tiles;
      tiles.start(lds.tiles[wave], (const T*)a.k + (head_k + gs) * D, (const T*)a.v + (head_k + gs) * D, n, wave);
      for (int t = wave; t < tiles_n; t += 4) {
        tiles.next();
        if (n - 32 * t >= 32) diff_fwd_step<false, T, D, 1>(tiles, qf, st, c, 32);
        else diff_fwd_step<true, T, D, 1>(tiles, qf, st, c, n - 32 * t);
        tiles.refill(t + 8);
      }
      tiles.finish();
    }
    __syncthreads();   // the rings are read no more
#pragma unroll
    for (int m = 0; m < 2; ++m) {
      float l = st.l[m][0] + __shfl_xor(st.l[m][0], 16, kWave);
      l += __shfl_xor(l, 32, kWave);
#pragma unroll
      for (int dt = 0; dt < D / 16; ++dt) store4(lds.sums.o[wave][m][r], dt, st.o[m][dt][0]);
      if (lane < 16) {
        lds.sums.stat[wave][m][r][0] = st.thresh[m][0] == -INFINITY ? -INFINITY : st.m[m][0];
        lds.sums.stat[wave][m][r][1] = l;
      }
    }
    __syncthreads();
    const int used = min(4, tiles_n);
    for (int i = threadIdx.x; i < 2 * 16 * (D / 4); i += 256) {
      const int col = i % (D / 4) * 4, m = i / (D / 4) / 16, q = i / (D / 4) % 16;
      if (row0 + q >= q_end) continue;
      float mx = -INFINITY, l = 0.f;
      for (int k = 0; k < used; ++k) mx = fmaxf(mx, lds.sums.stat[k][m][q][0]);
      floatx4_t o = {0.f, 0.f, 0.f, 0.f};
      for (int k = 0; k < used; ++k) {
        const float f = mx == -INFINITY ? 1.f : fast_exp2(lds.sums.stat[k][m][q][0] - mx);
        l = fmaf(lds.sums.stat[k][m][q][1], f, l);
        o += *(const floatx4_t*)&lds.sums.o[k][m][q][col] * f;
      }
      const int64_t at = ((int64_t)piece * a.H * a.Nq + head_q + row0 + q) * 2 + m;
      *(floatx4_t*)(a.part + at * D + col) = o;
      if (col == 0) *(floatx2_t*)(a.stat + at * 2) = floatx2_t{mx, l};
    }
    __syncthreads();   // the sums are read no more
  }
}

// The pieces of a row put together: a wave per row, D / 64 channels of both maps per lane.  chunk > 0: a piece for every `chunk` keys of the
// row's group (diff_few_kernel), else `pieces`.
template <typename T, int D>
__global__ __launch_bounds__(256) void diff_merge_kernel(DiffFwd a, int pieces, int chunk) {
  constexpr int V = D / 64;
  const int lane = threadIdx.x & 63;
  const int64_t rows = (int64_t)a.H * a.Nq, row = (int64_t)blockIdx.x * 4 + (threadIdx.x >> 6);
  if (row >= rows || row % a.Nq >= a.cu_q[a.G]) return;   // rows behind the last group stay as they are
  if (chunk > 0) {
    TileInfo ti;   // tiles of one row: the entries of cu_q are their own sums
    find_tile_presummed(a.cu_q, a.cu_q, a.G, 1, (int)(row % a.Nq), ti);
    pieces = (a.cu_k[ti.group + 1] - a.cu_k[ti.group] + chunk - 1) / chunk;
  }
  float o[2][V], lse[2], mx[2], l[2];
#pragma unroll
  for (int m = 0; m < 2; ++m) {
    mx[m] = -INFINITY;
    l[m] = 0.f;
#pragma unroll
    for (int i = 0; i < V; ++i) o[m][i] = 0.f;
  }
  bool empty = true;
  for (int p0 = 0; p0 < pieces; p0 += 64) {   // (maximum, sum) of 64 pieces at a time, a lane each; a sum of -1: no keys
    floatx4_t s = {-INFINITY, -1.f, -INFINITY, -1.f};
    if (p0 + lane < pieces) s = *(const floatx4_t*)(a.stat + ((p0 + lane) * rows + row) * 4);
    const bool none = s[1] == -1.f;
    if (__builtin_amdgcn_ballot_w64(!none) == 0) continue;
    empty = false;
    float f[2];
#pragma unroll
    for (int m = 0; m < 2; ++m) {
      const float now = fmaxf(mx[m], wave_max(s[2 * m])), before = mx[m] == now ? 1.f : fast_exp2(mx[m] - now);
      f[m] = none ? 0.f : now == -INFINITY ? 1.f : fast_exp2(s[2 * m] - now);
      mx[m] = now;
      l[m] = fmaf(l[m], before, wave_sum(none ? 0.f : s[2 * m + 1] * f[m]));
#pragma unroll
      for (int i = 0; i < V; ++i) o[m][i] *= before;
    }
    const int n = min(64, pieces - p0);
    for (int p = 0; p < n; p += 4) {   // four on their way
      float v[4][2][V], w[4][2];
#pragma unroll
      for (int u = 0; u < 4; ++u) {
        const float* part = a.part + ((p0 + min(p + u, n - 1)) * rows + row) * 2 * D + lane * V;
#pragma unroll
        for (int m = 0; m < 2; ++m) {
          w[u][m] = __shfl(f[m], min(p + u, n - 1), kWave);
#pragma unroll
          for (int i = 0; i < V; ++i) v[u][m][i] = part[m * D + i];
        }
      }
#pragma unroll
      for (int u = 0; u < 4; ++u)
        if (p + u < n)
#pragma unroll
          for (int m = 0; m < 2; ++m)
#pragma unroll
            for (int i = 0; i < V; ++i) o[m][i] = fmaf(v[u][m][i], w[u][m], o[m][i]);
    }
  }
#pragma unroll
  for (int m = 0; m < 2; ++m) {
#pragma unroll
    for (int i = 0; i < V; ++i) o[m][i] = empty ? 0.f : o[m][i] / l[m];
    lse[m] = empty ? -INFINITY : logf(l[m]) + mx[m] * 0.6931471805599453f;
  }
  const float lam = a.lambda[row / a.Nq];
  T* out = (T*)a.o + row * D + lane * V;
#pragma unroll
  for (int i = 0; i < V; ++i) {
    const float v = fmaf(-lam, o[1][i], o[0][i]);
    if constexpr (sizeof(T) == 4) out[i] = v;
    else out[i] = f32_to_bf16_bits(v);
    if (a.parts) {
      a.parts[row * D + lane * V + i] = o[0][i];
      a.parts[(rows + row) * D + lane * V + i] = o[1][i];
    }
  }
  if (lane < 2) a.lse[lane * rows + row] = lane ? lse[1] : lse[0];
}

// ---- backward ---------------------------------------------------------------------------------------------------------
struct DiffBwd {
  const void *d_o, *q, *k, *v;
  const float* lambda;
  const int32_t *cu_q, *cu_k, *tile_start;   // tiles of the side that the blocks own
  const floatx4_t* rows;                     // [H][Nq]: lse_1, lse_2 in powers of two, -delta_1, delta_2 - delta_1
  int64_t Nq, Nk;
  int H, G;
  float scale;
  void *d_q, *d_k, *d_v;
  float* share;   // [H][Nq]: a row's part of -dlambda
  // split: pieces of the other side's rows, [piece] of d_q and of share as they are above, and of d_k, then d_v, in fp32
  float *part_q, *part_share, *part_k;
  int q_pieces, k_pieces;
};

// The row constants: 16 lanes per row, bound by HBM (62,400 x 12 heads, bf16: 0.17 ms, 5.8 TB/s).  delta is made of the unrounded O_m: from
// rounded ones the gradients of groups of some hundred keys are a tenth further off (shorter groups: diff_delta_kernel).  share (fp32): the
// rows' parts of -dlambda, which are delta_2; of bf16 calls, whose O_2 comes from rounded weights, the dQ kernel makes them from the
// unrounded ones.
template <typename T, int D>
__global__ __launch_bounds__(256) void diff_rows_kernel(const T* __restrict__ d_o, const float* __restrict__ parts, const float* __restrict__ lse,
                                                        int64_t rows, floatx4_t* __restrict__ out, float* __restrict__ share) {
  const int64_t row = (int64_t)blockIdx.x * 16 + (threadIdx.x >> 4);
  const int t = threadIdx.x & 15;
  if (row >= rows) return;
  float a = 0.f, b = 0.f;
#pragma unroll
  for (int col = 4 * t; col < D; col += 64) {
    floatx4_t d;
    if constexpr (sizeof(T) == 4) {
      d = *(const floatx4_t*)(d_o + row * D + col);
    } else {
      const uintx2_t u = *(const uintx2_t*)(d_o + row * D + col);
      d = floatx4_t{bf16_lo_to_f32(u[0]), bf16_hi_to_f32(u[0]), bf16_lo_to_f32(u[1]), bf16_hi_to_f32(u[1])};
    }
    const floatx4_t x = *(const floatx4_t*)(parts + row * D + col), y = *(const floatx4_t*)(parts + (rows + row) * D + col);
#pragma unroll
    for (int e = 0; e < 4; ++e) {
      a = fmaf(d[e], x[e], a);
      b = fmaf(d[e], y[e], b);
    }
  }
  a = lanes_sum<16>(a);
  b = lanes_sum<16>(b);
  if (t == 0) {
    out[row] = floatx4_t{lse[row] * kLog2e, lse[rows + row] * kLog2e, -a, b - a};
    if constexpr (sizeof(T) == 4) share[row] = b;
  }
}

// Scores of both maps and dP of 16 rows of a tile: its first tensor's times x, its second's times y.
template <typename T, int D, int NC, typename Tiles>
__device__ __forceinline__ void diff_products(const Tiles& tiles, int t, const Frag<T> (&x)[NC][D / 32], const Frag<T> (&y)[NC][D / 32],
                                              floatx4_t (&s)[2][NC], floatx4_t (&dp)[NC]) {
  constexpr int KB = D / 64;
#pragma unroll
  for (int kb = 0; kb < 2 * KB; ++kb) {
    const Frag<T> f = tiles.nat(0, t, kb);
#pragma unroll
    for (int c = 0; c < NC; ++c) s[kb / KB][c] = mma(f, x[c][kb], kb % KB == 0 ? floatx4_t{0.f, 0.f, 0.f, 0.f} : s[kb / KB][c]);
  }
#pragma unroll
  for (int kb = 0; kb < 2 * KB; ++kb) {
    const Frag<T> f = tiles.nat(1, t, kb);
#pragma unroll
    for (int c = 0; c < NC; ++c) dp[c] = mma(f, y[c][kb], kb == 0 ? floatx4_t{0.f, 0.f, 0.f, 0.f} : dp[c]);
  }
}

// The row constants of bf16 calls of short groups, with delta_m = sum P_m dP from unrounded weights by a sweep of their own.  The forward's sums
// of V have weights rounded to operands, and where few keys carry a row delta's error is felt: dQ's is 1.43 of a plain rounding's instead of
// 1.49 at 70 keys a group, dK's 1.41 instead of 1.46.  Up to 256 keys of a mean group the sweep takes what reading `parts` does (backward of
// 10,007 x 12 heads, 40 groups 141 us against 138, 60,000 x 12, 1,000 groups 674 against 682, 1,560 x 4, 8 groups 34 against 29); at
// 500 keys it takes longer (20 groups 220 against 192) for 1.445 instead of 1.47.  The host knows the mean group only: a long group among short ones pays for
// three products more beside the backward's seven.
constexpr int64_t kDeltaKeys = 256;
__global__ __launch_bounds__(256, 3) void diff_delta_kernel(DiffBwd a, const float* __restrict__ lse, floatx4_t* __restrict__ out) {
  constexpr int NC = kCols<unsigned short>, D = kHeadDim;
  typedef unsigned short T;
  typedef DiffTiles<T, D, false, 1, 2> Tiles;   // a ring of two: three blocks a CU
  __shared__ Tiles::Lds lds;
  WorkTile w;
  if (!find_work<false>(a.cu_q, a.tile_start, a.G, a.H, kRows<T>, blockIdx.x, w)) return;
  const int head = w.head, ge = w.ti.row_end;
  const int gs = __builtin_amdgcn_readfirstlane(a.cu_k[w.ti.group]);
  const int n = __builtin_amdgcn_readfirstlane(a.cu_k[w.ti.group + 1]) - gs;
  if (n <= 0) return;
  const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), lane = threadIdx.x & 63, r = lane & 15, g = lane >> 4;
  const int row0 = w.ti.tile_row + 16 * NC * wave;
  const int64_t head_q = (int64_t)head * a.Nq, head_k = (int64_t)head * a.Nk;
  const bool active = row0 < ge;
  const float c = a.scale * kLog2e;
  bf16x8_t qf[NC][4], df[NC][4];
  diff_columns<T, D, NC>(qf, (const T*)a.q, row0, ge, head_q);
  diff_columns<T, D, NC>(df, (const T*)a.d_o, row0, ge, head_q);
  float l[2][NC], delta[2][NC];
#pragma unroll
  for (int q = 0; q < NC; ++q)
#pragma unroll
    for (int m = 0; m < 2; ++m) {
      l[m][q] = lse[(int64_t)m * a.H * a.Nq + head_q + min(row0 + 16 * q + r, ge - 1)] * kLog2e;
      delta[m][q] = 0.f;
    }
  Tiles tiles;
  tiles.start(lds, (const T*)a.k + (head_k + gs) * D, (const T*)a.v + (head_k + gs) * D, n);
  for (int st = 0; st < (n + 31) >> 5; ++st) {
    tiles.ready(st);
    if (!active) continue;
    const int left = n - 32 * st;
#pragma unroll
    for (int t = 0; t < 2; ++t) {
      floatx4_t s[2][NC], dp[NC];
      diff_products<T, D>(tiles, t, qf, df, s, dp);
#pragma unroll
      for (int m = 0; m < 2; ++m)
#pragma unroll
        for (int q = 0; q < NC; ++q) {
          float sum = 0.f;
#pragma unroll
          for (int i = 0; i < 4; ++i) {
            const float p = fast_exp2(fmaf(s[m][q][i], c, -l[m][q]));
            sum = fmaf(8 * g + 4 * t + i >= left ? 0.f : p, dp[q][i], sum);
          }
          delta[m][q] += sum;
        }
    }
  }
  tiles.finish();
  if (!active) return;
#pragma unroll
  for (int q = 0; q < NC; ++q) {
#pragma unroll
    for (int m = 0; m < 2; ++m) {
      delta[m][q] += __shfl_xor(delta[m][q], 16, kWave);
      delta[m][q] += __shfl_xor(delta[m][q], 32, kWave);
    }
    const int row = row0 + 16 * q + r;
    if (row < ge && g == 0) out[head_q + row] = floatx4_t{l[0][q], l[1][q], -delta[0][q], delta[1][q] - delta[0][q]};
  }
}

// dQ and the rows' shares of dlambda: a wave owns 16 NC queries and sweeps the keys.  Three products of a step, with Q and dO in registers: the
// compiler's order of a step was as fast as one written out like the forward's, and raised wave priorities were slower.  fp32, 4,096 x 2 heads
// of 64, 8 groups: 32 us.
template <typename T, int D>
__device__ __forceinline__ void diff_dq_block(DiffBwd a, int block, int piece, typename DiffTiles<T, D>::Lds& lds) {
  constexpr int NC = kCols<T>, KB = D / 64, DT = D / 16;
  WorkTile w;
  if (!find_work<false>(a.cu_q, a.tile_start, a.G, a.H, kRows<T>, block, w)) return;
  const int head = w.head, ge = w.ti.row_end;
  int gs = a.cu_k[w.ti.group], n = a.cu_k[w.ti.group + 1] - gs;
  if (a.q_pieces > 1) piece_range(piece, a.q_pieces, gs, n);
  gs = __builtin_amdgcn_readfirstlane(gs);
  n = __builtin_amdgcn_readfirstlane(n);
  const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), lane = threadIdx.x & 63, r = lane & 15, g = lane >> 4;
  const int row0 = w.ti.tile_row + 16 * NC * wave;
  const int64_t head_q = (int64_t)head * a.Nq, head_k = (int64_t)head * a.Nk;
  const bool active = row0 < ge;
  const float c = a.scale * kLog2e, lam = a.lambda[head];
  floatx4_t dq[DT][NC];
  float share[NC];   // sum of P_2 dP.  (With -delta_1 in dP from the start its sum over 60,000 rows is ten times as far off.)
#pragma unroll
  for (int q = 0; q < NC; ++q) {
    share[q] = 0.f;
#pragma unroll
    for (int dt = 0; dt < DT; ++dt) dq[dt][q] = floatx4_t{0.f, 0.f, 0.f, 0.f};
  }
  if (n > 0) {
    Frag<T> qf[NC][D / 32], df[NC][D / 32];
    diff_columns<T, D, NC>(qf, (const T*)a.q, row0, ge, head_q);
    diff_columns<T, D, NC>(df, (const T*)a.d_o, row0, ge, head_q);
    floatx4_t rc[NC];
#pragma unroll
    for (int q = 0; q < NC; ++q) {
      rc[q] = a.rows[head_q + min(row0 + 16 * q + r, ge - 1)];
      rc[q][2] = -rc[q][2];   // delta_1, delta_2
      rc[q][3] += rc[q][2];
    }
    DiffTiles<T, D> tiles;
    tiles.start(lds, (const T*)a.k + (head_k + gs) * D, (const T*)a.v + (head_k + gs) * D, n);
    auto step = [&](auto mask, int left) {
      constexpr bool kMask = mask.value;
      float d1[NC][8], d2[NC][8];
#pragma unroll
      for (int t = 0; t < 2; ++t) {
        floatx4_t s[2][NC], dp[NC];
        diff_products<T, D>(tiles, t, qf, df, s, dp);
#pragma unroll
        for (int q = 0; q < NC; ++q) {
          float sum = 0.f;   // four by themselves: fewer roundings at the size of the whole sum
#pragma unroll
          for (int i = 0; i < 4; ++i) {
            float p1 = fast_exp2(fmaf(s[0][q][i], c, -rc[q][0])), p2 = fast_exp2(fmaf(s[1][q][i], c, -rc[q][1]));
            if (kMask && 8 * g + 4 * t + i >= left) p1 = p2 = 0.f;
            if constexpr (sizeof(T) == 2) sum = fmaf(p2, dp[q][i], sum);
            d1[q][4 * t + i] = p1 * (dp[q][i] - rc[q][2]);
            d2[q][4 * t + i] = p2 * (dp[q][i] - rc[q][3]);
          }
          share[q] += sum;
        }
      }
      Frag<T> f1[NC], f2[NC];
#pragma unroll
      for (int q = 0; q < NC; ++q) {
        make_frag(f1[q], d1[q]);
        make_frag(f2[q], d2[q]);
      }
#pragma unroll
      for (int dt = 0; dt < DT; ++dt) {
        const Frag<T> f = tiles.tr(0, dt);
#pragma unroll
        for (int q = 0; q < NC; ++q) dq[dt][q] = mma(f, dt < DT / 2 ? f1[q] : f2[q], dq[dt][q]);
      }
    };
    const int full = n >> 5;
    for (int s = 0; s < full; ++s) {
      tiles.ready(s);
      if (active) step(std::false_type{}, 32);
    }
    if (n & 31) {
      tiles.ready(full);
      if (active) step(std::true_type{}, n & 31);
    }
    tiles.finish();
  }
  if (!active) return;
#pragma unroll
  for (int q = 0; q < NC; ++q) {
    const int row = row0 + 16 * q + r;
    float sh = share[q] + __shfl_xor(share[q], 16, kWave);
    sh += __shfl_xor(sh, 32, kWave);
    if (row >= ge) continue;
    auto store = [&](auto* out) {
#pragma unroll
      for (int dt = 0; dt < DT; ++dt) store4(out, dt, dq[dt][q] * (dt < DT / 2 ? a.scale : -lam * a.scale));
    };
    if (a.q_pieces > 1) {
      const int64_t at = (int64_t)piece * a.H * a.Nq + head_q + row;
      store(a.part_q + at * D);
      if (sizeof(T) == 2 && g == 0) a.part_share[at] = sh;
    } else {
      store((T*)a.d_q + (head_q + row) * D);
      if (sizeof(T) == 2 && g == 0) a.share[head_q + row] = sh;
    }
  }
}

// fp32 dK and dV: a wave owns 16 keys and sweeps the queries, with their row constants beside them in LDS.  4,096 x 2 heads of 64, 8 groups: 43 us.
template <int D>
__global__ __launch_bounds__(256, 1) void diff_dkdv_f32_kernel(DiffBwd a) {
  typedef float T;
  constexpr int NC = 1, KB = D / 64, DT = D / 16;
  __shared__ typename DiffTiles<T, D, true>::Lds lds;
  WorkTile w;
  if (!find_work<false>(a.cu_k, a.tile_start, a.G, a.H, kKeyRows<T>, blockIdx.x, w)) return;
  const int head = w.head, ge = w.ti.row_end;
  int gs = a.cu_q[w.ti.group], n = a.cu_q[w.ti.group + 1] - gs;
  if (a.k_pieces > 1) piece_range(blockIdx.y, a.k_pieces, gs, n);
  gs = __builtin_amdgcn_readfirstlane(gs);
  n = __builtin_amdgcn_readfirstlane(n);
  const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), lane = threadIdx.x & 63, r = lane & 15, g = lane >> 4;
  const int row0 = w.ti.tile_row + 16 * NC * wave;
  const int64_t head_q = (int64_t)head * a.Nq, head_k = (int64_t)head * a.Nk;
  const bool active = row0 < ge;
  const float c = a.scale * kLog2e, lam = a.lambda[head];
  floatx4_t dk[DT][NC], dv[DT][NC];
#pragma unroll
  for (int k = 0; k < NC; ++k)
#pragma unroll
    for (int dt = 0; dt < DT; ++dt) dk[dt][k] = dv[dt][k] = floatx4_t{0.f, 0.f, 0.f, 0.f};
  if (n > 0) {
    Frag<T> kf[NC][D / 32], vf[NC][D / 32];
    diff_columns<T, D, NC>(kf, (const T*)a.k, row0, ge, head_k);
    diff_columns<T, D, NC>(vf, (const T*)a.v, row0, ge, head_k);
    DiffTiles<T, D, true> tiles;
    tiles.start(lds, (const T*)a.q + (head_q + gs) * D, (const T*)a.d_o + (head_q + gs) * D, n, a.rows + head_q + gs);
    const int steps = (n + 31) >> 5;
    for (int st = 0; st < steps; ++st) {
      tiles.ready(st);
      if (!active) continue;
      const int left = n - 32 * st;
      float pa[NC][8], d1[NC][8], d2[NC][8];
#pragma unroll
      for (int t = 0; t < 2; ++t) {
        floatx4_t s[2][NC], dp[NC];
        diff_products<T, D>(tiles, t, kf, vf, s, dp);
        floatx4_t rc[4];
#pragma unroll
        for (int v = 0; v < 4; ++v) rc[v] = tiles.rows(v, 8 * g + 4 * t);
#pragma unroll
        for (int i = 0; i < 4; ++i) {
          const int q = 8 * g + 4 * t + i;
#pragma unroll
          for (int k = 0; k < NC; ++k) {
            float p1 = fast_exp2(fmaf(s[0][k][i], c, -rc[0][i])), p2 = fast_exp2(fmaf(s[1][k][i], c, -rc[1][i]));
            if (left < 32 && q >= left) p1 = p2 = 0.f;
            pa[k][4 * t + i] = fmaf(-lam, p2, p1);
            const float d = dp[k][i] + rc[2][i];
            d1[k][4 * t + i] = p1 * d;
            d2[k][4 * t + i] = p2 * (rc[3][i] - d);
          }
        }
      }
      Frag<T> fa[NC], f1[NC], f2[NC];
#pragma unroll
      for (int k = 0; k < NC; ++k) {
        make_frag(fa[k], pa[k]);
        make_frag(f1[k], d1[k]);
        make_frag(f2[k], d2[k]);
      }
#pragma unroll
      for (int dt = 0; dt < DT; ++dt) {
        const Frag<T> fd = tiles.tr(1, dt), fq = tiles.tr(0, dt);
#pragma unroll
        for (int k = 0; k < NC; ++k) {
          dv[dt][k] = mma(fd, fa[k], dv[dt][k]);
          dk[dt][k] = mma(fq, dt < DT / 2 ? f1[k] : f2[k], dk[dt][k]);
        }
      }
    }
    tiles.finish();
  }
  if (!active) return;
#pragma unroll
  for (int k = 0; k < NC; ++k) {
    const int row = row0 + 16 * k + r;
    if (row >= ge) continue;
    auto store = [&](auto* d_k, auto* d_v) {
#pragma unroll
      for (int dt = 0; dt < DT; ++dt) {
        store4(d_k, dt, dk[dt][k] * (dt < DT / 2 ? a.scale : lam * a.scale));
        store4(d_v, dt, dv[dt][k]);
      }
    };
    if (a.k_pieces > 1) {
      float* part = a.part_k + ((int64_t)blockIdx.y * 2 * a.H * a.Nk + head_k + row) * D;
      store(part, part + (int64_t)a.H * a.Nk * D);
    } else {
      store((T*)a.d_k + (head_k + row) * D, (T*)a.d_v + (head_k + row) * D);
    }
  }
}

// bf16 dK and dV: diff_keys.h.
__device__ __forceinline__ void diff_dkdv_block(DiffBwd a, int block, int piece, DiffKeySweep::Lds& lds) {
  constexpr int NC = DiffKeySweep::NC, D = kHeadDim;
  typedef unsigned short T;
  WorkTile w;
  if (!find_work<false>(a.cu_k, a.tile_start, a.G, a.H, kKeyRows<T>, block, w)) return;
  const int head = w.head, ge = w.ti.row_end;
  int gs = a.cu_q[w.ti.group], n = a.cu_q[w.ti.group + 1] - gs;
  if (a.k_pieces > 1) piece_range(piece, a.k_pieces, gs, n);
  gs = __builtin_amdgcn_readfirstlane(gs);
  n = __builtin_amdgcn_readfirstlane(n);
  const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), lane = threadIdx.x & 63;
  const int row0 = w.ti.tile_row + DiffKeySweep::kKeys * wave;
  const int64_t head_q = (int64_t)head * a.Nq, head_k = (int64_t)head * a.Nk;
  const float lam = a.lambda[head];
  DiffKeySweep k;
#pragma unroll
  for (int c = 0; c < NC; ++c)
#pragma unroll
    for (int dt = 0; dt < 8; ++dt) k.dk[dt][c] = k.dv[dt][c] = floatx4_t{0.f, 0.f, 0.f, 0.f};
  if (n > 0) {
    k.tiles.start(lds.tiles, (const T*)a.q + (head_q + gs) * D, (const T*)a.d_o + (head_q + gs) * D, n, a.rows + head_q + gs);
    if (row0 >= ge) {   // no keys: this wave moves its share of the tiles and keeps the barriers
      for (int s = 0; s < (n + 31) >> 5; ++s) k.tiles.ready(s);
      k.tiles.finish();
      return;
    }
    diff_columns<T, D, NC>(k.kf, (const T*)a.k, row0, ge, head_k);
    {
      bf16x8_t vf[NC][4];
      diff_columns<T, D, NC>(vf, (const T*)a.v, row0, ge, head_k);
      k.keep_values(lds, vf);
    }
    settle(k.kf);
    k.c = a.scale * kLog2e;
    k.lam = lam;
    k.tiles.ready(0);
    k.sweep(n);
    k.tiles.finish();
  }
#pragma unroll
  for (int c = 0; c < NC; ++c) {
    const int row = row0 + 16 * c + (lane & 15);
    if (row >= ge) continue;
    auto store = [&](auto* d_k, auto* d_v) {
#pragma unroll
      for (int dt = 0; dt < 8; ++dt) {
        store4(d_k, dt, k.dk[dt][c] * (dt < 4 ? a.scale : lam * a.scale));
        store4(d_v, dt, k.dv[dt][c]);
      }
    };
    if (a.k_pieces > 1) {
      float* part = a.part_k + ((int64_t)piece * 2 * a.H * a.Nk + head_k + row) * D;
      store(part, part + (int64_t)a.H * a.Nk * D);
    } else {
      store((T*)a.d_k + (head_k + row) * D, (T*)a.d_v + (head_k + row) * D);
    }
  }
}

// fp32 dQ.
template <int D>
__global__ __launch_bounds__(256, 2) void diff_dq_f32_kernel(DiffBwd a) {
  __shared__ typename DiffTiles<float, D>::Lds lds;
  diff_dq_block<float, D>(a, blockIdx.x, blockIdx.y, lds);
}

// bf16, both: blocks of keys (first of their pieces, then the next), then blocks of queries, which fill the others' last rounds: 10,007 x 12
// heads, 20 unequal groups 227 us, 62,400 x 12, 8 groups 10.6 ms.
__global__ __launch_bounds__(256, 2) void diff_bwd_kernel(DiffBwd a, const int32_t* __restrict__ q_tiles, int q_blocks, int k_blocks) {
  __shared__ union {
    DiffTiles<unsigned short, kHeadDim>::Lds q;
    DiffKeySweep::Lds k;
  } lds;
  const int b = blockIdx.x, keys = k_blocks * a.k_pieces;
  if (b < keys) {
    diff_dkdv_block(a, b % k_blocks, b / k_blocks, lds.k);
  } else {
    a.tile_start = q_tiles;
    diff_dq_block<unsigned short, kHeadDim>(a, (b - keys) % q_blocks, (b - keys) / q_blocks, lds.q);
  }
}

// Sums of the pieces, four channels a thread: d_q and share (pq != 1), d_k and d_v (pk != 1; 0: zeros).  Rows behind the last group stay.
template <typename T, int D>
__global__ __launch_bounds__(256) void diff_sum_kernel(DiffBwd a, int pq, int pk) {
  constexpr int kEach = D / 4;
  const int64_t q_rows = pq == 1 ? 0 : a.H * a.Nq, k_rows = pk == 1 ? 0 : a.H * a.Nk;
  const int col = threadIdx.x % kEach * 4;
  int64_t row = (int64_t)blockIdx.x * (256 / kEach) + threadIdx.x / kEach;
  auto sum = [&](const float* part, int pieces, int64_t stride, T* out) {
    floatx4_t v = {0.f, 0.f, 0.f, 0.f};
    for (int p = 0; p < pieces; ++p) v += *(const floatx4_t*)(part + p * stride * D + col);
    if constexpr (sizeof(T) == 4) *(floatx4_t*)(out + col) = v;
    else *(uintx2_t*)(out + col) = pack4(v, 1.f);
  };
  if (row < q_rows) {
    if (row % a.Nq >= a.cu_q[a.G]) return;
    sum(a.part_q + row * D, pq, q_rows, (T*)a.d_q + row * D);
    if (sizeof(T) == 2 && col == 0) {
      float s = 0.f;
      for (int p = 0; p < pq; ++p) s += a.part_share[p * q_rows + row];
      a.share[row] = s;
    }
    return;
  }
  row -= q_rows;
  if (row >= 2 * k_rows || row % a.Nk >= a.cu_k[a.G]) return;
  T* out = (T*)(row < k_rows ? a.d_k : a.d_v) + (row < k_rows ? row : row - k_rows) * D;
  sum(a.part_k + row * D, pk, 2 * k_rows, out);
}

// A block per head, in a fixed order.
__global__ __launch_bounds__(1024) void diff_dlambda_kernel(const float* __restrict__ share, const int32_t* __restrict__ cu_q, int G, int64_t Nq,
                                                           float* __restrict__ d_lambda) {
  __shared__ float acc[16];
  const float* p = share + blockIdx.x * Nq;
  const int n = Nq > 0 ? cu_q[G] : 0;
  constexpr int U = 16;   // loads on their way
  float u[U];
#pragma unroll
  for (int k = 0; k < U; ++k) u[k] = 0.f;
  for (int i = threadIdx.x; i < n; i += U * 1024)
#pragma unroll
    for (int k = 0; k < U; ++k) u[k] += i + 1024 * k < n ? p[i + 1024 * k] : 0.f;
#pragma unroll
  for (int h = U / 2; h > 0; h /= 2)
#pragma unroll
    for (int k = 0; k < h; ++k) u[k] += u[k + h];
  float s = wave_sum(u[0]);
  if ((threadIdx.x & 63) == 0) acc[threadIdx.x >> 6] = s;
  __syncthreads();
  if (threadIdx.x < 64) {
    s = lanes_sum<16>(threadIdx.x < 16 ? acc[threadIdx.x] : 0.f);
    if (threadIdx.x == 0) d_lambda[blockIdx.x] = 0.f - s;
  }
}

int check_diff(int64_t Nq, int64_t Nk, int H, int D, int G, float scale, int dtype) {
  if (Nq < 0 || Nk < 0 || H < 1 || D < 1 || G < 1) return MOGA_ERR_INVALID_ARG;
  if (!(scale > 0.f) || !(scale < INFINITY)) return MOGA_ERR_INVALID_ARG;
  if (dtype != MOGA_F32 && dtype != MOGA_BF16) return MOGA_ERR_UNSUPPORTED;
  if (dtype == MOGA_BF16 ? D != 128 : D != 64 && D != 128) return MOGA_ERR_UNSUPPORTED;
  // row offsets inside a group are 32-bit byte offsets
  if (Nq >= ((int64_t)1 << 24) || Nk >= ((int64_t)1 << 24) || G > MOGA_MAX_SEGMENTS) return MOGA_ERR_UNSUPPORTED;
  return MOGA_OK;
}

int rows_of(int dtype) { return dtype == MOGA_F32 ? kRows<float> : kRows<unsigned short>; }
int key_rows_of(int dtype) { return dtype == MOGA_F32 ? kKeyRows<float> : kKeyRows<unsigned short>; }
int64_t diff_blocks(int64_t N, int H, int G, int rows) { return (max_tiles(N, G, rows) * H + 7) / 8 * 8; }
size_t tile_bytes(int G) { return G > MOGA_MAX_GROUPS ? round_up(((size_t)G + 1) * sizeof(int32_t), 256) : 0; }

// Pieces of the rows that a tile sweeps, where tiles of `rows` rows leave CUs idle.  bf16: as many as fill two blocks a CU, none under 256 rows of a
// mean group.  Whole and in pieces, forward: 1,000 x 3 heads 34 and 29 us, 4,096 x 3 101 and 72, 16,384 x 1 370 and 243, 16,384 x 1, 4 groups 100 and 89;
// backward 55 and 41, 161 and 135, 771 and 490, 212 and 157.  It loses where tiles of several groups leave few CUs idle: 4,096 x 3, 8 groups
// 24 and 31, backward 40 and 49 (in pieces of 128 rows a seventh more), 8,192 x 3, 4 groups 59 and 74, 124 and 133, 1,000 x 12 35 and 45, 58 and 70.
// fp32, whose steps take ten times as long: none under 64 rows, and as many as make the fullest CU's work least: its blocks (an XCD deals its
// share out to 32 CUs) times a block's steps and what starting it costs, in microseconds, and the traffic of the partial results.  One block a
// CU takes 1.6 times what it would beside two others, two 1.1.  Groups of unequal length have some more tiles: half the cost is that of 5 % more.
// Backward, whole and in pieces: 1,000 x 2 x 64 175 and 68 us, 256 x 2 x 128 94 and 45, 6,000 x 4 x 128, 8 groups 449 and 378, 4,096 x 2 x 128, 8 groups 169
// and 138; forward 73 and 34, 39 and 22, 174 and 154, 70 and 65, but 4,096 x 2 x 64, 8 groups 40.6 and 42.4.  Of sizes taken together: without the second
// half of the cost a step of 4,096 x 2 x 64 in unequal groups took 128 us and not 120, the backward of 4,096 x 2 x 128 in equal ones 121 and not 138.
int diff_pieces(int64_t N, int64_t other, int H, int G, int rows, int D, int dtype) {
  if (dtype != MOGA_F32) {
    const int64_t blocks = std::max<int64_t>(1, std::min<int64_t>(max_tiles(N, G, rows), N)) * H;
    return (int)std::max<int64_t>(1, std::min({(int64_t)16, 2 * kCus / blocks, other / G / 256}));
  }
  const int64_t tiles = (std::min(N, G * (((N + G - 1) / G + rows - 1) / rows)) * H + 7) / 8, most = std::min<int64_t>(16, other / G / 64);
  const double step = D * 0.02, start = 2 * step, traffic = (double)N * H * D * 16 / 6e6;
  auto fullest = [](double blocks) {   // of an XCD
    const double k = std::ceil(blocks / 32);
    return k <= 1 ? 1.6 : k == 2 ? 2.2 : k;
  };
  int best = 1;
  double least = INFINITY;
  for (int p = 1; p <= most && tiles * p <= kCus; ++p) {
    const double block = other / G / 32. / p * step + start;
    const double cost = 0.5 * (fullest(tiles * p) + fullest(1.05 * tiles * p)) * block + (p > 1 ? p * traffic : 0.);
    if (cost < least) least = cost, best = p;
  }
  return best;
}

size_t diff_piece_bytes(int64_t Nq, int H, int D) { return (size_t)Nq * H * 2 * (D + 2) * sizeof(float); }

// How a forward call shares out its keys.  chunk > 0: diff_few_kernel, pieces of `chunk` keys, at most `pieces` of a group; else pieces of every
// tile of queries (1: whole).
struct DiffSplit { int pieces, chunk; };
// The sizes of the groups are on the device, and all queries of a call may be one group's, which diff_few_kernel takes 16 at a time, with the keys
// read again each time: four times at most.  By the mean alone a call of one group of 6,001 queries beside 399 of one, 4,000 keys each, one head, took 13.3 ms
// against 0.18 by tiles, and one of 3,800 (with as many keys) beside 256 of one with 1,000, 12 heads, 8.3 against 0.45; with 64 queries at most 61
// beside three of one take 45 us against 23.  Where every group has as many, beyond 64 tiles take 0.46 to 1.06 of the time (12 heads, 24 groups of 16 queries and
// 300 keys 20 us against 44, 64 of 16 and 4,000 284 against 298, 32 of 4 and 4,000 171 against 167), 1.27 at worst (one head, 43 of 4 and 16,384).
constexpr int64_t kFewQueries = 64;
DiffSplit diff_split(int64_t Nq, int64_t Nk, int H, int D, int G, int dtype) {
  // Up to 16 queries a mean group the matrix products of a tile of 128 are idle work, and three of its waves too: pieces of keys for two rounds of
  // blocks, one a CU (or one round more than what the groups' last pieces make), none under 256 keys, and as many as 256 MB hold (one group
  // might have all the keys).  A group's last piece is half a piece on average.
  const int64_t most = (256 << 20) / (int64_t)diff_piece_bytes(Nq, H, D);
  if (dtype == MOGA_BF16 && Nq <= std::min(kFewQueries, 16 * (int64_t)G) && Nk / G >= 128 && most >= 1) {
    const int64_t ends = (int64_t)G * H / 2, rounds = std::max<int64_t>(2, (ends + 2 * kCus - 1) / kCus);
    const int64_t even = Nk * H / std::max<int64_t>(1, rounds * kCus * 49 / 50 - ends);
    const int64_t chunk = round_up((size_t)std::min(Nk, std::max({(int64_t)256, even, (Nk + most - 1) / most})), 128);
    return {(int)((Nk + chunk - 1) / chunk), (int)chunk};
  }
  return {diff_pieces(Nq, Nk, H, G, rows_of(dtype), D, dtype), 0};
}

struct DiffBwdSplit {
  int q, k;
  size_t q_bytes, share_bytes, k_bytes;
  size_t bytes() const { return q_bytes + share_bytes + k_bytes; }
};
DiffBwdSplit diff_bwd_split(int64_t Nq, int64_t Nk, int H, int D, int G, int dtype) {
  DiffBwdSplit s = {diff_pieces(Nq, Nk, H, G, rows_of(dtype), D, dtype), diff_pieces(Nk, Nq, H, G, key_rows_of(dtype), D, dtype), 0, 0, 0};
  if (s.q > 1) s.q_bytes = (size_t)s.q * H * Nq * D * sizeof(float), s.share_bytes = round_up((size_t)s.q * H * Nq * sizeof(float), 256);
  if (s.k > 1) s.k_bytes = (size_t)s.k * 2 * H * Nk * D * sizeof(float);
  return s;
}
}  // namespace
}  // namespace moga

using namespace moga;

extern "C" size_t moga_diff_attn_fwd_ws_bytes(int G) { return tile_bytes(G); }
// With the pieces of the keys, for calls of few tiles.
extern "C" size_t moga_diff_attn_fwd_preferred(int64_t Nq, int64_t Nk, int H, int D, int G, int dtype) {
  if (Nq <= 0 || check_diff(Nq, Nk, H, D, G, 1.f, dtype) != MOGA_OK) return 0;
  const DiffSplit s = diff_split(Nq, Nk, H, D, G, dtype);
  return tile_bytes(G) + (s.pieces > 1 || s.chunk ? s.pieces * diff_piece_bytes(Nq, H, D) : 0);
}
extern "C" size_t moga_diff_attn_bwd_ws_bytes(int64_t Nq, int H, int G) {
  return Nq > 0 ? tile_bytes(G) * 2 + round_up((size_t)Nq * H * (sizeof(floatx4_t) + sizeof(float)), 256) : 0;
}
extern "C" size_t moga_diff_attn_bwd_preferred(int64_t Nq, int64_t Nk, int H, int D, int G, int dtype) {
  if (Nq <= 0 || check_diff(Nq, Nk, H, D, G, 1.f, dtype) != MOGA_OK) return 0;
  return moga_diff_attn_bwd_ws_bytes(Nq, H, G) + diff_bwd_split(Nq, Nk, H, D, G, dtype).bytes();
}

extern "C" int moga_diff_attn_fwd(const void* qh, const void* kh, const void* vh, int dtype, int64_t Nq, int64_t Nk, int H, int D,
                                  const float* lambda, const int32_t* cu_seqlens_q, const int32_t* cu_seqlens_k, int G, float softmax_scale,
                                  void* oh, float* parts, float* lse, void* ws, size_t ws_bytes, void* stream) {
  const int bad = check_diff(Nq, Nk, H, D, G, softmax_scale, dtype);
  if (bad) return bad;
  if (Nq == 0) return MOGA_OK;
  if (!qh || !lambda || !cu_seqlens_q || !cu_seqlens_k || !oh || !lse || (Nk > 0 && (!kh || !vh))) return MOGA_ERR_INVALID_ARG;
  if (!(aligned16(qh) && aligned16(kh) && aligned16(vh) && aligned16(oh) && aligned16(parts) && aligned16(ws))) return MOGA_ERR_INVALID_ARG;
  const size_t need = moga_diff_attn_fwd_ws_bytes(G);
  if (need && (!ws || ws_bytes < need)) return MOGA_ERR_WORKSPACE;
  const bool room = ws && ws_bytes >= moga_diff_attn_fwd_preferred(Nq, Nk, H, D, G, dtype);
  const DiffSplit split = room ? diff_split(Nq, Nk, H, D, G, dtype) : DiffSplit{1, 0};
  const int pieces = split.pieces;
  const int64_t blocks = split.chunk ? diff_blocks(Nk, H, G, split.chunk) : diff_blocks(Nq, H, G, rows_of(dtype)), rows = Nq * H;
  if (!grid_fits(split.chunk ? blocks : blocks * pieces, 256) || !grid_fits((rows + 3) / 4, 256)) return MOGA_ERR_UNSUPPORTED;
  hipStream_t st = (hipStream_t)stream;
  int32_t* ts = G > MOGA_MAX_GROUPS ? (int32_t*)ws : nullptr;
  DiffFwd a = {qh, kh, vh, lambda, cu_seqlens_q, cu_seqlens_k, ts, Nq, Nk, H, G, softmax_scale, oh, parts, lse, nullptr, nullptr};
  if (pieces > 1 || split.chunk) {
    a.part = (float*)((char*)ws + tile_bytes(G));
    a.stat = a.part + (size_t)pieces * rows * 2 * D;
  }
  if (split.chunk) {
    if (ts) tile_start_kernel<<<1, 1024, 0, st>>>(cu_seqlens_k, G, split.chunk, ts);
    diff_few_kernel<<<(unsigned)blocks, 256, 0, st>>>(a, split.chunk);
    diff_merge_kernel<unsigned short, 128><<<(unsigned)((rows + 3) / 4), 256, 0, st>>>(a, pieces, split.chunk);
    return launch_status();
  }
  if (ts) tile_start_kernel<<<1, 1024, 0, st>>>(cu_seqlens_q, G, rows_of(dtype), ts);
  const dim3 grid((unsigned)blocks, (unsigned)pieces);
#define MOGA_DIFF_FWD(T, D)                                                          \
  do {                                                                               \
    if (pieces > 1) {                                                                \
      diff_fwd_kernel<T, D, true><<<grid, 256, 0, st>>>(a);                          \
      diff_merge_kernel<T, D><<<(unsigned)((rows + 3) / 4), 256, 0, st>>>(a, pieces, 0); \
    } else {                                                                         \
      diff_fwd_kernel<T, D, false><<<grid, 256, 0, st>>>(a);                         \
    }                                                                                \
  } while (0)
  if (dtype == MOGA_BF16) MOGA_DIFF_FWD(unsigned short, 128);
  else if (D == 64) MOGA_DIFF_FWD(float, 64);
  else MOGA_DIFF_FWD(float, 128);
#undef MOGA_DIFF_FWD
  return launch_status();
}

extern "C" int moga_diff_attn_bwd(const void* d_oh, const void* qh, const void* kh, const void* vh, const float* parts,
                                  const float* lse, int dtype, int64_t Nq, int64_t Nk, int H, int D, const float* lambda,
                                  const int32_t* cu_seqlens_q, const int32_t* cu_seqlens_k, int G, float softmax_scale, void* d_qh, void* d_kh,
                                  void* d_vh, float* d_lambda, void* ws, size_t ws_bytes, void* stream) {
  const int bad = check_diff(Nq, Nk, H, D, G, softmax_scale, dtype);
  if (bad) return bad;
  if (Nq == 0 && Nk == 0 && !d_lambda) return MOGA_OK;
  if (!lambda || !cu_seqlens_q || !cu_seqlens_k || !d_lambda) return MOGA_ERR_INVALID_ARG;
  if (Nq > 0 && (!d_oh || !qh || !parts || !lse || !d_qh)) return MOGA_ERR_INVALID_ARG;
  if (Nk > 0 && (!kh || !vh || !d_kh || !d_vh)) return MOGA_ERR_INVALID_ARG;
  if (!(aligned16(d_oh) && aligned16(qh) && aligned16(kh) && aligned16(vh) && aligned16(parts) && aligned16(d_qh) &&
        aligned16(d_kh) && aligned16(d_vh) && aligned16(ws)))
    return MOGA_ERR_INVALID_ARG;
  const size_t need = moga_diff_attn_bwd_ws_bytes(Nq, H, G);
  if (need && (!ws || ws_bytes < need)) return MOGA_ERR_WORKSPACE;
  const int64_t q_blocks = diff_blocks(Nq, H, G, rows_of(dtype)), k_blocks = Nk > 0 ? diff_blocks(Nk, H, G, key_rows_of(dtype)) : 0,
                rows = Nq * H;
  DiffBwdSplit split = {1, 1, 0, 0, 0};
  if (Nq > 0 && ws_bytes >= moga_diff_attn_bwd_preferred(Nq, Nk, H, D, G, dtype)) split = diff_bwd_split(Nq, Nk, H, D, G, dtype);
  if (Nq == 0) split.k = 0;   // keys without queries: zeros
  const int64_t sum_blocks = ((split.q != 1 ? rows : 0) + (split.k != 1 ? 2 * Nk * H : 0) + 1024 / D - 1) / (1024 / D);
  const int64_t joint = q_blocks * split.q + k_blocks * split.k;
  if (!grid_fits(joint, 256) || !grid_fits((rows + 15) / 16, 256) || !grid_fits(sum_blocks, 256))
    return MOGA_ERR_UNSUPPORTED;
  hipStream_t st = (hipStream_t)stream;
  int32_t *tq = nullptr, *tk = nullptr;
  if (G > MOGA_MAX_GROUPS && need) {
    tq = (int32_t*)ws;
    tk = (int32_t*)((char*)ws + tile_bytes(G));
    tile_start_kernel<<<1, 1024, 0, st>>>(cu_seqlens_q, G, rows_of(dtype), tq);
    tile_start_kernel<<<1, 1024, 0, st>>>(cu_seqlens_k, G, key_rows_of(dtype), tk);
  }
  floatx4_t* rc = (floatx4_t*)((char*)ws + 2 * tile_bytes(G));
  float* share = (float*)(rc + rows);
  DiffBwd a = {d_oh, qh, kh, vh, lambda, cu_seqlens_q, cu_seqlens_k, tq, rc, Nq, Nk, H, G, softmax_scale, d_qh, d_kh, d_vh, share, nullptr, nullptr, nullptr,
               split.q, split.k};
  if (split.q > 1 || split.k > 1) {
    char* room = (char*)ws + need;
    a.part_q = (float*)room;
    a.part_share = (float*)(room + split.q_bytes);
    a.part_k = (float*)(room + split.q_bytes + split.share_bytes);
  }
  DiffBwd b = a;
  b.tile_start = tk;
#define MOGA_DIFF_BWD(T, D)                                                                                                            \
  do {                                                                                                                                 \
    if (sizeof(T) == 2 && Nk <= kDeltaKeys * G) diff_delta_kernel<<<(unsigned)q_blocks, 256, 0, st>>>(a, lse, rc);                      \
    else diff_rows_kernel<T, D><<<(unsigned)((rows + 15) / 16), 256, 0, st>>>((const T*)d_oh, parts, lse, rows, rc, share);             \
    if constexpr (sizeof(T) == 4) {                                                                                                    \
      diff_dq_f32_kernel<D><<<dim3((unsigned)q_blocks, split.q), 256, 0, st>>>(a);                                                     \
      if (Nk > 0) diff_dkdv_f32_kernel<D><<<dim3((unsigned)k_blocks, split.k), 256, 0, st>>>(b);                                        \
    } else {                                                                                                                           \
      diff_bwd_kernel<<<(unsigned)joint, 256, 0, st>>>(b, tq, (int)q_blocks, (int)k_blocks);                                            \
    }                                                                                                                                  \
  } while (0)
  if (Nq > 0) {
    if (dtype == MOGA_BF16) MOGA_DIFF_BWD(unsigned short, 128);
    else if (D == 64) MOGA_DIFF_BWD(float, 64);
    else MOGA_DIFF_BWD(float, 128);
  }
  if (sum_blocks > 0) {
    if (dtype == MOGA_BF16) diff_sum_kernel<unsigned short, 128><<<(unsigned)sum_blocks, 256, 0, st>>>(a, split.q, split.k);
    else if (D == 64) diff_sum_kernel<float, 64><<<(unsigned)sum_blocks, 256, 0, st>>>(a, split.q, split.k);
    else diff_sum_kernel<float, 128><<<(unsigned)sum_blocks, 256, 0, st>>>(a, split.q, split.k);
  }
#undef MOGA_DIFF_BWD
  diff_dlambda_kernel<<<H, 1024, 0, st>>>(share, cu_seqlens_q, G, Nq, d_lambda);
  return launch_status();
}

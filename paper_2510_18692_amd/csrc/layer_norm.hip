// Layer norm over the last axis, forward and backward, with the gradient of weight and bias.
//
//   mu = mean x, rstd = 1 / sqrt(mean (x - mu)^2 + eps), xh = (x - mu) rstd, y = xh w + b
//   g = dy w, dx = rstd (g - mean g - xh mean(g xh)), dw = sum over rows of dy xh, db = sum over rows of dy
//
// Bound by HBM: a row is read once into registers, where both passes over it (mean, then centred squares) run, and written once, while the
// next row is on its way.  A row belongs to 16 lanes, a wave, or a block of as many waves as give a lane 16 columns or fewer (of 8 waves beyond
// 8,192): the weights, their two sums, x and dy of 16 columns leave room for three waves a SIMD.
#include <algorithm>
#include <cmath>

#include "moga_common.h"

namespace moga {
namespace {

constexpr int kNormMaxC = 16384;

// 16 bytes of T at T's own alignment: rows of odd length start anywhere, and the hardware loads them all the same.
template <typename T>
struct __attribute__((packed, aligned(sizeof(T)))) Bytes16 { unsigned w[4]; };

template <typename T> constexpr int kPer16 = 16 / (int)sizeof(T);

__device__ __forceinline__ void unpack(const Bytes16<float>& b, float (&f)[4]) {
#pragma unroll
  for (int i = 0; i < 4; ++i) f[i] = __uint_as_float(b.w[i]);
}
__device__ __forceinline__ void unpack(const Bytes16<unsigned short>& b, float (&f)[8]) {
#pragma unroll
  for (int i = 0; i < 4; ++i) {
    f[2 * i] = bf16_lo_to_f32(b.w[i]);
    f[2 * i + 1] = bf16_hi_to_f32(b.w[i]);
  }
}
__device__ __forceinline__ Bytes16<float> pack(const float (&f)[4]) {
  Bytes16<float> b;
#pragma unroll
  for (int i = 0; i < 4; ++i) b.w[i] = __float_as_uint(f[i]);
  return b;
}
__device__ __forceinline__ Bytes16<unsigned short> pack(const float (&f)[8]) {   // to nearest even
  Bytes16<unsigned short> b;
#pragma unroll
  for (int i = 0; i < 4; ++i) b.w[i] = pack_bf16x2(f[2 * i], f[2 * i + 1]);
  return b;
}
__device__ __forceinline__ float to_f32(float v) { return v; }
__device__ __forceinline__ float to_f32(unsigned short v) { return bf16_bits_to_f32(v); }
__device__ __forceinline__ void from_f32(float& d, float v) { d = v; }
__device__ __forceinline__ void from_f32(unsigned short& d, float v) { d = f32_to_bf16_bits(v); }

// Columns col .. col + V - 1 of a row of C, as they lie there, with the next row's first ones past its end (clear_past); zeros past the last row's.
// Element by element, in every row's last piece, the loads would be waited for where they are issued: 4,099 x 1535 backward (a call of two
// launches) bf16 44 us instead of 32, fp32 31 instead of 28.
template <typename T>
__device__ __forceinline__ Bytes16<T> load_part(const T* __restrict__ row, int col, int C, bool last_row) {
  constexpr int V = kPer16<T>;
  if (col + V <= C || (col < C && C >= V && !last_row)) return *(const Bytes16<T>*)(row + col);
  float f[V];
#pragma unroll
  for (int i = 0; i < V; ++i) f[i] = col + i < C ? to_f32(row[col + i]) : 0.f;
  return pack(f);   // exact: values of T
}
template <int V>
__device__ __forceinline__ void clear_past(float (&f)[V], int col, int C) {
  if (col + V > C)
#pragma unroll
    for (int i = 0; i < V; ++i)
      if (col + i >= C) f[i] = 0.f;
}
template <typename T, int V>
__device__ __forceinline__ void store_part(T* __restrict__ row, int col, int C, const float (&f)[V]) {
  if (col + V <= C) {
    *(Bytes16<T>*)(row + col) = pack(f);
  } else {
#pragma unroll
    for (int i = 0; i < V; ++i)
      if (col + i < C) from_f32(row[col + i], f[i]);
  }
}
// fp32 weights of the same columns; `other` where there are none.
template <int V>
__device__ __forceinline__ void load_weights(const float* __restrict__ w, int col, int C, float other, float (&f)[V]) {
  if (w && col + V <= C) {
#pragma unroll
    for (int i = 0; i < V; i += 4) {
      const Bytes16<float> b = *(const Bytes16<float>*)(w + col + i);
#pragma unroll
      for (int e = 0; e < 4; ++e) f[i + e] = __uint_as_float(b.w[e]);
    }
  } else {
#pragma unroll
    for (int i = 0; i < V; ++i) f[i] = w && col + i < C ? w[col + i] : other;
  }
}

// How the rows are dealt out: LANES = 16 or 64 to a row, four waves a block; LANES = 0: a row to a block of any number of waves.
template <int LANES>
struct Deal {
  int lanes, lane;   // of the row
  int64_t row, step;
  __device__ __forceinline__ Deal() {
    lanes = LANES ? LANES : blockDim.x;
    lane = LANES ? threadIdx.x % LANES : threadIdx.x;
    const int rows = LANES ? 256 / LANES : 1;
    row = (int64_t)blockIdx.x * rows + (LANES ? threadIdx.x / LANES : 0);
    step = (int64_t)gridDim.x * rows;
  }
};

// Sums over the lanes of a row.  A row of a whole block goes through LDS: one barrier a sum, two buffers in turn.
constexpr int kMaxWaves = 8;
template <int LANES, int K>
struct RowSum {
  float (*lds)[kMaxWaves][K];   // [2][waves][K]
  int turn = 0;
  __device__ __forceinline__ void operator()(float (&v)[K]) {
#pragma unroll
    for (int k = 0; k < K; ++k) v[k] = lanes_sum<(LANES ? LANES : 64)>(v[k]);
    if constexpr (LANES == 0) {
      if ((threadIdx.x & 63) == 0)
#pragma unroll
        for (int k = 0; k < K; ++k) lds[turn][threadIdx.x >> 6][k] = v[k];
      __syncthreads();
      const int waves = blockDim.x >> 6, lane = threadIdx.x & 15;
#pragma unroll
      for (int k = 0; k < K; ++k) v[k] = lanes_sum<16>(lane < waves ? lds[turn][lane & (kMaxWaves - 1)][k] : 0.f);
      turn ^= 1;
    }
  }
};

// PARTS loads per lane; lane t holds the columns (part * lanes + t) * V ..
template <typename T, int LANES, int PARTS>
__global__ __launch_bounds__(LANES ? 256 : 64 * kMaxWaves) void layer_norm_fwd_kernel(const T* __restrict__ x, const float* __restrict__ w,
                                                                            const float* __restrict__ b, int64_t N, int C, float eps,
                                                                            T* __restrict__ y, float* __restrict__ mean,
                                                                            float* __restrict__ rstd) {
  constexpr int V = kPer16<T>;
  __shared__ float lds[2][kMaxWaves][1];
  RowSum<LANES, 1> sum{lds};
  Deal<LANES> d;
  int col[PARTS];
  Bytes16<T> next[PARTS];
  float wf[PARTS][V], bf[PARTS][V];
#pragma unroll
  for (int p = 0; p < PARTS; ++p) {
    col[p] = (p * d.lanes + d.lane) * V;
    if (d.row < N) next[p] = load_part(x + d.row * C, col[p], C, d.row + 1 == N);
  }
#pragma unroll
  for (int p = 0; p < PARTS; ++p) {
    load_weights(w, col[p], C, 1.f, wf[p]);
    load_weights(b, col[p], C, 0.f, bf[p]);
  }
  const float n = (float)C;   // divided by: the mean of equal values is their value
  for (; d.row < N; d.row += d.step) {
    float f[PARTS][V];
    float s[1] = {0.f};
#pragma unroll
    for (int p = 0; p < PARTS; ++p) {
      unpack(next[p], f[p]);
      clear_past(f[p], col[p], C);
    }
    if (d.row + d.step < N)
#pragma unroll
      for (int p = 0; p < PARTS; ++p) next[p] = load_part(x + (d.row + d.step) * C, col[p], C, d.row + d.step + 1 == N);
#pragma unroll
    for (int p = 0; p < PARTS; ++p)
#pragma unroll
      for (int i = 0; i < V; ++i) s[0] += f[p][i];
    sum(s);
    const float mu = s[0] / n;
    s[0] = 0.f;
#pragma unroll
    for (int p = 0; p < PARTS; ++p)
#pragma unroll
      for (int i = 0; i < V; ++i) {
        f[p][i] = col[p] + i < C ? f[p][i] - mu : 0.f;
        s[0] = fmaf(f[p][i], f[p][i], s[0]);
      }
    sum(s);
    const float r = 1.f / sqrtf(s[0] / n + eps);
#pragma unroll
    for (int p = 0; p < PARTS; ++p) {
#pragma unroll
      for (int i = 0; i < V; ++i) f[p][i] = fmaf(f[p][i] * r, wf[p][i], bf[p][i]);
      store_part(y + d.row * C, col[p], C, f[p]);
    }
    if (mean && d.lane == 0) {
      mean[d.row] = mu;
      rstd[d.row] = r;
    }
  }
}

// dx, and this block's share of dw and db at part[block][2][C] (DW).  The shares of the rows that run beside each other in a block are
// added in a fixed order, and so are the blocks': results repeat bit by bit.
template <typename T, int LANES, int PARTS, bool DW>
__global__ __launch_bounds__(LANES ? 256 : 64 * kMaxWaves) void layer_norm_bwd_kernel(const T* __restrict__ dy, const T* __restrict__ x,
                                                                            const float* __restrict__ w, const float* __restrict__ mean,
                                                                            const float* __restrict__ rstd, int64_t N, int C,
                                                                            T* __restrict__ dx, float* __restrict__ part) {
#pragma clang fp contract(off)   // g is one value in its mean and in what the mean is taken from
  constexpr int V = kPer16<T>;
  __shared__ float lds[2][kMaxWaves][2];
  RowSum<LANES, 2> sum{lds};
  Deal<LANES> d;
  int col[PARTS];
  Bytes16<T> next_x[PARTS], next_g[PARTS];
  float next_mu = 0.f, next_r = 0.f;
  auto fetch = [&](int64_t row) {
#pragma unroll
    for (int p = 0; p < PARTS; ++p) {
      next_x[p] = load_part(x + row * C, col[p], C, row + 1 == N);
      next_g[p] = load_part(dy + row * C, col[p], C, row + 1 == N);
    }
    next_mu = mean[row];
    next_r = rstd[row];
  };
#pragma unroll
  for (int p = 0; p < PARTS; ++p) col[p] = (p * d.lanes + d.lane) * V;
  if (d.row < N) fetch(d.row);
  float wf[PARTS][V], dw[PARTS][V], db[PARTS][V];
#pragma unroll
  for (int p = 0; p < PARTS; ++p) {
    load_weights(w, col[p], C, 1.f, wf[p]);
#pragma unroll
    for (int i = 0; i < V; ++i) dw[p][i] = db[p][i] = 0.f;
  }
  const float n = (float)C;
  for (; d.row < N; d.row += d.step) {
    float f[PARTS][V], g[PARTS][V];
#pragma unroll
    for (int p = 0; p < PARTS; ++p) {
      unpack(next_x[p], f[p]);
      unpack(next_g[p], g[p]);
      clear_past(f[p], col[p], C);
      clear_past(g[p], col[p], C);
    }
    const float mu = next_mu, r = next_r;
    if (d.row + d.step < N) fetch(d.row + d.step);
    float s[2] = {0.f, 0.f};
#pragma unroll
    for (int p = 0; p < PARTS; ++p)
#pragma unroll
      for (int i = 0; i < V; ++i) {
        f[p][i] = (f[p][i] - mu) * r;   // past the row's end g is 0
        if constexpr (DW) {
          dw[p][i] = fmaf(g[p][i], f[p][i], dw[p][i]);
          db[p][i] += g[p][i];
        }
        g[p][i] *= wf[p][i];
        s[0] += g[p][i];
        s[1] = fmaf(g[p][i], f[p][i], s[1]);
      }
    sum(s);
    const float m0 = s[0] / n, m1 = s[1] / n;
#pragma unroll
    for (int p = 0; p < PARTS; ++p) {
#pragma unroll
      for (int i = 0; i < V; ++i) f[p][i] = r * (g[p][i] - m0 - f[p][i] * m1);
      store_part(dx + d.row * C, col[p], C, f[p]);
    }
  }
  if constexpr (DW) {
    float* out = part + (size_t)blockIdx.x * 2 * C;
    if constexpr (LANES == 0) {
#pragma unroll
      for (int p = 0; p < PARTS; ++p)
#pragma unroll
        for (int i = 0; i < V; ++i)
          if (col[p] + i < C) {
            out[col[p] + i] = dw[p][i];
            out[C + col[p] + i] = db[p][i];
          }
    } else {
      __shared__ float acc[2][LANES * PARTS * V];
      const int wave = threadIdx.x >> 6;
      if constexpr (LANES == 16) {   // the four rows of a wave
#pragma unroll
        for (int p = 0; p < PARTS; ++p)
#pragma unroll
          for (int i = 0; i < V; ++i) {
            dw[p][i] = __int_as_float(combine_xor<32>(combine_xor<16>(__float_as_int(dw[p][i]), AddF{}), AddF{}));
            db[p][i] = __int_as_float(combine_xor<32>(combine_xor<16>(__float_as_int(db[p][i]), AddF{}), AddF{}));
          }
      }
      for (int k = 0; k < 4; ++k) {
        if (wave == k && (threadIdx.x & 63) < LANES) {
#pragma unroll
          for (int p = 0; p < PARTS; ++p)
#pragma unroll
            for (int i = 0; i < V; ++i) {
              acc[0][col[p] + i] = k == 0 ? dw[p][i] : acc[0][col[p] + i] + dw[p][i];
              acc[1][col[p] + i] = k == 0 ? db[p][i] : acc[1][col[p] + i] + db[p][i];
            }
        }
        __syncthreads();
      }
      for (int c = threadIdx.x; c < C; c += 256) {
        out[c] = acc[0][c];
        out[C + c] = acc[1][c];
      }
    }
  }
}

// Sum over the blocks: 16 columns a block, whose 16 threads each take every 16th share.
__global__ __launch_bounds__(256) void layer_norm_dw_kernel(const float* __restrict__ part, int blocks, int C, float* __restrict__ dw,
                                                            float* __restrict__ db) {
  __shared__ float acc[16][17];
  const int c = threadIdx.x & 15, k = threadIdx.x >> 4;
  const int64_t col = (int64_t)blockIdx.x * 16 + c;
  constexpr int U = 16;   // loads on their way
  float s[U];
#pragma unroll
  for (int u = 0; u < U; ++u) s[u] = 0.f;
  if (col < 2 * C) {
    for (int b = k; b < blocks; b += 16 * U)
#pragma unroll
      for (int u = 0; u < U; ++u) s[u] += b + 16 * u < blocks ? part[(size_t)(b + 16 * u) * 2 * C + col] : 0.f;
  }
#pragma unroll
  for (int h = U / 2; h > 0; h /= 2)
#pragma unroll
    for (int u = 0; u < h; ++u) s[u] += s[u + h];
  acc[k][c] = s[0];
  __syncthreads();
  if (k == 0 && col < 2 * C) {
    float t = 0.f;
#pragma unroll
    for (int j = 0; j < 16; ++j) t += acc[j][c];
    if (col < C) {
      if (dw) dw[col] = t;
    } else if (db) {
      db[col - C] = t;
    }
  }
}

// 16 columns a lane at most: a row goes to 16 lanes up to 256 columns, to a wave up to 1,024, else to a block of a wave per 1,024; beyond 8,192
// columns to 8 waves, which have registers for 32 a lane.
struct NormShape {
  int lanes, parts, waves, rows;   // lanes of a row (0: the block), loads a lane; waves and rows of a block
};
NormShape norm_shape(int C, int dtype) {
  const int v = dtype == MOGA_F32 ? 4 : 8, waves = std::min(kMaxWaves, (C + 1023) / 1024);
  auto parts = [&](int lanes) { return (C + lanes * v - 1) / (lanes * v); };
  if (C <= 256) return {16, parts(16), 4, 16};
  if (C <= 1024) return {64, parts(64), 4, 4};
  return {0, parts(64 * waves), waves, 1};
}
// Blocks for rows_each rows a lane group, up to what fills the chip `fill` waves deep a CU.
int64_t norm_blocks(int64_t N, int C, int dtype, int64_t rows_each, int fill) {
  const NormShape s = norm_shape(C, dtype);
  return std::max<int64_t>(1, std::min<int64_t>(256 * std::max(1, fill / s.waves), (N + s.rows * rows_each - 1) / (s.rows * rows_each)));
}
int64_t norm_bwd_blocks(int64_t N, int C, int dtype) { return norm_blocks(N, C, dtype, 8, 16); }

// f(lanes, parts) with both as constants.
template <typename T, typename F>
void with_shape(const NormShape& s, F&& f) {
#define MOGA_SHAPE(L, P) f(std::integral_constant<int, L>{}, std::integral_constant<int, P>{})
#define MOGA_SHAPES(L)                                        \
  do {                                                        \
    if (s.parts == 1) MOGA_SHAPE(L, 1);                       \
    else if (s.parts == 2) MOGA_SHAPE(L, 2);                  \
    else if constexpr (L == 0 || sizeof(T) == 4) {            \
      if (s.parts == 3) MOGA_SHAPE(L, 3);                     \
      else if (s.parts == 4) MOGA_SHAPE(L, 4);                \
      else if constexpr (L == 0 && sizeof(T) == 4) {          \
        if (s.parts <= 6) MOGA_SHAPE(L, 6);                   \
        else MOGA_SHAPE(L, 8);                                \
      }                                                       \
    }                                                         \
  } while (0)
  if (s.lanes == 16) MOGA_SHAPES(16);
  else if (s.lanes == 64) MOGA_SHAPES(64);
  else MOGA_SHAPES(0);
#undef MOGA_SHAPES
#undef MOGA_SHAPE
}

int check_norm(int64_t N, int C, int dtype) {
  if (N < 0 || C < 1) return MOGA_ERR_INVALID_ARG;
  if (dtype != MOGA_F32 && dtype != MOGA_BF16) return MOGA_ERR_UNSUPPORTED;
  if (C > kNormMaxC || N >= ((int64_t)1 << 31)) return MOGA_ERR_UNSUPPORTED;
  return MOGA_OK;
}

template <typename T>
void launch_fwd(const void* x, const float* w, const float* b, int64_t N, int C, float eps, void* y, float* mean, float* rstd, int dtype,
                hipStream_t st) {
  const NormShape s = norm_shape(C, dtype);
  const unsigned blocks = (unsigned)norm_blocks(N, C, dtype, 1, 32);
  with_shape<T>(s, [&](auto lanes, auto parts) {
    layer_norm_fwd_kernel<T, lanes.value, parts.value><<<blocks, 64 * s.waves, 0, st>>>((const T*)x, w, b, N, C, eps, (T*)y, mean, rstd);
  });
}

template <typename T>
void launch_bwd(const void* dy, const void* x, const float* w, const float* mean, const float* rstd, int64_t N, int C, void* dx, float* part,
                int dtype, unsigned blocks, hipStream_t st) {
  const NormShape s = norm_shape(C, dtype);
  with_shape<T>(s, [&](auto lanes, auto parts) {
    if (part)
      layer_norm_bwd_kernel<T, lanes.value, parts.value, true><<<blocks, 64 * s.waves, 0, st>>>((const T*)dy, (const T*)x, w, mean, rstd, N, C,
                                                                                                (T*)dx, part);
    else
      layer_norm_bwd_kernel<T, lanes.value, parts.value, false><<<blocks, 64 * s.waves, 0, st>>>((const T*)dy, (const T*)x, w, mean, rstd, N, C,
                                                                                                 (T*)dx, part);
  });
}

}  // namespace
}  // namespace moga

using namespace moga;

extern "C" size_t moga_layer_norm_bwd_ws_bytes(int64_t N, int C, int dtype) {
  return check_norm(N, C, dtype) == MOGA_OK ? (size_t)norm_bwd_blocks(N, C, dtype) * 2 * C * sizeof(float) : 0;
}

extern "C" int moga_layer_norm_fwd(const void* x, int dtype, const float* weight, const float* bias, int64_t N, int C, float eps, void* y,
                                   float* mean, float* rstd, void* stream) {
  const int bad = check_norm(N, C, dtype);
  if (bad) return bad;
  if (!(eps >= 0.f) || !(eps < INFINITY)) return MOGA_ERR_INVALID_ARG;
  if (N == 0) return MOGA_OK;
  if (!x || !y || !mean != !rstd) return MOGA_ERR_INVALID_ARG;
  if (!(aligned16(x) && aligned16(y) && aligned16(weight) && aligned16(bias))) return MOGA_ERR_INVALID_ARG;
  if (dtype == MOGA_F32) launch_fwd<float>(x, weight, bias, N, C, eps, y, mean, rstd, dtype, (hipStream_t)stream);
  else launch_fwd<unsigned short>(x, weight, bias, N, C, eps, y, mean, rstd, dtype, (hipStream_t)stream);
  return launch_status();
}

extern "C" int moga_layer_norm_bwd(const void* d_y, const void* x, int dtype, const float* weight, const float* mean, const float* rstd,
                                   int64_t N, int C, void* d_x, float* d_weight, float* d_bias, void* ws, size_t ws_bytes, void* stream) {
  const int bad = check_norm(N, C, dtype);
  if (bad) return bad;
  hipStream_t st = (hipStream_t)stream;
  const bool dw = d_weight || d_bias;
  unsigned blocks = 0;
  if (N == 0 && !dw) return MOGA_OK;
  if (N > 0) {
    if (!d_y || !x || !mean || !rstd || !d_x) return MOGA_ERR_INVALID_ARG;
    if (!(aligned16(d_y) && aligned16(x) && aligned16(weight) && aligned16(d_x) && aligned16(d_weight) && aligned16(d_bias) && aligned16(ws)))
      return MOGA_ERR_INVALID_ARG;
    if (dw && (!ws || ws_bytes < moga_layer_norm_bwd_ws_bytes(N, C, dtype))) return MOGA_ERR_WORKSPACE;
    blocks = (unsigned)norm_bwd_blocks(N, C, dtype);
    float* part = dw ? (float*)ws : nullptr;
    if (dtype == MOGA_F32) launch_bwd<float>(d_y, x, weight, mean, rstd, N, C, d_x, part, dtype, blocks, st);
    else launch_bwd<unsigned short>(d_y, x, weight, mean, rstd, N, C, d_x, part, dtype, blocks, st);
  }
  // of no rows: zeros
  if (dw) layer_norm_dw_kernel<<<(2 * C + 15) / 16, 256, 0, st>>>((const float*)ws, (int)blocks, C, d_weight, d_bias);
  return launch_status();
}

// Layer norm over the last axis, forward and backward, with the gradient of weight and bias.
//
//   mu = mean x, rstd = 1 / sqrt(mean (x - mu)^2 + eps), xh = (x - mu) rstd, y = xh w + b
//   g = dy w, dx = rstd (g - mean g - xh mean(g xh)), dw = sum over rows of dy xh, db = sum over rows of dy
//
// Bound by HBM: a row is read once into registers, where both passes over it (mean, then centred squares) run, and written once.
// A row belongs to 16 lanes, a wave or a block, so that a lane holds at most eight loads of 16 bytes.
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

// Columns col .. col + V - 1 of a row of C; zeros past its end.
template <typename T, int V>
__device__ __forceinline__ void load_part(const T* __restrict__ row, int col, int C, float (&f)[V]) {
  if (col + V <= C) {
    unpack(*(const Bytes16<T>*)(row + col), f);
  } else {
#pragma unroll
    for (int i = 0; i < V; ++i) f[i] = col + i < C ? to_f32(row[col + i]) : 0.f;
  }
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
#pragma unroll
  for (int i = 0; i < V; ++i) f[i] = w && col + i < C ? w[col + i] : other;
}

// Sums over the lanes of a row.  A row of a whole block goes through LDS: one barrier a sum, two buffers in turn.
template <int LANES, int K>
struct RowSum {
  float (*lds)[4][K];   // [2][4 waves][K]
  int turn = 0;
  __device__ __forceinline__ void operator()(float (&v)[K]) {
#pragma unroll
    for (int k = 0; k < K; ++k) v[k] = lanes_sum<(LANES < 64 ? LANES : 64)>(v[k]);
    if constexpr (LANES > 64) {
      if ((threadIdx.x & 63) == 0)
#pragma unroll
        for (int k = 0; k < K; ++k) lds[turn][threadIdx.x >> 6][k] = v[k];
      __syncthreads();
#pragma unroll
      for (int k = 0; k < K; ++k) v[k] = (lds[turn][0][k] + lds[turn][1][k]) + (lds[turn][2][k] + lds[turn][3][k]);
      turn ^= 1;
    }
  }
};

// LANES per row, PARTS loads per lane; lane t holds the columns (part * LANES + t) * V ..
template <typename T, int LANES, int PARTS>
__global__ __launch_bounds__(256) void layer_norm_fwd_kernel(const T* __restrict__ x, const float* __restrict__ w, const float* __restrict__ b,
                                                             int64_t N, int C, float eps, T* __restrict__ y, float* __restrict__ mean,
                                                             float* __restrict__ rstd) {
  constexpr int V = kPer16<T>, ROWS = 256 / LANES;
  __shared__ float lds[2][4][1];
  RowSum<LANES, 1> sum{lds};
  const int t = threadIdx.x % LANES;
  float wf[PARTS][V], bf[PARTS][V];
#pragma unroll
  for (int p = 0; p < PARTS; ++p) {
    load_weights(w, (p * LANES + t) * V, C, 1.f, wf[p]);
    load_weights(b, (p * LANES + t) * V, C, 0.f, bf[p]);
  }
  const float n = (float)C;   // divided by: the mean of equal values is their value
  for (int64_t row = (int64_t)blockIdx.x * ROWS + threadIdx.x / LANES; row < N; row += (int64_t)gridDim.x * ROWS) {
    float f[PARTS][V];
    float s[1] = {0.f};
#pragma unroll
    for (int p = 0; p < PARTS; ++p) load_part(x + row * C, (p * LANES + t) * V, C, f[p]);
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
        f[p][i] = (p * LANES + t) * V + i < C ? f[p][i] - mu : 0.f;
        s[0] = fmaf(f[p][i], f[p][i], s[0]);
      }
    sum(s);
    const float r = 1.f / sqrtf(s[0] / n + eps);
#pragma unroll
    for (int p = 0; p < PARTS; ++p) {
#pragma unroll
      for (int i = 0; i < V; ++i) f[p][i] = fmaf(f[p][i] * r, wf[p][i], bf[p][i]);
      store_part(y + row * C, (p * LANES + t) * V, C, f[p]);
    }
    if (mean && t == 0) {
      mean[row] = mu;
      rstd[row] = r;
    }
  }
}

// dx, and this block's share of dw and db at part[block][2][C] (DW).  The shares of the rows that run beside each other in a block are
// added in a fixed order, and so are the blocks': results repeat bit by bit.
template <typename T, int LANES, int PARTS, bool DW>
__global__ __launch_bounds__(256) void layer_norm_bwd_kernel(const T* __restrict__ dy, const T* __restrict__ x, const float* __restrict__ w,
                                                             const float* __restrict__ mean, const float* __restrict__ rstd, int64_t N, int C,
                                                             T* __restrict__ dx, float* __restrict__ part) {
#pragma clang fp contract(off)   // g is one value in its mean and in what the mean is taken from
  constexpr int V = kPer16<T>, ROWS = 256 / LANES;
  __shared__ float lds[2][4][2];
  RowSum<LANES, 2> sum{lds};
  const int t = threadIdx.x % LANES;
  float wf[PARTS][V], dw[PARTS][V], db[PARTS][V];
#pragma unroll
  for (int p = 0; p < PARTS; ++p) {
    load_weights(w, (p * LANES + t) * V, C, 1.f, wf[p]);
#pragma unroll
    for (int i = 0; i < V; ++i) dw[p][i] = db[p][i] = 0.f;
  }
  const float n = (float)C;
  for (int64_t row = (int64_t)blockIdx.x * ROWS + threadIdx.x / LANES; row < N; row += (int64_t)gridDim.x * ROWS) {
    float f[PARTS][V], g[PARTS][V];
#pragma unroll
    for (int p = 0; p < PARTS; ++p) {
      load_part(x + row * C, (p * LANES + t) * V, C, f[p]);
      load_part(dy + row * C, (p * LANES + t) * V, C, g[p]);
    }
    const float mu = mean[row], r = rstd[row];
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
      store_part(dx + row * C, (p * LANES + t) * V, C, f[p]);
    }
  }
  if constexpr (DW) {
    float* out = part + (size_t)blockIdx.x * 2 * C;
    if constexpr (LANES == 256) {
#pragma unroll
      for (int p = 0; p < PARTS; ++p)
#pragma unroll
        for (int i = 0; i < V; ++i) {
          const int col = (p * LANES + t) * V + i;
          if (col < C) {
            out[col] = dw[p][i];
            out[C + col] = db[p][i];
          }
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
              const int col = (p * LANES + t) * V + i;
              acc[0][col] = k == 0 ? dw[p][i] : acc[0][col] + dw[p][i];
              acc[1][col] = k == 0 ? db[p][i] : acc[1][col] + db[p][i];
            }
        }
        __syncthreads();
      }
      for (int col = threadIdx.x; col < C; col += 256) {
        out[col] = acc[0][col];
        out[C + col] = acc[1][col];
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
  float s[4] = {0.f, 0.f, 0.f, 0.f};
  if (col < 2 * C) {
    int b = k;
    for (; b + 48 < blocks; b += 64)
#pragma unroll
      for (int u = 0; u < 4; ++u) s[u] += part[(size_t)(b + 16 * u) * 2 * C + col];
    for (; b < blocks; b += 16) s[0] += part[(size_t)b * 2 * C + col];
  }
  acc[k][c] = (s[0] + s[1]) + (s[2] + s[3]);
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

// Lanes per row: 16 up to two loads a lane, a wave up to four, else a block.
int norm_lanes(int C, int dtype) {
  const int v = dtype == MOGA_F32 ? 4 : 8;
  return C <= 2 * 16 * v ? 16 : C <= 4 * 64 * v ? 64 : 256;
}
int64_t norm_blocks(int64_t N, int C, int dtype, int64_t rows_each, int64_t most) {
  const int64_t rows = 256 / norm_lanes(C, dtype);
  return std::max<int64_t>(1, std::min(most, (N + rows * rows_each - 1) / (rows * rows_each)));
}
int64_t norm_bwd_blocks(int64_t N, int C, int dtype) { return norm_blocks(N, C, dtype, 8, 1024); }

// f(lanes, parts) with both as constants.
template <typename T, typename F>
void with_shape(int C, int dtype, F&& f) {
  const int lanes = norm_lanes(C, dtype), per = lanes * kPer16<T>, parts = (C + per - 1) / per;
#define MOGA_SHAPE(L, P) f(std::integral_constant<int, L>{}, std::integral_constant<int, P>{})
  if (lanes == 16) {
    if (parts == 1) MOGA_SHAPE(16, 1);
    else MOGA_SHAPE(16, 2);
  } else if (lanes == 64) {
    if (parts == 1) MOGA_SHAPE(64, 1);
    else if (parts == 2) MOGA_SHAPE(64, 2);
    else if (parts == 3) MOGA_SHAPE(64, 3);
    else MOGA_SHAPE(64, 4);
  } else {
    if (parts <= 2) MOGA_SHAPE(256, 2);
    else if (parts == 3) MOGA_SHAPE(256, 3);
    else if (parts == 4) MOGA_SHAPE(256, 4);
    else if (parts <= 6) MOGA_SHAPE(256, 6);
    else if (parts <= 8) MOGA_SHAPE(256, 8);
    else if constexpr (sizeof(T) == 4) {
      if (parts <= 12) MOGA_SHAPE(256, 12);
      else MOGA_SHAPE(256, 16);
    }
  }
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
  const unsigned blocks = (unsigned)norm_blocks(N, C, dtype, 1, 2048);
  with_shape<T>(C, dtype, [&](auto lanes, auto parts) {
    layer_norm_fwd_kernel<T, lanes.value, parts.value><<<blocks, 256, 0, st>>>((const T*)x, w, b, N, C, eps, (T*)y, mean, rstd);
  });
}

template <typename T>
void launch_bwd(const void* dy, const void* x, const float* w, const float* mean, const float* rstd, int64_t N, int C, void* dx, float* part,
                int dtype, unsigned blocks, hipStream_t st) {
  with_shape<T>(C, dtype, [&](auto lanes, auto parts) {
    if (part)
      layer_norm_bwd_kernel<T, lanes.value, parts.value, true><<<blocks, 256, 0, st>>>((const T*)dy, (const T*)x, w, mean, rstd, N, C, (T*)dx, part);
    else
      layer_norm_bwd_kernel<T, lanes.value, parts.value, false><<<blocks, 256, 0, st>>>((const T*)dy, (const T*)x, w, mean, rstd, N, C, (T*)dx, part);
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

// Rows of a norm: pieces of 16 bytes at any element's alignment, how rows are dealt out to lanes, and sums over the lanes of a row.
#pragma once

#include "moga_common.h"

namespace moga {

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
template <int LANES, int K, int WAVES = kMaxWaves>
struct RowSum {
  float (*lds)[WAVES][K];   // [2][waves][K]
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
      for (int k = 0; k < K; ++k) v[k] = lanes_sum<16>(lane < waves ? lds[turn][min(lane, WAVES - 1)][k] : 0.f);
      turn ^= 1;
    }
  }
};

}  // namespace moga

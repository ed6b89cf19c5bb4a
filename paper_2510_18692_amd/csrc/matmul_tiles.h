// Tiles of matrix products C[M][N] = sum_k A(m, k) B(n, k), the operands as they lie in memory.
//
// A block owns BM x BN of C and walks K in steps of 128 bytes of an operand's row (64 bf16, 32 fp32).  Either operand lies with k last ("rows":
// an activation, or a weight as it is) or with k first ("columns": the same tensor as the operand of its gradient, without a transposed copy).
// Both are staged global -> LDS by direct loads, 16 bytes a lane, two steps in turn, and read back as MFMA operands: rows with 16-byte reads, bf16
// columns with transposed 8-byte reads, fp32 columns with 4-byte reads.  Chunks of a staged row are exchanged (xor) so that the lanes of a read fall
// on different banks; the exchange is made in the global addresses, since a direct load fills LDS in lane order.
// Rows, columns and k past the operand's end are read as zeros: their buffer offset is put past the buffer's range.
#pragma once

#include "lds_pipe.h"

namespace moga {

constexpr unsigned kBufferBytes = 0x7ffffff0u, kPastBuffer = 0x80000000u;

// 16 bytes a lane from `base + voff` to LDS (the wave's 1 KB at lds_wave_base); zeros where voff is kPastBuffer.
__device__ __forceinline__ void lds_dma16_buffer(const void* base, unsigned voff, unsigned lds_wave_base) {
  const uint64_t a = (uint64_t)(uintptr_t)base;
  const uintx4_t rsrc = {(unsigned)__builtin_amdgcn_readfirstlane((unsigned)a), (unsigned)__builtin_amdgcn_readfirstlane((unsigned)(a >> 32)) & 0xffffu,
                         kBufferBytes, 0x00020000u};
  lds_wave_base = __builtin_amdgcn_readfirstlane(lds_wave_base);
  asm volatile("s_mov_b32 m0, %0\n\ts_nop 0\n\tbuffer_load_dwordx4 %1, %2, 0 offen lds" : : "s"(lds_wave_base), "v"(voff), "s"(rsrc) : "memory");
}

template <typename T> struct Frag;
template <> struct Frag<unsigned short> { bf16x8_t v; };
template <> struct Frag<float> { floatx4_t v; };

__device__ __forceinline__ floatx4_t mfma_frag(Frag<unsigned short> a, Frag<unsigned short> b, floatx4_t c) {
  return __builtin_amdgcn_mfma_f32_16x16x32_bf16(a.v, b.v, c, 0, 0, 0);
}
// k = 4 g + j of lane group g in product j, in both operands
__device__ __forceinline__ floatx4_t mfma_frag(Frag<float> a, Frag<float> b, floatx4_t c) {
#pragma unroll
  for (int j = 0; j < 4; ++j) c = __builtin_amdgcn_mfma_f32_16x16x4f32(a.v[j], b.v[j], c, 0, 0, 0);
  return c;
}

// One operand of a block: ROWS rows (or columns) by 128 bytes of k, staged by the block; a wave reads TILES tiles of 16 from tile `first`, a multiple
// of TILES, on.
template <typename T, bool KFIRST, int ROWS, int THREADS, int TILES>
struct Operand {
  static constexpr int ES = sizeof(T), V = 16 / ES, BK = 128 / ES, L = ROWS * 8 / THREADS, CPR = ROWS * ES / 16;
  static constexpr unsigned kBytes = ROWS * 128;
  const unsigned char* base;   // of this block's rows at its first k; wave-uniform
  const unsigned char* base2;  // of the second half of the rows of each 64 (rows_paired)
  int64_t step_bytes;
  unsigned voff[L];
  int kofs[KFIRST ? L : 1];
  unsigned read[KFIRST ? TILES : 2];   // lane's LDS offsets
  int k_left;                          // k from the present step on

  __device__ __forceinline__ static int swizzle(int k) {   // columns: exchanged 16-byte chunks of row k
    return ES == 2 ? ((k & 3) | ((k >> 1) & 4)) * 2 : ((k >> 2) & 3) * 4;
  }

  // rows r0 .. of a matrix [R][ld], or columns r0 .. of a matrix [..][ld]; k_count of k from k0 on
  __device__ __forceinline__ void init(const T* p, int64_t ld, int64_t r0, int64_t R, int64_t k0, int k_count, int first) {
    const int t = threadIdx.x;
    k_left = k_count;
    base = (const unsigned char*)(KFIRST ? p + k0 * ld + r0 : p + r0 * ld + k0);
    step_bytes = KFIRST ? (int64_t)BK * ld * ES : 128;
    const int64_t left = R - r0;
#pragma unroll
    for (int i = 0; i < L; ++i) {
      const int q = i * THREADS + t;
      if constexpr (KFIRST) {
        const int k = q / CPR, c = (q % CPR) ^ swizzle(k);
        kofs[i] = k;
        voff[i] = c * V < left ? (unsigned)(k * ld * ES + c * 16) : kPastBuffer;
      } else {
        const int j = q >> 3, c = (q & 7) ^ ((j >> 1) & 7);
        kofs[0] = c * V;   // the same in every i
        voff[i] = j < left ? (unsigned)(j * ld * ES + c * 16) : kPastBuffer;
      }
    }
    init_read(first);
  }
  // Of each 64 staged rows 32 are rows f0 + .. of a matrix [2 F][ld] and 32 the same rows of its second half.
  __device__ __forceinline__ void init_paired(const T* p, int64_t ld, int64_t f0, int64_t F, int k_count, int first) {
    static_assert(!KFIRST);
    k_left = k_count;
    base = (const unsigned char*)(p + f0 * ld);
    base2 = base + F * ld * ES;
    step_bytes = 128;
#pragma unroll
    for (int i = 0; i < L; ++i) {
      const int q = i * THREADS + threadIdx.x, j = q >> 3, c = (q & 7) ^ ((j >> 1) & 7), f = (j >> 6) * 32 + (j & 31);
      kofs[0] = c * V;
      voff[i] = f < F - f0 ? (unsigned)(f * ld * ES + c * 16) : kPastBuffer;
    }
    init_read(first);
  }
  __device__ __forceinline__ void init_read(int first) {
    const int l = threadIdx.x & 63, r = l & 15, g = l >> 4;
    if constexpr (!KFIRST) {
      read[0] = first * 2048 + r * 128 + ((g ^ (r >> 1)) & 7) * 16;
      read[1] = read[0] ^ 64;
    } else {
      static_assert(TILES <= 8);
      const int k = ES == 2 ? 8 * g + (r >> 2) : 4 * g;
#pragma unroll
      for (int j = 0; j < TILES; ++j) {
        const int col = (first + j) * 16 + (ES == 2 ? (r & 3) * 4 : r), c = (col / V) ^ swizzle(k);
        read[j] = k * ROWS * ES + c * 16 + col % V * ES;
      }
    }
  }

  // The i-th of the thread's loads of the present step
  template <bool PAIRED = false>
  __device__ __forceinline__ void stage(unsigned lds, int i) const {
    const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    const unsigned char* b = base;
    if (PAIRED && ((i * (THREADS / 8) + wave * 8) & 32)) b = base2;
    lds_dma16_buffer(b, kofs[KFIRST ? i : 0] < k_left ? voff[i] : kPastBuffer, lds + i * THREADS * 16 + wave * 1024);
  }
  template <bool PAIRED = false>
  __device__ __forceinline__ void advance() {
    base += step_bytes;
    if (PAIRED) base2 += step_bytes;
    k_left -= BK;
  }

  // Operand of the wave's tile, half kk of the step
  __device__ __forceinline__ Frag<T> get(unsigned lds, int tile, int kk) const {
    Frag<T> f;
    if constexpr (!KFIRST) {
      f.v = __builtin_bit_cast(decltype(f.v), *(const uintx4_t __attribute__((address_space(3)))*)(uintptr_t)(lds + read[kk] + tile * 2048));
    } else if constexpr (ES == 2) {
      const unsigned at = lds + read[tile] + kk * 32 * ROWS * 2;
      f.v = concat_tr(lds_read_tr16_addr(at), lds_read_tr16_addr(at + 4 * ROWS * 2));
    } else {
      const unsigned at = lds + read[tile] + kk * 16 * ROWS * 4;
#pragma unroll
      for (int j = 0; j < 4; ++j) f.v[j] = *(const float __attribute__((address_space(3)))*)(uintptr_t)(at + j * ROWS * 4);
    }
    return f;
  }
};

// Block b of `tiles` in an order in which the blocks of an XCD (every eighth) are neighbours.
__device__ __forceinline__ unsigned xcd_order(unsigned b, unsigned tiles) {
  const unsigned x = b & 7, per = tiles >> 3, rem = tiles & 7;
  return x * per + min(x, rem) + (b >> 3);
}

}  // namespace moga

// What the products of few rows with 8-bit weights share: a lane's codes of weight columns
// and of a row, and the partial sums of a workgroup's waves.
#pragma once
#include "fp8_block.h"

namespace smoe {

template <int NJ>
using Stream8Part = f32x4[16][4 * NJ + 1];  // one wave's 16 x 16 NJ partial (padded rows)

// the largest of the lanes l % 16 + {0, 16, 32, 48}
__device__ __forceinline__ uint32_t max_of_row(uint32_t m) {
  m = max(m, (uint32_t)__shfl_xor((int)m, 16, kWave));
  return max(m, (uint32_t)__shfl_xor((int)m, 32, kWave));
}

// A lane's 32 values of a row's block of 128, from bf16 (4 x 8) or fp32 (8 x 4), and
// their codes and scale byte
template <bool F32>
struct RowBlock8 {
  static constexpr int N = F32 ? 8 : 4;
  u32x4 v[N];
  // x: the row; k: 16 g of the block's first k; valid: whether the block's second half exists
  __device__ __forceinline__ void load(const void* x, uint32_t k, bool second) {
    const char* p = (const char*)x + (size_t)k * (F32 ? 4 : 2);
#pragma unroll
    for (int i = 0; i < N; ++i) {
      const bool hi = i >= N / 2;
      v[i] = !hi || second ? *(const u32x4*)(p + (hi ? 64 * (F32 ? 4 : 2) : 0) + 16 * (i % (N / 2))) : u32x4{0, 0, 0, 0};
    }
  }
  __device__ __forceinline__ i32x8 codes(int* scale) const {
    uint32_t m;
    if constexpr (F32) {
      float a[32];
#pragma unroll
      for (int i = 0; i < 32; ++i) a[i] = __uint_as_float(v[i / 4][i % 4]);
      m = __float_as_uint(finite_amax(a));
    } else {
      uint32_t w[16];
#pragma unroll
      for (int i = 0; i < 16; ++i) w[i] = v[i / 4][i % 4];
      m = finite_amax_bf16(w) << 16;
    }
    *scale = scale_byte(max_of_row(m));
    const float sv = scale_value(*scale);
    i32x8 q;
#pragma unroll
    for (int i = 0; i < 8; ++i) {
      if constexpr (F32) {
        const u32x4 x = v[i];
        q[i] = (int)pack_fp8x4(__uint_as_float(x[0]), __uint_as_float(x[1]), __uint_as_float(x[2]), __uint_as_float(x[3]), sv);
      } else {
        q[i] = (int)pack_fp8x4_bf16(v[i / 2][2 * (i & 1)], v[i / 2][2 * (i & 1) + 1], sv);
      }
    }
    return q;
  }
};

// A lane's codes of NJ times 16 weight columns and one block of 128 k
template <int NJ>
struct Weights8 {
  u32x4 v[NJ][2];
  __device__ __forceinline__ void load(const uint8_t* w, const uint32_t (&row)[NJ], uint32_t k) {
#pragma unroll
    for (int j = 0; j < NJ; ++j) {
      v[j][0] = *(const u32x4*)(w + (size_t)(row[j] + k));
      v[j][1] = *(const u32x4*)(w + (size_t)(row[j] + k + 64));
    }
  }
  __device__ __forceinline__ i32x8 frag(int j) const {
    const u32x4 lo = v[j][0], hi = v[j][1];
    return i32x8{(int)lo[0], (int)lo[1], (int)lo[2], (int)lo[3], (int)hi[0], (int)hi[1], (int)hi[2], (int)hi[3]};
  }
};

// the sum over the waves of columns 4 c4 .. 4 c4 + 3 of the tile
template <int KW, int NJ>
__device__ __forceinline__ f32x4 stream8_sum(const Stream8Part<NJ>* part, int row, int c4) {
  f32x4 s = part[0][row][c4];
#pragma unroll 7  // (all 15 of 16 waves at once spilled)
  for (int w = 1; w < KW; ++w)
#pragma unroll
    for (int q = 0; q < 4; ++q) s[q] += part[w][row][c4][q];
  return s;
}

}  // namespace smoe

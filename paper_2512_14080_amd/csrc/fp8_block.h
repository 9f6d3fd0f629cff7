// The 8-bit block format: e4m3 codes (no infinities, largest value 448) of blocks
// of up to 128 values, and one power-of-two scale per block.
//   amax  = the largest finite |x| of the block
//   e     = the least integer >= -126 with amax <= 448 * 2^e
//   code  = e4m3(x * 2^-e), to nearest even; infinities and NaN become the NaN code
//   scale = the byte e + 127, which stands for 2^e
// A power of two only moves the exponent: x * 2^-e is exact (e4m3 keeps four
// significant bits wherever the block lies), the codes are a function of the
// values alone, and the matrix instruction takes the byte as it is
// (v_mfma_scale_f32_*_f8f6f4), so a product needs no pass over its accumulators
// per block of 128.
#pragma once
#include "device_common.h"

namespace smoe {

constexpr int kQBlock = 128;

__host__ __device__ inline int q_blocks(int cols) { return (cols + kQBlock - 1) / kQBlock; }
// columns padded to whole blocks
__host__ __device__ inline int q_pad(int cols) { return q_blocks(cols) * kQBlock; }
// bytes of a row's scales: whole dwords, which the products load
__host__ __device__ inline int q_stride(int blocks) { return (blocks + 3) / 4 * 4; }

// Expert weights as the products read them, k contiguous (np = q_pad(n)):
//   W1q [E][np / 128][2 halves of 64][gate, up][64 columns][d]   W1s [E][np / 128][gate, up][q_stride(d / 128)]
//   W2q [E][d columns][np]                                       W2s [E][d / 128][q_stride(np / 128)]
// W1's rows come in the order of a tile of 128 gate and 128 up columns whose two
// column groups of waves hold 64 of each; columns and k past n are zero.
__host__ __device__ inline int w1q_row(int col, int up) {
  return ((col >> 6) * 2 + up) * 64 + (col & 63);
}
__host__ __device__ inline size_t w1q_bytes(int d, int n) { return (size_t)2 * q_pad(n) * d; }
__host__ __device__ inline size_t w2q_bytes(int d, int n) { return (size_t)d * q_pad(n); }
__host__ __device__ inline size_t w1s_bytes(int d, int n) { return (size_t)q_blocks(n) * 2 * q_stride(d / kQBlock); }
__host__ __device__ inline size_t w2s_bytes(int d, int n) { return (size_t)(d / kQBlock) * q_stride(q_blocks(n)); }
// the scales of a kept H row: its gate blocks, then its up blocks
__host__ __device__ inline int h8_stride(int n) { return q_stride(2 * q_blocks(n)); }

// amax_bits: of a finite fp32 value >= 0.  Its exponent less that of 448 = 1.75 * 2^8,
// and one more where its fraction is above 1.75
__device__ __forceinline__ int scale_byte(uint32_t amax_bits) { return max((int)((amax_bits + 0x1FFFFFu) >> 23) - 8, 1); }
__device__ __forceinline__ float scale_value(int b) { return __uint_as_float((uint32_t)b << 23); }
__device__ __forceinline__ float scale_inverse(int b) { return __uint_as_float((uint32_t)(254 - b) << 23); }

// four values (|x| <= 448, or not finite) -> four codes
__device__ __forceinline__ uint32_t pack_fp8x4(float a, float b, float c, float d) {
  const int v = __builtin_amdgcn_cvt_pk_fp8_f32(a, b, 0, false);
  return (uint32_t)__builtin_amdgcn_cvt_pk_fp8_f32(c, d, v, true);
}
// four codes -> four values
__device__ __forceinline__ f32x4 unpack_fp8x4(uint32_t v) {
  const auto lo = __builtin_amdgcn_cvt_pk_f32_fp8((int)v, false), hi = __builtin_amdgcn_cvt_pk_f32_fp8((int)v, true);
  return f32x4{lo[0], lo[1], hi[0], hi[1]};
}
// |x|, 0 for what is not finite
__device__ __forceinline__ float finite_abs(float x) {
  const float a = fabsf(x);
  return a < INFINITY ? a : 0.f;
}

}  // namespace smoe

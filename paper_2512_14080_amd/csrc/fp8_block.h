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

// (cols >= 1, up to the largest int)
__host__ __device__ inline int q_blocks(int cols) { return (cols - 1) / kQBlock + 1; }
// columns padded to whole blocks
__host__ __device__ inline int q_pad(int cols) { return q_blocks(cols) * kQBlock; }
// bytes of a row's scales: whole dwords, which the products load
__host__ __device__ inline int q_stride(int blocks) { return (blocks + 3) / 4 * 4; }

// Expert weights as the products read them, k contiguous (np = q_pad(n)):
//   W1q [E][np / 128][4 quarters][gate, up][32 columns][d]   W1s [E][np / 128][gate, up][q_stride(d / 128)]
//   W2q [E][d columns][np]                                   W2s [E][d / 128][q_stride(np / 128)]
// W1's rows alternate between 32 gate and the 32 matching up columns, so that any
// wave of a tile holds both; columns and k past n are zero.
__host__ __device__ inline int w1q_row(int col, int up) { return ((col >> 5) * 2 + up) * 32 + (col & 31); }
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

// The scaled conversions divide or multiply by the scale as they convert: for every
// scale byte, the codes of x * 2^-e and the values of code * 2^e, bit for bit.
typedef short i16x2 __attribute__((ext_vector_type(2)));
// four values (|x| <= 448 * scale, or not finite) -> four codes
__device__ __forceinline__ uint32_t pack_fp8x4(float a, float b, float c, float d, float scale) {
  const i16x2 v = __builtin_amdgcn_cvt_scalef32_pk_fp8_f32(i16x2{0, 0}, a, b, scale, false);
  return __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_fp8_f32(v, c, d, scale, true));
}
// the same from two bf16 pairs
__device__ __forceinline__ uint32_t pack_fp8x4_bf16(uint32_t ab, uint32_t cd, float scale) {
  const i16x2 v = __builtin_amdgcn_cvt_scalef32_pk_fp8_bf16(i16x2{0, 0}, __builtin_bit_cast(bf16x2v, ab), scale, false);
  return __builtin_bit_cast(uint32_t,
                            __builtin_amdgcn_cvt_scalef32_pk_fp8_bf16(v, __builtin_bit_cast(bf16x2v, cd), scale, true));
}
// four codes -> four values
__device__ __forceinline__ f32x4 unpack_fp8x4(uint32_t v, float scale) {
  const auto lo = __builtin_amdgcn_cvt_scalef32_pk_f32_fp8(v, scale, false);
  const auto hi = __builtin_amdgcn_cvt_scalef32_pk_f32_fp8(v, scale, true);
  return f32x4{lo[0], lo[1], hi[0], hi[1]};
}
// codes 8 i .. 8 i + 7 of a fragment as bf16 values, code * scale: exact within bf16's
// range (2^-133 up; a value above 3.3e38 may have a code that stands for 2^128)
typedef int i32x8 __attribute__((ext_vector_type(8)));
__device__ __forceinline__ bf16x8 codes_bf16(const i32x8& q, int i, float scale) {
  u32x4 v;
#pragma unroll
  for (int h = 0; h < 2; ++h) {
    v[2 * h] = __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(q[2 * i + h], scale, false));
    v[2 * h + 1] = __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(q[2 * i + h], scale, true));
  }
  return __builtin_bit_cast(bf16x8, v);
}
// the largest |x| of N bf16 pairs, finite ones only, as bf16 bits
typedef uint16_t u16x2 __attribute__((ext_vector_type(2)));
template <int N>
__device__ __forceinline__ uint32_t finite_amax_bf16(const uint32_t (&w)[N]) {
  u16x2 m = {0, 0};
#pragma unroll
  for (int i = 0; i < N; ++i) m = __builtin_elementwise_max(m, __builtin_bit_cast(u16x2, w[i] & 0x7FFF7FFFu));
  uint32_t a = max((uint32_t)m[0], (uint32_t)m[1]);
  if (__builtin_expect(__any(a >= 0x7F80u), 0)) {
    a = 0;
#pragma unroll
    for (int i = 0; i < N; ++i) {
      const uint32_t lo = w[i] & 0x7FFFu, hi = w[i] >> 16 & 0x7FFFu;
      a = max(a, max(lo < 0x7F80u ? lo : 0u, hi < 0x7F80u ? hi : 0u));
    }
  }
  return a;
}
// |x|, 0 for what is not finite
__device__ __forceinline__ float finite_abs(float x) {
  const float a = fabsf(x);
  return a < INFINITY ? a : 0.f;
}

// the largest |x| of N fp32 values, finite ones only
template <int N>
__device__ __forceinline__ float finite_amax(const float (&x)[N]) {
  float m = 0.f;
#pragma unroll
  for (int i = 0; i < N; ++i) m = fmaxf(m, fabsf(x[i]));  // (passes over NaN)
  if (__builtin_expect(__any(m == INFINITY), 0)) {
    m = 0.f;
#pragma unroll
    for (int i = 0; i < N; ++i) m = fmaxf(m, finite_abs(x[i]));
  }
  return m;
}

// Rows of `blocks` blocks that one launch takes, 16 lanes a block: it holds fewer than
// 2^32 work-items, and 2^27 blocks (32 GB of whole ones, 2 GB of rows of 8 columns) are half
inline int64_t quant_rows(int blocks) { return (1 << 27) / blocks; }

// Block u of the rows X [.., cols] (`blocks` blocks a row), by 16 lanes with 8 columns
// (16 bytes) each: the largest |x| is a maximum over the lane's values and the lanes.
__device__ __forceinline__ void quantize_unit(const uint16_t* __restrict__ X, int u, int blocks, int cols, int stride,
                                              uint8_t* __restrict__ q, uint8_t* __restrict__ scale) {
  const int l = threadIdx.x & 15, row = u / blocks, b = u - row * blocks, c = b * kQBlock + 8 * l;
  u32x4 v = {0, 0, 0, 0};
  if (c < cols) v = *(const u32x4*)(X + (size_t)row * cols + c);
  const uint32_t w[4] = {v[0], v[1], v[2], v[3]};
  uint32_t m = finite_amax_bf16(w);
#pragma unroll
  for (int o = 8; o > 0; o >>= 1) m = max(m, (uint32_t)__shfl_xor((int)m, o, 16));
  const int sb = scale_byte(m << 16);
  const float sv = scale_value(sb);
  if (c < cols)
    *(u32x2*)(q + (size_t)row * cols + c) = u32x2{pack_fp8x4_bf16(v[0], v[1], sv), pack_fp8x4_bf16(v[2], v[3], sv)};
  // (the last block's first lanes also fill the row's scales to a whole dword)
  if (l == 0 || (b == blocks - 1 && b + l < stride)) scale[(size_t)row * stride + b + l] = l ? 127 : sb;
}

// and back
__device__ __forceinline__ void dequantize_unit(const uint8_t* __restrict__ q, const uint8_t* __restrict__ scale, int u,
                                                int blocks, int cols, int stride, uint16_t* __restrict__ X) {
  const int l = threadIdx.x & 15, row = u / blocks, b = u - row * blocks, c = b * kQBlock + 8 * l;
  if (c >= cols) return;
  const float s = scale_value(scale[(size_t)row * stride + b]);
  const u32x2 v = *(const u32x2*)(q + (size_t)row * cols + c);
  u32x4 out;
#pragma unroll
  for (int i = 0; i < 2; ++i) {
    const f32x4 x = unpack_fp8x4(v[i], s);
    out[2 * i] = pack_bf2(x[0], x[1]);
    out[2 * i + 1] = pack_bf2(x[2], x[3]);
  }
  *(u32x4*)(X + (size_t)row * cols + c) = out;
}

}  // namespace smoe

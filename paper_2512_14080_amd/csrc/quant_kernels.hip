// The 8-bit block format (fp8_block.h) to and from bf16: rows of activations, and
// the expert weights in the layout that the 8-bit products read.
#include <algorithm>

#include "fp8_block.h"
#include "launch.h"

namespace smoe {

constexpr int kRowThreads = 256;

// ---------------------------------------------------------------- rows
__global__ __launch_bounds__(kRowThreads) void quantize_rows_kernel(const uint16_t* __restrict__ X, int units, int blocks,
                                                                    int cols, int stride, uint8_t* __restrict__ q,
                                                                    uint8_t* __restrict__ scale) {
  const int u = blockIdx.x * (kRowThreads / 16) + (threadIdx.x >> 4);
  if (u < units) quantize_unit(X, u, blocks, cols, stride, q, scale);
}

__global__ __launch_bounds__(kRowThreads) void dequantize_rows_kernel(const uint8_t* __restrict__ q,
                                                                      const uint8_t* __restrict__ scale, int units,
                                                                      int blocks, int cols, int stride,
                                                                      uint16_t* __restrict__ X) {
  const int u = blockIdx.x * (kRowThreads / 16) + (threadIdx.x >> 4);
  if (u < units) dequantize_unit(q, scale, u, blocks, cols, stride, X);
}

static int row_groups(int units) { return (units + kRowThreads / 16 - 1) / (kRowThreads / 16); }

// rows * blocks of a row < 2^31, in launches of at most quant_rows(blocks) rows (a loop in
// the kernel instead took 279 us for 131072 rows of 4096 columns, not 264)
hipError_t launch_quantize_rows(const uint16_t* X, int64_t rows, int cols, uint8_t* q, uint8_t* scale, hipStream_t s) {
  const int blocks = q_blocks(cols), stride = q_stride(blocks);
  for (int64_t first = 0; first < rows; first += quant_rows(blocks)) {
    const int units = (int)std::min(rows - first, quant_rows(blocks)) * blocks;
    quantize_rows_kernel<<<row_groups(units), kRowThreads, 0, s>>>(X + first * cols, units, blocks, cols, stride,
                                                                   q + first * cols, scale + first * stride);
    const hipError_t err = hipGetLastError();
    if (err != hipSuccess) return err;
  }
  return hipSuccess;
}
hipError_t launch_dequantize_rows(const uint8_t* q, const uint8_t* scale, int64_t rows, int cols, uint16_t* X,
                                  hipStream_t s) {
  const int blocks = q_blocks(cols), stride = q_stride(blocks);
  for (int64_t first = 0; first < rows; first += quant_rows(blocks)) {
    const int units = (int)std::min(rows - first, quant_rows(blocks)) * blocks;
    dequantize_rows_kernel<<<row_groups(units), kRowThreads, 0, s>>>(q + first * cols, scale + first * stride, units, blocks,
                                                                     cols, stride, X + first * cols);
    const hipError_t err = hipGetLastError();
    if (err != hipSuccess) return err;
  }
  return hipSuccess;
}

// ---------------------------------------------------------------- expert weights
// One 128 x 128 block of one matrix: k rows k0 .., columns c0 .. of a half.
struct WeightBlock {
  int e, kb, nb, up;   // expert, block of k, block of columns, half (W1)
  bool w1;
  __device__ __forceinline__ bool init(const QExpertsArgs& a, int id) {
    const int kd = a.d / kQBlock, nn = q_blocks(a.n);
    w1 = id < a.E * kd * nn * 2;
    if (w1) {
      kb = id % kd;
      id /= kd;
      up = id & 1;
      id >>= 1;
      nb = id % nn;
      e = id / nn;
    } else {
      id -= a.E * kd * nn * 2;
      kb = id % nn;
      id /= nn;
      nb = id % kd;
      e = id / kd;
      up = 0;
    }
    return e < a.E;
  }
  // first element of the block in the bf16 matrix, its leading dimension, and the
  // columns and k rows that exist
  __device__ __forceinline__ size_t source(const QExpertsArgs& a, int* ld, int* cols, int* ks) const {
    if (w1) {
      *ld = 2 * a.n;
      *cols = a.n - kQBlock * nb;
      *ks = kQBlock;
      return ((size_t)e * a.d + kQBlock * kb) * (2 * a.n) + (size_t)up * a.n + kQBlock * nb;
    }
    *ld = a.d;
    *cols = kQBlock;
    *ks = a.n - kQBlock * kb;
    return ((size_t)e * a.n + kQBlock * kb) * a.d + kQBlock * nb;
  }
  // codes of column c of the block, from the block's first k on
  __device__ __forceinline__ size_t codes(const QExpertsArgs& a, int c) const {
    if (w1) return (size_t)e * w1q_bytes(a.d, a.n) + (size_t)(256 * nb + w1q_row(c, up)) * a.d + kQBlock * kb;
    return (size_t)e * w2q_bytes(a.d, a.n) + (size_t)(kQBlock * nb + c) * q_pad(a.n) + kQBlock * kb;
  }
  __device__ __forceinline__ size_t scales(const QExpertsArgs& a, int* blocks) const {
    if (w1) {
      *blocks = a.d / kQBlock;
      return (size_t)e * w1s_bytes(a.d, a.n) + (size_t)(2 * nb + up) * q_stride(*blocks) + kb;
    }
    *blocks = q_blocks(a.n);
    return (size_t)e * w2s_bytes(a.d, a.n) + (size_t)nb * q_stride(*blocks) + kb;
  }
};

constexpr int kPitch = kQBlock + 16;  // LDS bytes of a column's 128 codes

// A thread loads 8 columns of 8 consecutive k rows and so holds 8 codes of each of
// its columns; they go through LDS, and out as whole 128-byte runs of k.
__global__ __launch_bounds__(256) void quantize_experts_kernel(const QExpertsArgs a) {
  __shared__ __attribute__((aligned(16))) char tile[kQBlock * kPitch];
  __shared__ uint32_t wmax[4];
  WeightBlock w;
  if (!w.init(a, blockIdx.x)) return;
  int ld, cols, ks;
  const uint16_t* src = (w.w1 ? a.W1 : a.W2) + w.source(a, &ld, &cols, &ks);
  const int c = 8 * (threadIdx.x & 15), k = 8 * (threadIdx.x >> 4);
  u32x4 v[8];
#pragma unroll
  for (int i = 0; i < 8; ++i) {
    v[i] = u32x4{0, 0, 0, 0};
    if (c < cols && k + i < ks) v[i] = *(const u32x4*)(src + (size_t)(k + i) * ld + c);
  }
  uint32_t words[32];
#pragma unroll
  for (int i = 0; i < 32; ++i) words[i] = v[i / 4][i % 4];
  uint32_t m = finite_amax_bf16(words);
  m = dpp_reduce(m, [](uint32_t x, uint32_t y) { return max(x, y); });
  if (lane_id() == 0) wmax[threadIdx.x >> 6] = m;
  __syncthreads();
  const int sb = scale_byte(max(max(wmax[0], wmax[1]), max(wmax[2], wmax[3])) << 16);
  const float sv = scale_value(sb);
#pragma unroll
  for (int j = 0; j < 8; ++j) {
    // column c + j of eight rows as bf16 pairs
    uint32_t x[4];
#pragma unroll
    for (int i = 0; i < 4; ++i)
      x[i] = __builtin_amdgcn_perm(v[2 * i + 1][j >> 1], v[2 * i][j >> 1], j & 1 ? 0x07060302u : 0x05040100u);
    *(u32x2*)(tile + (c + j) * kPitch + k) = u32x2{pack_fp8x4_bf16(x[0], x[1], sv), pack_fp8x4_bf16(x[2], x[3], sv)};
  }
  __syncthreads();
  uint8_t* q = w.w1 ? a.W1q : a.W2q;
#pragma unroll
  for (int i = 0; i < 4; ++i) {
    const int col = (threadIdx.x >> 3) + 32 * i, at = 16 * (threadIdx.x & 7);
    *(u32x4*)(q + w.codes(a, col) + at) = *(const u32x4*)(tile + col * kPitch + at);
  }
  int blocks;
  uint8_t* s = (w.w1 ? a.W1s : a.W2s) + w.scales(a, &blocks);
  const int i = threadIdx.x;
  if (i == 0 || (w.kb == blocks - 1 && w.kb + i < q_stride(blocks))) s[i] = i ? 127 : sb;
}

__global__ __launch_bounds__(256) void dequantize_experts_kernel(const QExpertsArgs a) {
  __shared__ __attribute__((aligned(16))) char tile[kQBlock * kPitch];
  WeightBlock w;
  if (!w.init(a, blockIdx.x)) return;
  const uint8_t* q = w.w1 ? a.W1q : a.W2q;
#pragma unroll
  for (int i = 0; i < 4; ++i) {
    const int col = (threadIdx.x >> 3) + 32 * i, at = 16 * (threadIdx.x & 7);
    *(u32x4*)(tile + col * kPitch + at) = *(const u32x4*)(q + w.codes(a, col) + at);
  }
  int blocks, ld, cols, ks;
  const float s = scale_value(((w.w1 ? a.W1s : a.W2s) + w.scales(a, &blocks))[0]);
  uint16_t* dst = (w.w1 ? a.W1out : a.W2out) + w.source(a, &ld, &cols, &ks);
  __syncthreads();
  const int c = 8 * (threadIdx.x & 15), k = 8 * (threadIdx.x >> 4);
  if (c >= cols || k >= ks) return;  // (n is a multiple of 64: eight k rows all exist or none)
  f32x4 lo[8], hi[8];
#pragma unroll
  for (int j = 0; j < 8; ++j) {
    const u32x2 v = *(const u32x2*)(tile + (c + j) * kPitch + k);
    lo[j] = unpack_fp8x4(v[0], s);
    hi[j] = unpack_fp8x4(v[1], s);
  }
#pragma unroll
  for (int i = 0; i < 8; ++i) {
    u32x4 o;
#pragma unroll
    for (int j = 0; j < 4; ++j)
      o[j] = i < 4 ? pack_bf2(lo[2 * j][i & 3], lo[2 * j + 1][i & 3]) : pack_bf2(hi[2 * j][i & 3], hi[2 * j + 1][i & 3]);
    *(u32x4*)(dst + (size_t)(k + i) * ld + c) = o;
  }
}

static int weight_blocks(const QExpertsArgs& a) { return a.E * (a.d / kQBlock) * q_blocks(a.n) * 3; }

hipError_t launch_quantize_experts(const QExpertsArgs& a, hipStream_t s) {
  quantize_experts_kernel<<<weight_blocks(a), 256, 0, s>>>(a);
  return hipGetLastError();
}
hipError_t launch_dequantize_experts(const QExpertsArgs& a, hipStream_t s) {
  dequantize_experts_kernel<<<weight_blocks(a), 256, 0, s>>>(a);
  return hipGetLastError();
}

}  // namespace smoe

// The expert products of the 8-bit forward: H = X~ W1~_e over the gathered rows,
// A = SwiGLU(H) into 8-bit blocks, Y = A~ W2~_e, on the block-scaled matrix
// instruction v_mfma_scale_f32_32x32x64_f8f6f4.  Every scale covers 128 k, so one
// byte of the row's and one of the weights' serve two instructions.
#include "fp8_block.h"
#include "launch.h"

namespace smoe {

typedef int i32x8 __attribute__((ext_vector_type(8)));
typedef int i32x4q __attribute__((ext_vector_type(4)));

// A wave computes 32 rows x 32 weight columns straight from memory; a workgroup's
// four waves take 128 columns.  Lane l holds 32 consecutive k of row (or column)
// l % 32: bytes 32 (l / 32) .. of each 64.  D = W x X, so a lane ends with one row
// and the columns 8 g + 4 (l / 32) + [0, 4).
__device__ __forceinline__ f32x16 product_32x32(const uint8_t* w, const uint8_t* ws, const uint8_t* x, const uint8_t* xs,
                                                int k) {
  f32x16 acc;
#pragma unroll
  for (int i = 0; i < 16; ++i) acc[i] = 0.f;
  for (int k0 = 0; k0 < k; k0 += 64) {
    const int sw = ws[k0 / kQBlock], sx = xs[k0 / kQBlock];
    acc = __builtin_amdgcn_mfma_scale_f32_32x32x64_f8f6f4(*(const i32x8*)(w + k0), *(const i32x8*)(x + k0), acc, 0, 0, 0,
                                                         sw, 0, sx);
  }
  return acc;
}

// rows [32 (blockIdx.y % 8), + 32) of m-tile blockIdx.y / 8
struct RowBlock {
  int e, row, rows;
  __device__ __forceinline__ bool init(const int32_t* mtiles) {
    const i32x4q* list = (const i32x4q*)mtiles;
    const int idx = blockIdx.y / 8, sub = 32 * (blockIdx.y % 8);
    if (idx >= list[0][0]) return false;
    const i32x4q t = list[1 + idx];
    e = t[0];
    row = t[3] + sub;
    rows = t[2] - sub;
    return rows > 0;
  }
};

__global__ __launch_bounds__(256) void quant_up_kernel(const QuantArgs a) {
  RowBlock rb;
  if (!rb.init(a.mtiles)) return;
  const int lane = lane_id(), h = lane >> 5, np = q_pad(a.n);
  const int col = 128 * blockIdx.x + 32 * (threadIdx.x >> 6);
  const int r = rb.row + min(lane & 31, rb.rows - 1), t = a.row_token[r];
  const int c = col + (lane & 31);  // this lane's weight row: half c / 64 % 2, block c / 256
  const uint8_t* w = a.W1q + (size_t)rb.e * w1q_bytes(a.d, a.n) + (size_t)c * a.d + 32 * h;
  const uint8_t* ws = a.W1s + (size_t)rb.e * w1s_bytes(a.d, a.n) + (2 * (c / 256) + (c >> 6 & 1)) * q_stride(a.d / kQBlock);
  const f32x16 acc = product_32x32(w, ws, a.X8 + (size_t)t * a.d + 32 * h, a.Xs + (size_t)t * q_stride(a.d / kQBlock), a.d);
  if ((lane & 31) >= rb.rows) return;
  float* o = a.H32 + (size_t)r * (2 * np) + col + 4 * h;
#pragma unroll
  for (int g = 0; g < 4; ++g) *(f32x4*)(o + 8 * g) = f32x4{acc[4 * g], acc[4 * g + 1], acc[4 * g + 2], acc[4 * g + 3]};
}

// the block scale of values held by 16 lanes, 8 each
__device__ __forceinline__ int lanes16_scale(const float (&x)[8]) {
  float m = 0.f;
#pragma unroll
  for (int i = 0; i < 8; ++i) m = fmaxf(m, finite_abs(x[i]));
#pragma unroll
  for (int o = 8; o > 0; o >>= 1) m = fmaxf(m, __shfl_xor(m, o, 16));
  return scale_byte(__float_as_uint(m));
}
__device__ __forceinline__ u32x2 codes8(const float (&x)[8], int sb) {
  const float inv = scale_inverse(sb);
  return u32x2{pack_fp8x4(x[0] * inv, x[1] * inv, x[2] * inv, x[3] * inv),
               pack_fp8x4(x[4] * inv, x[5] * inv, x[6] * inv, x[7] * inv)};
}

// A = SwiGLU(H + b1) into 8-bit blocks, and H's own where it is kept: 16 lanes per
// block of 128 columns
__global__ __launch_bounds__(256) void quant_act_kernel(const QuantArgs a) {
  const int nb = q_blocks(a.n), np = q_pad(a.n);
  const int u = blockIdx.x * 16 + (threadIdx.x >> 4), l = threadIdx.x & 15;
  const int row = u / nb, b = u - row * nb, c = b * kQBlock + 8 * l;
  if (row >= a.offsets[a.E]) return;
  const float* hp = a.H32 + (size_t)row * (2 * np) + 256 * b;
  float g[8], up[8], act[8];
  const float* b1 = a.b1 && c < a.n ? a.b1 + (size_t)a.row_expert[row] * (2 * a.n) + c : nullptr;
#pragma unroll
  for (int i = 0; i < 8; ++i) {
    g[i] = hp[w1q_row(8 * l, 0) + i] + (b1 ? b1[i] : 0.f);
    up[i] = hp[w1q_row(8 * l, 1) + i] + (b1 ? b1[a.n + i] : 0.f);
    float sg;
    act[i] = silu_sig(g[i], &sg) * up[i];
  }
  const int sa = lanes16_scale(act);
  *(u32x2*)(a.A8 + (size_t)row * np + c) = codes8(act, sa);
  if (l == 0) a.As[(size_t)row * q_stride(nb) + b] = sa;
  if (!a.H8) return;
  const int sg = lanes16_scale(g), su = lanes16_scale(up);
  if (c < a.n) {
    uint8_t* h8 = a.H8 + (size_t)row * (2 * a.n) + c;
    *(u32x2*)h8 = codes8(g, sg);
    *(u32x2*)(h8 + a.n) = codes8(up, su);
  }
  if (l == 0) {
    uint8_t* hs = a.Hs + (size_t)row * h8_stride(a.n) + b;
    hs[0] = sg;
    hs[nb] = su;
  }
}

__global__ __launch_bounds__(256) void quant_down_kernel(const QuantArgs a) {
  RowBlock rb;
  if (!rb.init(a.mtiles)) return;
  const int lane = lane_id(), h = lane >> 5, np = q_pad(a.n), nb = q_blocks(a.n);
  const int col = 128 * blockIdx.x + 32 * (threadIdx.x >> 6);
  const int r = rb.row + min(lane & 31, rb.rows - 1);
  const uint8_t* w = a.W2q + (size_t)rb.e * w2q_bytes(a.d, a.n) + (size_t)(col + (lane & 31)) * np + 32 * h;
  const uint8_t* ws = a.W2s + (size_t)rb.e * w2s_bytes(a.d, a.n) + blockIdx.x * q_stride(nb);
  const f32x16 acc = product_32x32(w, ws, a.A8 + (size_t)r * np + 32 * h, a.As + (size_t)r * q_stride(nb), np);
  if ((lane & 31) >= rb.rows) return;
  const int c = col + 4 * h;
  const float* b2 = a.b2 ? a.b2 + (size_t)rb.e * a.d + c : nullptr;
#pragma unroll
  for (int g = 0; g < 4; ++g) {
    float y[4];
#pragma unroll
    for (int i = 0; i < 4; ++i) y[i] = acc[4 * g + i] + (b2 ? b2[8 * g + i] : 0.f);
    *(u32x2*)(a.Y + (size_t)r * a.d + c + 8 * g) = pack_bf16x4(y[0], y[1], y[2], y[3]);
  }
}

hipError_t launch_quant_up(const QuantArgs& a, hipStream_t s) {
  const int mt = a.capacity / kMTile + a.E;
  quant_up_kernel<<<dim3(2 * q_pad(a.n) / 128, 8 * mt), 256, 0, s>>>(a);
  quant_act_kernel<<<(a.capacity * q_blocks(a.n) + 15) / 16, 256, 0, s>>>(a);
  return hipGetLastError();
}
hipError_t launch_quant_down(const QuantArgs& a, hipStream_t s) {
  const int mt = a.capacity / kMTile + a.E;
  quant_down_kernel<<<dim3(a.d / 128, 8 * mt), 256, 0, s>>>(a);
  return hipGetLastError();
}

}  // namespace smoe

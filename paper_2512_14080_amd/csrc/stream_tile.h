// A column tile of a product of few rows: C[rows, 8 CG columns] of a workgroup whose
// waves split the reduction, weights straight from memory into registers (k outer, as
// W1, W2 and a dense W lie).
//
// A wave's step is 32 KB k.  A lane (g = lane / 16, l = lane % 16) loads 16 bytes (8
// columns) of 8 consecutive k rows and transposes its 8 x 8 block with 32 v_perm_b32;
// MFMA j (16x16x32) takes column 8 cg + j of every lane.  The 16 lane columns are CG =
// 16 / KB column groups times KB blocks of 32 k, and the 16 rows of the other operand
// RT = 16 / KB rows times the same KB blocks: the product of a k block with another
// one's rows is not looked at.  So KB = 1 takes 16 rows and 128 columns, and KB = 2 and
// 4 cut the tile to 64 columns of 8 rows and 32 of 4, with as many bytes in flight and
// no more instructions: few rows get more workgroups for their bytes.
//
// Loads are buffer loads: what is past the matrix or past the reduction reads as zero,
// so neither a k beyond the end nor a column beyond the last one needs a branch (and
// no Inf or NaN beside the matrix enters a sum).
#pragma once
#include "device_common.h"

namespace smoe {

typedef __amdgpu_buffer_rsrc_t Rsrc;
// [p, p + bytes), at most 2^31 - 1 of them
__device__ __forceinline__ Rsrc buffer_of(const void* p, uint32_t bytes) {
  const uint64_t u = (uint64_t)p;
  const uint32_t lo = __builtin_amdgcn_readfirstlane((uint32_t)u), hi = __builtin_amdgcn_readfirstlane((uint32_t)(u >> 32));
  return __builtin_amdgcn_make_buffer_rsrc((void*)((uint64_t)hi << 32 | lo), 0, __builtin_amdgcn_readfirstlane(bytes),
                                           0x00027000);
}
constexpr uint32_t kBufferOut = 0x80000000u;  // an offset past any of them, and so with up to 2^31 added
// SHARED: what other workgroups of the same launch write (and read): such values go past
// the caches that an XCD has to itself, loads and stores alike (the access of an
// agent-scope atomic), so that no cache has to be written back or invalidated.  A write-back
// of the L2 costs 3.2 us when every CU asks for it, an invalidation 1.8.
constexpr int kSharedAccess = 16;  // sc1
template <bool SHARED = false>
__device__ __forceinline__ u32x4 load16(Rsrc r, uint32_t off) {
  return __builtin_bit_cast(u32x4, __builtin_amdgcn_raw_buffer_load_b128(r, (int)off, 0, SHARED ? kSharedAccess : 0));
}
__device__ __forceinline__ void store16_shared(Rsrc r, uint32_t off, u32x4 v) {
  __builtin_amdgcn_raw_buffer_store_b128(__builtin_bit_cast(__attribute__((__vector_size__(16))) unsigned int, v), r, (int)off, 0,
                                         kSharedAccess);
}
__device__ __forceinline__ void store8_shared(Rsrc r, uint32_t off, u32x2 v) {
  __builtin_amdgcn_raw_buffer_store_b64(__builtin_bit_cast(__attribute__((__vector_size__(8))) unsigned int, v), r, (int)off, 0,
                                        kSharedAccess);
}

// 8 rows (k) x 8 columns of bf16, one row per register quad -> per column the
// 8 k values (an MFMA operand)
__device__ __forceinline__ bf16x8 column_of8(const u32x4 (&w)[8], int j) {
  const uint32_t sel = (j & 1) ? 0x07060302u : 0x05040100u;
  u32x4 f;
#pragma unroll
  for (int p = 0; p < 4; ++p) f[p] = __builtin_amdgcn_perm(w[2 * p + 1][j >> 1], w[2 * p][j >> 1], sel);
  return __builtin_bit_cast(bf16x8, f);
}

// The lane index from a volatile asm: address arithmetic on it is done where it is used and
// not hoisted out of a loop over items, where it would hold registers.
__device__ __forceinline__ int opaque_lane() {
  int l;
  asm volatile("v_mbcnt_lo_u32_b32 %0, -1, 0\n\tv_mbcnt_hi_u32_b32 %0, -1, %0" : "=v"(l));
  return l;
}

template <int KB>
struct RowTile {
  static_assert(KB == 1 || KB == 2 || KB == 4, "k blocks of a step");
  static constexpr int CG = 16 / KB, RT = 16 / KB, COLS = 8 * CG, KSTEP = 32 * KB;
  // a lane's column group, k block and row of the other operand
  static __device__ __forceinline__ int cg(int lane) { return lane & (CG - 1); }
  static __device__ __forceinline__ int kk(int lane) { return (lane & 15) / CG; }
  static __device__ __forceinline__ int row(int lane) { return lane & (RT - 1); }
  // the lane's first k within a step
  static __device__ __forceinline__ int k0(int lane) { return 32 * kk(lane) + 8 * (lane >> 4); }
  // one wave's partial sums: [k block][row][half of 8 columns][column group]
  typedef f32x4 Part[KB][RT][2][CG];

  static __device__ __forceinline__ void put(Part& part, const f32x4 (&acc)[8], int lane) {
    const int g = lane >> 4;
    if (KB > 1 && g * KB / 4 != kk(lane)) return;  // (another k block's rows)
#pragma unroll
    for (int r = 0; r < 4; ++r)
#pragma unroll
      for (int h = 0; h < 2; ++h)
        part[kk(lane)][(4 * g + r) % RT][h][cg(lane)] = f32x4{acc[4 * h][r], acc[4 * h + 1][r], acc[4 * h + 2][r], acc[4 * h + 3][r]};
  }
  // the sum over kw waves and the k blocks of columns 4 c4 .. 4 c4 + 3, in a fixed order
  static __device__ __forceinline__ f32x4 sum_of(const Part* part, int kw, int row, int c4) {
    f32x4 s = f32x4{0.f, 0.f, 0.f, 0.f};
    for (int w = 0; w < kw; ++w)
#pragma unroll
      for (int b = 0; b < KB; ++b) {
        const f32x4 v = part[w][b][row][c4 & 1][c4 >> 1];
#pragma unroll
        for (int q = 0; q < 4; ++q) s[q] += v[q];
      }
    return s;
  }
  template <int KW>
  static __device__ __forceinline__ f32x4 sum(const Part* part, int row, int c4) {
    f32x4 s = f32x4{0.f, 0.f, 0.f, 0.f};
#pragma unroll 8 / KB  // (all the loads at once spilled)
    for (int w = 0; w < KW; ++w)
#pragma unroll
      for (int b = 0; b < KB; ++b) {
        const f32x4 v = part[w][b][row][c4 & 1][c4 >> 1];
#pragma unroll
        for (int q = 0; q < 4; ++q) s[q] += v[q];
      }
    return s;
  }
};

template <int MB>
__device__ __forceinline__ void zero_acc(f32x4 (&acc)[MB][8]) {
#pragma unroll
  for (int b = 0; b < MB; ++b)
#pragma unroll
    for (int j = 0; j < 8; ++j) acc[b][j] = f32x4{0.f, 0.f, 0.f, 0.f};
}

// A wave's share of a reduction: steps wave, wave + kw, ... of k in [kbeg, kend), NBUF of
// them in flight.  w: the matrix, with ldw bytes from a k row to the next and the lane's
// column at byte wcol (kBufferOut: none); x: the rows, xoff the byte of k = 0 of the lane's
// row (kBufferOut: none).  prime() requests the first steps' weights (8 NBUF loads, always),
// add() the rest; SHARED: the rows are other workgroups' of this launch.
template <int KB, int NBUF>
struct RowStream {
  using Tile = RowTile<KB>;
  Rsrc w;
  uint32_t ldw, wcol;
  int kl, kend, ns, step;
  u32x4 wv[NBUF][8];

  __device__ __forceinline__ void load_w(int buf, int s) {
    const int k = kl + step * s;
    const uint32_t o = k < kend ? wcol + (uint32_t)k * ldw : kBufferOut;
#pragma unroll
    for (int i = 0; i < 8; ++i) wv[buf][i] = load16(w, o + i * ldw);
  }
  __device__ __forceinline__ void prime(Rsrc w_, uint32_t ldw_, uint32_t wcol_, int kbeg, int kend_, int wave,
                                        int kw, int lane) {
    w = w_;
    ldw = ldw_;
    wcol = wcol_;
    kend = kend_;
    step = Tile::KSTEP * kw;
    ns = (kend - kbeg - Tile::KSTEP * wave + step - 1) / step;
    kl = kbeg + Tile::k0(lane) + Tile::KSTEP * wave;
    // (a wave without a step requests nothing: its k is past the end)
#pragma unroll
    for (int q = 0; q < NBUF; ++q) load_w(q, q);
  }
  template <bool SHARED, int MB>
  __device__ __forceinline__ void add(f32x4 (&acc)[MB][8], Rsrc x_, const uint32_t (&xoff)[MB]) {
    if (ns <= 0) return;
    bf16x8 xv[NBUF][MB];
    auto load_x = [&](int buf, int s) {
      const int k = kl + step * s;
#pragma unroll
      for (int b = 0; b < MB; ++b)
        xv[buf][b] = __builtin_bit_cast(bf16x8, load16<SHARED>(x_, k < kend ? xoff[b] + 2 * (uint32_t)k : kBufferOut));
    };
#pragma unroll
    for (int q = 0; q < NBUF; ++q) load_x(q, q);
    for (int s = 0;; s += NBUF) {
#pragma unroll
      for (int q = 0; q < NBUF; ++q) {
#pragma unroll
        for (int j = 0; j < 8; ++j) {
          const bf16x8 wf = column_of8(wv[q], j);
#pragma unroll
          for (int b = 0; b < MB; ++b)
            acc[b][j] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(xv[q][b], wf, acc[b][j], 0, 0, 0);
        }
        if (s + q + 1 >= ns) return;
        __builtin_amdgcn_sched_barrier(0);  // (not ahead of the products: it would take registers of their own)
        load_w(q, s + q + NBUF);
        load_x(q, s + q + NBUF);
        __builtin_amdgcn_sched_barrier(0);
      }
    }
  }
};

}  // namespace smoe

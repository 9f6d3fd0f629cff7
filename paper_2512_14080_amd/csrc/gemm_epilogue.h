// Epilogues, tile order and launch of the GEMMs on the core of gemm_core.h, shared by the
// layer's and the dense ones.
#pragma once
#include <algorithm>

#include "gemm_core.h"

namespace smoe {

// One 32-column accumulator block of a row, as bf16: v[g] holds columns
// 8g + 4*(lane/32) + [0, 4) (the MFMA output layout).  One lane-pair swap per
// dword (v_permlane32_swap exchanges the upper half of its first operand with
// the lower half of its second) leaves every lane with 8 consecutive
// columns, so each lane stores 16 bytes: lane < 32 columns 8g .. 8g+7 and
// lane >= 32 columns 8g+8 .. 8g+15, for g = 0, 2.
__device__ __forceinline__ void store_block_bf16(uint16_t* row_block, const u32x2 (&v)[4]) {
  const int hi = (threadIdx.x >> 5) & 1;
#pragma unroll
  for (int g = 0; g < 4; g += 2) {
    const auto a = __builtin_amdgcn_permlane32_swap(v[g][0], v[g + 1][0], false, false);
    const auto b = __builtin_amdgcn_permlane32_swap(v[g][1], v[g + 1][1], false, false);
    *(u32x4*)(row_block + 8 * g + 8 * hi) = u32x4{a[0], b[0], a[1], b[1]};
  }
}

// The inverse: 16-byte loads of a 32-column block, returned in the
// accumulator layout of store_block_bf16 (the swap is its own inverse).
__device__ __forceinline__ void load_block_bf16(const uint16_t* row_block, u32x2 (&v)[4]) {
  const int hi = (threadIdx.x >> 5) & 1;
#pragma unroll
  for (int g = 0; g < 4; g += 2) {
    const u32x4 x = *(const u32x4*)(row_block + 8 * g + 8 * hi);
    const auto a = __builtin_amdgcn_permlane32_swap(x[0], x[2], false, false);
    const auto b = __builtin_amdgcn_permlane32_swap(x[1], x[3], false, false);
    v[g] = u32x2{a[0], b[0]};
    v[g + 1] = u32x2{a[1], b[1]};
  }
}

// Order of the tiles of an M-tile x N-tile grid.  The 32 workgroups of an XCD run
// neighbouring ids at about the same time and share operands through its L2.
// Row by row, 32 ids are whole rows of a few columns, but 1 x 32 tiles (33
// operand slabs) of a wide matrix, whose weights are then read again for every
// m-tile.  In blocks of B rows (1, 4 or 8), column by column within a block,
// they are 4 x 8 tiles (12 slabs).  us, row by row / B = 4 / B = 8:
//   E = 8, d = 4096, n = 14336, 1024 rows each  up 2280 / 2070 / 2083   down 1262 / 1220 / 1207
//   E = 128, d = 4096, n = 512, 2048 rows       dX~ 2108 / 2105 / 2147  down 1293 / 1293 / 1321
//   E = 256, d = 2048, n = 128, skewed          dX~ 449 / 453 / 432     down 353 / 356 / 335
//   E = 64, d = 4096, n = 2048, 256 rows        up 790 / 814 / 820      dW2 485 / 469 / 460
__device__ __forceinline__ void tile_order(int id, int rows, int cols, int B, int* row, int* col) {
  const int q = id / cols, c = id - q * cols;
  *row = q;
  *col = c;
  if ((q | (B - 1)) < rows) {  // (a last block of fewer rows goes row by row)
    const int r = (q & (B - 1)) * cols + c;
    *row = (q & ~(B - 1)) + (r & (B - 1));
    *col = B == 1 ? c : r >> (B == 4 ? 2 : 3);
  }
}

// fp32 tile of a partial slab [M][ld]
template <class Cfg>
__device__ __forceinline__ void store_part_f32(float* out, int64_t ld, int m0, int n0, int mrows, int ncols,
                                               Acc<Cfg>& t) {
#pragma unroll
  for (int i = 0; i < Cfg::RM; ++i) {
    if (t.m_of(i) >= mrows) continue;
    float* o = out + (size_t)(m0 + t.m_of(i)) * ld + n0;
#pragma unroll
    for (int j = 0; j < Cfg::RN; ++j)
#pragma unroll
      for (int g = 0; g < 4; ++g) {
        if (t.n_of(j, g) >= ncols) continue;
        f32x4 v;
#pragma unroll
        for (int q = 0; q < 4; ++q) v[q] = t.acc[i][j][4 * g + q];
        *(f32x4*)(o + t.n_of(j, g)) = v;
      }
  }
}

struct ColOffset {
  int c0;
  __device__ __forceinline__ int operator()(int c) const { return c0 + c; }
};

// Adds bias[colmap(c)] to every accumulator of tile-local column c (the
// expert biases of the projections).  A lane's accumulator block (j, g) holds
// four consecutive columns, which colmap keeps consecutive; columns from `cols`
// on (past the matrix, never stored) are left alone (ALL: there are none).
template <class Cfg, bool ALL = false, class ColMap>
__device__ __forceinline__ void add_col_bias(Acc<Cfg>& t, const float* bias, ColMap colmap, int cols) {
#pragma unroll
  for (int j = 0; j < Cfg::RN; ++j)
#pragma unroll
    for (int g = 0; g < 4; ++g) {
      const int c = colmap(t.n_of(j, g));
      if (!ALL && c >= cols) continue;
      const f32x4 b = *(const f32x4*)(bias + c);
#pragma unroll
      for (int i = 0; i < Cfg::RM; ++i)
#pragma unroll
        for (int r = 0; r < 4; ++r) t.acc[i][j][4 * g + r] += b[r];
    }
}

// Row-contiguous stores of a wave's output: the two 32-column accumulator
// blocks j, j+1 of one 32-row block (64 columns, 128 bytes of a bf16 row) go
// through the wave's own 2 KB of LDS, 16 rows at a time, and come back so
// that 8 lanes hold one 128-byte row segment.  Each store instruction then
// writes 8 whole cache lines instead of 32-byte pieces of 32 rows.  The LDS
// operations of one wave complete in order, so no barrier is needed; the
// 16-byte chunk c of staged row r sits at chunk c ^ ((r >> 1) & 7), which
// keeps both the writes (one chunk of 16 rows) and the reads (two whole
// rows per 16 lanes) free of bank conflicts.  The stores are nontemporal:
// these outputs (H and A, Y, dH and A', dX~, the weight gradients) are
// consumed by a later kernel that streams them once, and left in the cache
// as dirty lines they only add write-back traffic at the end of the
// producing kernel (plain stores measured slower for up and no better for dH).
constexpr int kStageBytesPerWave = 16 * 128;
template <class Cfg>
constexpr bool kStagedStores = Cfg::RN % 2 == 0 && Cfg::LDS_BYTES + Cfg::NW * kStageBytesPerWave + 256 <= 160 * 1024;
// store instructions per wave of store_rows_bf16_any on a full tile: staged
// (through the idle last stage or the epilogue area), four per 64-column row
// block; direct, two per 32 columns
template <class Cfg>
constexpr int kStoresPerFullTile =
    Cfg::RN % 2 == 0 && (Cfg::STAGE_BYTES >= Cfg::NW * 4096 || kStagedStores<Cfg>) ? Cfg::RM * (Cfg::RN / 2) * 4
                                                                                   : Cfg::RM * Cfg::RN * 2;
// Epilogue address arithmetic uses the lane index from a volatile asm, so
// it stays in the epilogue instead of being hoisted out of the tile loop.
__device__ __forceinline__ int epilogue_lane() { return volatile_lane(); }

__device__ __forceinline__ void store_rows64_staged(char* wl, uint16_t* blk, int64_t ld, int rows_valid,
                                                    const u32x2 (&v0)[4], const u32x2 (&v1)[4]) {
  const int lane = epilogue_lane();
  const int r = lane & 31, hi = lane >> 5;
  u32x4 c[2][2];  // [block][g/2]: 16 bytes, chunk 4*block + g + hi of row r
#pragma unroll
  for (int g = 0; g < 4; g += 2) {
    {
      const auto a = __builtin_amdgcn_permlane32_swap(v0[g][0], v0[g + 1][0], false, false);
      const auto b = __builtin_amdgcn_permlane32_swap(v0[g][1], v0[g + 1][1], false, false);
      c[0][g / 2] = u32x4{a[0], b[0], a[1], b[1]};
    }
    {
      const auto a = __builtin_amdgcn_permlane32_swap(v1[g][0], v1[g + 1][0], false, false);
      const auto b = __builtin_amdgcn_permlane32_swap(v1[g][1], v1[g + 1][1], false, false);
      c[1][g / 2] = u32x4{a[0], b[0], a[1], b[1]};
    }
  }
#pragma unroll
  for (int q = 0; q < 2; ++q) {
    if ((r >> 4) == q) {
      const int rr = r & 15;
#pragma unroll
      for (int b = 0; b < 2; ++b)
#pragma unroll
        for (int g = 0; g < 4; g += 2) {
          const int ch = 4 * b + g + hi;
          *(u32x4*)(wl + rr * 128 + ((ch ^ ((rr >> 1) & 7)) << 4)) = c[b][g / 2];
        }
    }
    // other lanes' data is read back: keep the compiler from reordering or
    // forwarding across this point (the hardware keeps one wave's LDS
    // operations in order)
    asm volatile("" ::: "memory");
#pragma unroll
    for (int t = 0; t < 2; ++t) {
      const int R = 8 * t + (lane >> 3), C = lane & 7;
      const u32x4 x = *(const u32x4*)(wl + R * 128 + ((C ^ ((R >> 1) & 7)) << 4));
      const int row = 16 * q + R;
      if (row < rows_valid) __builtin_nontemporal_store(x, (u32x4*)(blk + (row * (int)ld + 8 * C)));
    }
    asm volatile("" ::: "memory");  // reads of this round before the next round's writes
  }
}

// Two-step form of the staging above for 32 rows at once, used where an
// output's two 32-column blocks are produced one after the other: each block
// is written into a wave-private 4 KB area as soon as it is computed (chunk
// 4 * jj + g + hi of row r, same swizzle), and the 32 rows are then stored as
// whole lines.  The area must not be touched by other waves in between.
__device__ __forceinline__ void stage_block32(char* wl, int jj, const u32x2 (&v)[4]) {
  const int lane = epilogue_lane();
  const int r = lane & 31, hi = lane >> 5;
#pragma unroll
  for (int g = 0; g < 4; g += 2) {
    const auto a = __builtin_amdgcn_permlane32_swap(v[g][0], v[g + 1][0], false, false);
    const auto b = __builtin_amdgcn_permlane32_swap(v[g][1], v[g + 1][1], false, false);
    const int ch = 4 * jj + g + hi;
    *(u32x4*)(wl + r * 128 + ((ch ^ ((r >> 1) & 7)) << 4)) = u32x4{a[0], b[0], a[1], b[1]};
  }
}

__device__ __forceinline__ void store_staged32(const char* wl, uint16_t* blk, int64_t ld, int rows_valid) {
  asm volatile("" ::: "memory");  // the staged writes of every lane precede these reads
  const int lane = epilogue_lane();
#pragma unroll
  for (int t = 0; t < 4; ++t) {
    const int R = 8 * t + (lane >> 3), C = lane & 7;
    const u32x4 x = *(const u32x4*)(wl + R * 128 + ((C ^ ((R >> 1) & 7)) << 4));
    if (R < rows_valid) __builtin_nontemporal_store(x, (u32x4*)(blk + (R * (int)ld + 8 * C)));
  }
  asm volatile("" ::: "memory");  // and precede the next writes to the area
}

template <class Cfg>
__device__ __forceinline__ void store_rows_bf16(uint16_t* out, int64_t ld, int row_base, int mrows, int n0, int ncols,
                                                Acc<Cfg>& t, char* epi) {
  if constexpr (!kStagedStores<Cfg>) {
#pragma unroll
    for (int i = 0; i < Cfg::RM; ++i) {
      const int m = t.m_of(i);
      if (m >= mrows) continue;
      uint16_t* y = out + (size_t)(row_base + m) * ld + n0;
#pragma unroll
      for (int j = 0; j < Cfg::RN; ++j) {
        if (t.n_of(j, 0) >= ncols) continue;
        u32x2 v[4];
#pragma unroll
        for (int g = 0; g < 4; ++g)
          v[g] = pack_bf16x4(t.acc[i][j][4 * g], t.acc[i][j][4 * g + 1], t.acc[i][j][4 * g + 2], t.acc[i][j][4 * g + 3]);
        store_block_bf16(y + t.n_of(j, 0) - 4 * ((threadIdx.x >> 5) & 1), v);
      }
    }
    return;
  }
  char* wl = epi + (threadIdx.x >> 6) * kStageBytesPerWave;
  const int wm0 = t.m_of(0) - (threadIdx.x & 31);
#pragma unroll
  for (int i = 0; i < Cfg::RM; ++i) {
    const int m0 = wm0 + 32 * i;  // first tile row of the block
    if (m0 >= mrows) continue;
#pragma unroll
    for (int j = 0; j + 1 < Cfg::RN; j += 2) {
      if (t.n_of(j, 0) >= ncols) continue;
      u32x2 v0[4], v1[4];
#pragma unroll
      for (int g = 0; g < 4; ++g) {
        v0[g] = pack_bf16x4(t.acc[i][j][4 * g], t.acc[i][j][4 * g + 1], t.acc[i][j][4 * g + 2], t.acc[i][j][4 * g + 3]);
        v1[g] = pack_bf16x4(t.acc[i][j + 1][4 * g], t.acc[i][j + 1][4 * g + 1], t.acc[i][j + 1][4 * g + 2],
                            t.acc[i][j + 1][4 * g + 3]);
      }
      const int col = n0 + t.n_of(j, 0) - 4 * ((threadIdx.x >> 5) & 1);
      store_rows64_staged(wl, out + (size_t)(row_base + m0) * ld + col, ld, mrows - m0, v0, v1);
    }
  }
}

// As store_rows_bf16, for ops whose last stage buffer is idle during the
// epilogue (no DMA writes it before the next tile's first barrier): each 32 x
// 64 block pair goes through the wave's 4 KB share of it in one round
// (stage_block32 twice, then store_staged32) instead of two 16-row rounds
// through the 2 KB epilogue area.
template <class Cfg>
__device__ __forceinline__ void store_rows_bf16_stage(uint16_t* out, int64_t ld, int row_base, int mrows, int n0,
                                                      int ncols, Acc<Cfg>& t, char* epi) {
  static_assert(Cfg::RN % 2 == 0 && Cfg::STAGE_BYTES >= Cfg::NW * 4096, "a 4 KB share of the last stage per wave");
  char* st = epi - Cfg::STAGE_BYTES + (threadIdx.x >> 6) * 4096;
  const int wm0 = t.m_of(0) - (threadIdx.x & 31);
#pragma unroll
  for (int i = 0; i < Cfg::RM; ++i) {
    const int m0 = wm0 + 32 * i;  // first tile row of the block
    if (m0 >= mrows) continue;
#pragma unroll
    for (int j = 0; j + 1 < Cfg::RN; j += 2) {
      if (t.n_of(j, 0) >= ncols) continue;
      u32x2 v0[4], v1[4];
#pragma unroll
      for (int g = 0; g < 4; ++g) {
        v0[g] = pack_bf16x4(t.acc[i][j][4 * g], t.acc[i][j][4 * g + 1], t.acc[i][j][4 * g + 2], t.acc[i][j][4 * g + 3]);
        v1[g] = pack_bf16x4(t.acc[i][j + 1][4 * g], t.acc[i][j + 1][4 * g + 1], t.acc[i][j + 1][4 * g + 2],
                            t.acc[i][j + 1][4 * g + 3]);
      }
      const int col = n0 + t.n_of(j, 0) - 4 * ((threadIdx.x >> 5) & 1);
      stage_block32(st, 0, v0);
      stage_block32(st, 1, v1);
      store_staged32(st, out + (size_t)(row_base + m0) * ld + col, ld, mrows - m0);
    }
  }
}

// the one-round form where the last stage buffer allows it
template <class Cfg>
__device__ __forceinline__ void store_rows_bf16_any(uint16_t* out, int64_t ld, int row_base, int mrows, int n0,
                                                    int ncols, Acc<Cfg>& t, char* epi) {
  if constexpr (Cfg::RN % 2 == 0 && Cfg::STAGE_BYTES >= Cfg::NW * 4096)
    store_rows_bf16_stage<Cfg>(out, ld, row_base, mrows, n0, ncols, t, epi);
  else
    store_rows_bf16<Cfg>(out, ld, row_base, mrows, n0, ncols, t, epi);
}

// ------------------------------------------------------------------ launch
// One persistent workgroup per CU (the grid is a multiple of 8 for the XCD
// split), fewer when there are fewer tiles than CUs.
inline int cu_count() {
  static int cached[64] = {0};
  int dev = 0;
  if (hipGetDevice(&dev) != hipSuccess || dev < 0 || dev >= 64) return 256;
  if (!cached[dev]) {
    int n = 0;
    if (hipDeviceGetAttribute(&n, hipDeviceAttributeMultiprocessorCount, dev) != hipSuccess || n <= 0) n = 256;
    cached[dev] = n;
  }
  return cached[dev];
}

template <class Op>
inline int run_grid(int tiles_bound) {
  return (std::min(tiles_bound, cu_count() * Op::Cfg::OCC) + 7) & ~7;
}
template <class Op>
inline hipError_t run(const typename Op::Params& p, int tiles_bound, hipStream_t s) {
  if (tiles_bound <= 0) return hipSuccess;
  using Cfg = typename Op::Cfg;
  grouped_gemm_kernel<Op><<<dim3(run_grid<Op>(tiles_bound)), dim3(Cfg::THREADS), 0, s>>>(p);
  return hipGetLastError();
}

}  // namespace smoe

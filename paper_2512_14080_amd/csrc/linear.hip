// The dense matrix product with its epilogue, and its backward pass:
//   H = X W + b,  Y = act(H) + R;   dP = dY act'(H),  dX = dP W^T + G,  dW = X^T dP,
//   db = column sums of dP
// with act none, ReLU, SiLU, GELU (erf) or SwiGLU (W [k,2n], gate columns first).
//
// Few rows are bound by reading W once: its columns stream into registers
// (stream_tile.h), a workgroup per column tile, and where the tiles are fewer than the
// CUs per k slice as well, whose partial sums a second launch joins; and more rows the
// same way by groups of 16 or 32, while that is about one round over the CUs: such a
// product is bound by its start and its chain of loads, which eight waves share.  Large
// ones run on the grouped-GEMM core (one group), in the tiles that take the least rounds
// over the CUs, bound by the matrix pipe.  The epilogue works on the fp32 accumulators:
// bias, activation and residual cost no pass of their own, and Y is rounded once.
//
// Measured: one row, 1024 x 1536 5.5 us; 45 rows, 1000 x 2824, gelu 8.9; 1777 rows,
// 4096 x 14336, swiglu 389 (1.07 PFLOP/s); forward and backward of 8192 rows, 8192 x 4096
// 1.40 ms (1.18 PFLOP/s), of 32768 rows, 1536 x 512, swiglu 343 us.
#include "gemm_epilogue.h"
#include "launch.h"
#include "stream_tile.h"

namespace smoe {

// ---------------------------------------------------------------- activations
__device__ __forceinline__ float act_value(int act, float h) {
  switch (act) {
    case MOE_ACT_RELU: return h < 0.f ? 0.f : h;  // (NaN stays)
    case MOE_ACT_SILU: {
      float s;
      return silu_sig(h, &s);
    }
    case MOE_ACT_GELU: return 0.5f * h * (1.f + erff(h * 0.70710678118654752f));
    default: return h;
  }
}
// d act'(h); ReLU lets d through or not, so that an infinite d of a unit that is off is none
__device__ __forceinline__ float act_grad(int act, float h, float d) {
  switch (act) {
    case MOE_ACT_RELU: return h > 0.f ? d : 0.f;
    case MOE_ACT_SILU: {
      const float s = fast_sigmoid(h);
      return d * (s * (1.f + h * (1.f - s)));
    }
    case MOE_ACT_GELU:
      return d * (0.5f * (1.f + erff(h * 0.70710678118654752f)) + h * 0.39894228040143268f * __expf(-0.5f * h * h));
    default: return d;
  }
}

// Four consecutive output columns from col on of row t: v the product (GATED: v the gate's,
// u the up branch's), without the bias
template <bool GATED>
__device__ __forceinline__ void finish4(const LinearArgs& a, size_t t, int col, f32x4 v, f32x4 u) {
  const int N = GATED ? 2 * a.n : a.n;
  if (a.b) {
    const f32x4 b = *(const f32x4*)(a.b + col);
#pragma unroll
    for (int q = 0; q < 4; ++q) v[q] += b[q];
    if constexpr (GATED) {
      const f32x4 c = *(const f32x4*)(a.b + a.n + col);
#pragma unroll
      for (int q = 0; q < 4; ++q) u[q] += c[q];
    }
  }
  if (a.H) {
    *(u32x2*)(a.H + t * N + col) = pack_bf16x4(v[0], v[1], v[2], v[3]);
    if constexpr (GATED) *(u32x2*)(a.H + t * N + a.n + col) = pack_bf16x4(u[0], u[1], u[2], u[3]);
  }
#pragma unroll
  for (int q = 0; q < 4; ++q) {
    if constexpr (GATED) {
      float s;
      v[q] = silu_sig(v[q], &s) * u[q];
    } else {
      v[q] = act_value(a.act, v[q]);
    }
  }
  if (a.R) {
    const u32x2 r = *(const u32x2*)(a.R + t * a.ldr + col);
    v[0] += bf_lo(r[0]);
    v[1] += bf_hi(r[0]);
    v[2] += bf_lo(r[1]);
    v[3] += bf_hi(r[1]);
  }
  *(u32x2*)(a.Y + t * a.ldy + col) = pack_bf16x4(v[0], v[1], v[2], v[3]);
}

// ---------------------------------------------------------------- few rows
constexpr int kFewWaves8 = 8, kFewThreads = 64 * kFewWaves8;
// grid: column tiles, k slices, groups of MB blocks of 16 / KB rows
template <bool GATED, int KB, int MB>
__global__ __launch_bounds__(kFewThreads, 2) void linear_few_kernel(const LinearArgs a, int slice) {
  using Tile = RowTile<KB>;
  constexpr int CG = Tile::CG, C4 = Tile::COLS / 4, OUT = GATED ? Tile::COLS / 2 : Tile::COLS;
  __shared__ typename Tile::Part part[kFewWaves8];
  const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), lane = lane_id();
  const int n = a.n, N = GATED ? 2 * n : n, c0 = OUT * blockIdx.x;
  const int kbeg = blockIdx.y * slice, kend = min(a.k, kbeg + slice);
  const int c = GATED ? c0 + 8 * (Tile::cg(lane) & (CG / 2 - 1)) : c0 + 8 * Tile::cg(lane);
  const uint32_t wcol = c < n ? 2 * (c + (GATED && Tile::cg(lane) >= CG / 2 ? n : 0)) : kBufferOut;
  const int t0 = Tile::RT * MB * blockIdx.z;
  RowStream<KB, 2> stream;
  stream.prime(buffer_of(a.W, (uint32_t)a.k * N * 2), N * 2, wcol, kbeg, kend, wave, kFewWaves8, lane);
  uint32_t xoff[MB];
#pragma unroll
  for (int b = 0; b < MB; ++b) {
    const int t = t0 + Tile::RT * b + Tile::row(lane);
    xoff[b] = t < a.T ? (uint32_t)t * a.ldx * 2 : kBufferOut;
  }
  f32x4 acc[MB][8];
  zero_acc(acc);
  stream.template add<false>(acc, buffer_of(a.X, ((uint32_t)(a.T - 1) * a.ldx + a.k) * 2), xoff);
#pragma unroll
  for (int b = 0; b < MB; ++b) {
    const int first = t0 + Tile::RT * b;
    if (first >= a.T) break;
    if (b) __syncthreads();
    Tile::put(part[wave], acc[b], lane);
    __syncthreads();
    const int rows = min(Tile::RT, a.T - first);
    if (gridDim.y > 1) {
      for (int i = threadIdx.x; i < rows * C4; i += kFewThreads) {
        const int row = i / C4, c4 = i % C4;
        const int col = GATED ? c0 + 4 * (c4 % (C4 / 2)) : c0 + 4 * c4;
        if (col >= n) continue;
        float* out = a.part + ((size_t)blockIdx.y * a.T + first + row) * N + col + (GATED && c4 >= C4 / 2 ? n : 0);
        *(f32x4*)out = Tile::template sum<kFewWaves8>(part, row, c4);
      }
      continue;
    }
    for (int i = threadIdx.x; i < rows * OUT / 4; i += kFewThreads) {
      const int row = i / (OUT / 4), c4 = i % (OUT / 4), col = c0 + 4 * c4;
      if (col >= n) continue;
      const f32x4 v = Tile::template sum<kFewWaves8>(part, row, c4);
      const f32x4 u = GATED ? Tile::template sum<kFewWaves8>(part, row, c4 + C4 / 2) : v;
      finish4<GATED>(a, first + row, col, v, u);
    }
  }
}

// Partial sums [slices][T][N] joined in slice order, then the epilogue.  grid: rows x, columns y
template <bool GATED>
__global__ __launch_bounds__(256) void linear_join_kernel(const LinearArgs a, int slices) {
  const int N = GATED ? 2 * a.n : a.n, col = 4 * (blockIdx.y * 256 + threadIdx.x);
  const size_t t = blockIdx.x, slab = (size_t)a.T * N;
  if (col >= a.n) return;
  const float* p = a.part + t * N + col;
  f32x4 v = *(const f32x4*)p, u = v;
  if constexpr (GATED) u = *(const f32x4*)(p + a.n);
#pragma unroll 4
  for (int s = 1; s < slices; ++s) {
    const f32x4 x = *(const f32x4*)(p + s * slab);
#pragma unroll
    for (int q = 0; q < 4; ++q) v[q] += x[q];
    if constexpr (GATED) {
      const f32x4 y = *(const f32x4*)(p + s * slab + a.n);
#pragma unroll
      for (int q = 0; q < 4; ++q) u[q] += y[q];
    }
  }
  finish4<GATED>(a, t, col, v, u);
}

// ---------------------------------------------------------------- tiles
// 32 columns of a row from col on (8 consecutive ones of each lane's 16-byte pieces), n of
// them in all, a multiple of 8: the residual in the accumulator layout, and a store
__device__ __forceinline__ void load_cols(const uint16_t* row, int col, int n, u32x2 (&v)[4]) {
  const int hi = (threadIdx.x >> 5) & 1;
#pragma unroll
  for (int g = 0; g < 4; g += 2) {
    const int c = col + 8 * g + 8 * hi;
    const u32x4 x = c < n ? *(const u32x4*)(row + c) : u32x4{0, 0, 0, 0};
    const auto a = __builtin_amdgcn_permlane32_swap(x[0], x[2], false, false);
    const auto b = __builtin_amdgcn_permlane32_swap(x[1], x[3], false, false);
    v[g] = u32x2{a[0], b[0]};
    v[g + 1] = u32x2{a[1], b[1]};
  }
}
__device__ __forceinline__ void store_cols(uint16_t* row, int col, int n, const u32x2 (&v)[4]) {
  const int hi = (threadIdx.x >> 5) & 1;
#pragma unroll
  for (int g = 0; g < 4; g += 2) {
    const auto a = __builtin_amdgcn_permlane32_swap(v[g][0], v[g + 1][0], false, false);
    const auto b = __builtin_amdgcn_permlane32_swap(v[g][1], v[g + 1][1], false, false);
    const int c = col + 8 * g + 8 * hi;
    if (c < n) *(u32x4*)(row + c) = u32x4{a[0], b[0], a[1], b[1]};
  }
}
// the wave's staged 32 x 64 block (stage_block32) to columns col .. of n
__device__ __forceinline__ void store_staged_cols(const char* wl, uint16_t* row0, int64_t ld, int rows_valid, int col, int n) {
  asm volatile("" ::: "memory");  // the staged writes of every lane precede these reads
  const int lane = epilogue_lane();
#pragma unroll
  for (int t = 0; t < 4; ++t) {
    const int R = 8 * t + (lane >> 3), C = lane & 7;
    const u32x4 x = *(const u32x4*)(wl + R * 128 + ((C ^ ((R >> 1) & 7)) << 4));
    if (R < rows_valid && col + 8 * C < n) __builtin_nontemporal_store(x, (u32x4*)(row0 + R * ld + col + 8 * C));
  }
  asm volatile("" ::: "memory");  // and precede the next writes to the area
}
template <class Cfg>
constexpr bool kWholeLines = Cfg::STAGE_BYTES >= Cfg::NW * 4096;

// id -> tile of M x N in blocks (tile_order); splits: the k chunk is the slowest index
template <class Cfg>
__device__ __forceinline__ bool dense_tile(int M, int N, int K, int splits, int chunk, int id, TileInfo& ti) {
  const int mt = (M + Cfg::BM - 1) / Cfg::BM, nt = (N + Cfg::BN - 1) / Cfg::BN;
  const int split = id / (mt * nt);
  if (split >= splits) return false;
  int m, n;
  tile_order(id - split * mt * nt, mt, nt, nt >= 8 ? 4 : 1, &m, &n);
  ti.e = split;
  ti.m0 = ti.row_base = m * Cfg::BM;
  ti.n0 = n * Cfg::BN;
  ti.mrows = min((int)Cfg::BM, M - ti.m0);
  ti.ncols = min((int)Cfg::BN, N - ti.n0);
  ti.k_begin = split * chunk;
  ti.k_len = min(chunk, K - ti.k_begin);
  return true;
}

// The output columns [col0, col0 + cols).  PART: fp32 partial sums of a k chunk to a.part, else
// the epilogue
// (the activation is a constant: a choice among them in the unrolled epilogue kept the
// accumulators out of the registers)
template <class Cfg_, int ACT, bool TAIL, bool PART>
struct OpLinear {
  using Cfg = Cfg_;
  static constexpr bool GATED = ACT == MOE_ACT_SWIGLU;
  static constexpr int M_MODE = TAIL ? ROWS_TAIL : ROWS, N_MODE = KOUTER;
  static constexpr int Wn = Cfg::BN / Cfg::WN, RC = GATED ? Cfg::RN / 2 : Cfg::RN;  // output blocks of a wave
  static constexpr bool LINES = kWholeLines<Cfg> && RC % 2 == 0;
  static constexpr int EPI_LDS = 0;
  // of a full tile: Y's alone
  static constexpr int EPI_STORES = PART ? Cfg::RM * Cfg::RN * 4 : LINES ? Cfg::RM * (RC / 2) * 4 : Cfg::RM * RC * 2;
  struct Params { LinearArgs a; int splits, chunk; };
  struct ColMap {  // (as the layer's up-projection: a wave holds gate columns and the matching up columns)
    int c0, n;
    __device__ __forceinline__ int operator()(int c) const {
      if constexpr (!GATED) return c0 + c;
      const int w = c / Wn, q = c % Wn;
      return q < Wn / 2 ? c0 + w * (Wn / 2) + q : n + c0 + w * (Wn / 2) + (q - Wn / 2);
    }
  };
  static __device__ int columns(const Params& p) { return GATED ? 2 * p.a.n : p.a.n; }  // of W
  // (GATED: tiles of BN / 2 gate columns, counted as BN of twice the columns of whole tiles)
  static __device__ int tile_columns(const Params& p) {
    return GATED ? (p.a.cols + Cfg::BN / 2 - 1) / (Cfg::BN / 2) * Cfg::BN : p.a.cols;
  }
  static __device__ int count(const Params& p, int*) {
    return p.splits * ((p.a.T + Cfg::BM - 1) / Cfg::BM) * ((tile_columns(p) + Cfg::BN - 1) / Cfg::BN);
  }
  static __device__ bool tile(const Params& p, int id, TileInfo& ti, int*) {
    const bool ok = dense_tile<Cfg>(p.a.T, tile_columns(p), p.a.k, p.splits, p.chunk, id, ti);
    if (GATED && (ti.n0 + Cfg::BN) / 2 > p.a.cols) ti.ncols = 0;  // (not a full tile)
    return ok;
  }
  static __device__ int first_col(const Params& p, const TileInfo& ti) { return p.a.col0 + (GATED ? ti.n0 / 2 : ti.n0); }
  template <class Side>
  static __device__ void init_m(const Params& p, const TileInfo& ti, Side& s) {
    s.init(p.a.X + ti.k_begin, p.a.ldx, nullptr, ti.row_base, ti.mrows);
    if constexpr (TAIL) s.k_len = ti.k_len;
  }
  static __device__ void init_n(const Params& p, const TileInfo& ti, KOuterSide<Cfg::BN, Cfg::BK, Cfg::NW>& s) {
    s.init(p.a.W, columns(p), nullptr, ti.k_begin, ti.k_len, columns(p), ColMap{first_col(p, ti), p.a.n});
  }
  static __device__ void epilogue(const Params& p, const TileInfo& ti, Acc<Cfg>& t, char* epi) {
    const LinearArgs& a = p.a;
    const int n = a.n, end = a.col0 + a.cols, N = columns(p), wn = t.wave_n(), lane = epilogue_lane();
    const int wm0 = Cfg::wave_m(threadIdx.x >> 6) * (Cfg::BM / Cfg::WM);
    const int c0 = first_col(p, ti) + wn * (GATED ? Wn / 2 : Wn);  // this wave's first output column
    if constexpr (PART) {
#pragma unroll
      for (int i = 0; i < Cfg::RM; ++i) {
        const int m = wm0 + 32 * i + (lane & 31);
        if (m >= ti.mrows) continue;
        float* out = a.part + ((size_t)ti.e * a.T + ti.row_base + m) * N;
#pragma unroll
        for (int j = 0; j < Cfg::RN; ++j)
#pragma unroll
          for (int g = 0; g < 4; ++g) {
            const int c = c0 + 32 * (j % RC) + 8 * g + 4 * (lane >> 5);
            if (c >= end) continue;
            f32x4 v;
#pragma unroll
            for (int q = 0; q < 4; ++q) v[q] = t.acc[i][j][4 * g + q];
            *(f32x4*)(out + c + (j >= RC ? n : 0)) = v;
          }
      }
      return;
    }
    if (a.b) {
#pragma unroll
      for (int j = 0; j < Cfg::RN; ++j)
#pragma unroll
        for (int g = 0; g < 4; ++g) {
          const int c = c0 + 32 * (j % RC) + 8 * g + 4 * (lane >> 5);
          if (c >= end) continue;
          const f32x4 b = *(const f32x4*)(a.b + c + (j >= RC ? n : 0));
#pragma unroll
          for (int i = 0; i < Cfg::RM; ++i)
#pragma unroll
            for (int q = 0; q < 4; ++q) t.acc[i][j][4 * g + q] += b[q];
        }
    }
    // the last stage's buffer is idle until the next tile's first barrier
    char* st = LINES ? epi - Cfg::STAGE_BYTES + (threadIdx.x >> 6) * 4096 : nullptr;
#pragma unroll
    for (int i = 0; i < Cfg::RM; ++i) {
      const int m0 = wm0 + 32 * i, m = m0 + (lane & 31);
      if (m0 >= ti.mrows) continue;
      const size_t r0 = (size_t)ti.row_base + m0;
      const size_t row = (size_t)ti.row_base + min(m, ti.mrows - 1);  // (this lane's, for its loads)
      auto pack = [&](int j, u32x2(&v)[4]) {
#pragma unroll
        for (int g = 0; g < 4; ++g)
          v[g] = pack_bf16x4(t.acc[i][j][4 * g], t.acc[i][j][4 * g + 1], t.acc[i][j][4 * g + 2], t.acc[i][j][4 * g + 3]);
      };
      // block jj of the outputs as bf16
      auto values = [&](int jj, u32x2(&v)[4]) {
        u32x2 r[4] = {};
        const int col = c0 + 32 * jj;
        if (a.R) load_cols(a.R + row * a.ldr, col, end, r);
#pragma unroll
        for (int g = 0; g < 4; ++g) {
          float y[4];
#pragma unroll
          for (int q = 0; q < 4; ++q) {
            const float h = t.acc[i][jj][4 * g + q];
            if constexpr (GATED) {
              float s;
              y[q] = silu_sig(h, &s) * t.acc[i][jj + RC][4 * g + q];
            } else {
              y[q] = act_value(ACT, h);
            }
          }
          y[0] += bf_lo(r[g][0]);
          y[1] += bf_hi(r[g][0]);
          y[2] += bf_lo(r[g][1]);
          y[3] += bf_hi(r[g][1]);
          v[g] = pack_bf16x4(y[0], y[1], y[2], y[3]);
        }
      };
      if constexpr (LINES) {
#pragma unroll
        for (int jj = 0; jj < RC; jj += 2) {
          const int col = c0 + 32 * jj;
          if (col >= end) continue;
          u32x2 v[4];
          if (a.H) {
#pragma unroll
            for (int half = 0; half < (GATED ? 2 : 1); ++half) {
              pack(jj + half * RC, v);
              stage_block32(st, 0, v);
              pack(jj + 1 + half * RC, v);
              stage_block32(st, 1, v);
              store_staged_cols(st, a.H + r0 * N + half * n, N, ti.mrows - m0, col, end);
            }
          }
          values(jj, v);
          stage_block32(st, 0, v);
          values(jj + 1, v);
          stage_block32(st, 1, v);
          store_staged_cols(st, a.Y + r0 * a.ldy, a.ldy, ti.mrows - m0, col, end);
        }
      } else {
#pragma unroll
        for (int jj = 0; jj < RC; ++jj) {
          const int col = c0 + 32 * jj;
          if (col >= end) continue;
          u32x2 v[4];
          if (a.H) {
            pack(jj, v);
            if (m < ti.mrows) store_cols(a.H + row * N, col, end, v);
            if constexpr (GATED) {
              pack(jj + RC, v);
              if (m < ti.mrows) store_cols(a.H + row * N + n, col, end, v);
            }
          }
          values(jj, v);
          if (m < ti.mrows) store_cols(a.Y + row * a.ldy, col, end, v);
        }
      }
    }
  }
};

// dX [T,k] = dP [T,N] W^T (+ G): as OpLinear's plain form with k for the columns, N for the
// reduction, W's rows for the N side
template <class Cfg_, bool TAIL, bool PART>
struct OpLinearDX {
  using Cfg = Cfg_;
  using Fwd = OpLinear<Cfg_, MOE_ACT_NONE, TAIL, PART>;
  static constexpr int M_MODE = TAIL ? ROWS_TAIL : ROWS, N_MODE = M_MODE;
  static constexpr int EPI_LDS = 0, EPI_STORES = Fwd::EPI_STORES;
  using Params = typename Fwd::Params;  // X: dP, k: N; n: k; R: G; Y: dX
  static __device__ int count(const Params& p, int* sh) { return Fwd::count(p, sh); }
  static __device__ bool tile(const Params& p, int id, TileInfo& ti, int* sh) { return Fwd::tile(p, id, ti, sh); }
  template <class Side>
  static __device__ void init_m(const Params& p, const TileInfo& ti, Side& s) { Fwd::init_m(p, ti, s); }
  template <class Side>
  static __device__ void init_n(const Params& p, const TileInfo& ti, Side& s) {
    s.init(p.a.W + ti.k_begin, p.a.k, nullptr, p.a.col0 + ti.n0, ti.ncols);
    if constexpr (TAIL) s.k_len = ti.k_len;
  }
  static __device__ void epilogue(const Params& p, const TileInfo& ti, Acc<Cfg>& t, char* epi) {
    Fwd::epilogue(p, ti, t, epi);
  }
};

// dW [k,N] = X^T dP over chunks of the T rows; PART: fp32 slabs [chunk][k][N]
template <class Cfg_, bool PART>
struct OpLinearDW {
  using Cfg = Cfg_;
  static constexpr int M_MODE = KOUTER, N_MODE = KOUTER, EPI_LDS = 0;
  static_assert(kWholeLines<Cfg> && Cfg::RN % 2 == 0, "stored in whole lines");
  struct Params { LinearArgs a; const uint16_t* dP; int64_t ldp; uint16_t* dW; int N, splits, chunk; };
  static __device__ int count(const Params& p, int*) {
    return p.splits * ((p.a.k + Cfg::BM - 1) / Cfg::BM) * ((p.N + Cfg::BN - 1) / Cfg::BN);
  }
  static __device__ bool tile(const Params& p, int id, TileInfo& ti, int*) {
    return dense_tile<Cfg>(p.a.k, p.N, p.a.T, p.splits, p.chunk, id, ti);
  }
  static __device__ void init_m(const Params& p, const TileInfo& ti, KOuterSide<Cfg::BM, Cfg::BK, Cfg::NW>& s) {
    s.init(p.a.X, p.a.ldx, nullptr, ti.k_begin, ti.k_len, p.a.k, ColOffset{ti.m0});
  }
  static __device__ void init_n(const Params& p, const TileInfo& ti, KOuterSide<Cfg::BN, Cfg::BK, Cfg::NW>& s) {
    s.init(p.dP, p.ldp, nullptr, ti.k_begin, ti.k_len, p.N, ColOffset{ti.n0});
  }
  static __device__ void epilogue(const Params& p, const TileInfo& ti, Acc<Cfg>& t, char* epi) {
    // (the limits are formed here: held across the k loop they cost registers)
    const int mrows = p.a.k - ti.m0, ncols = p.N - ti.n0;
    if constexpr (PART) {
      store_part_f32<Cfg>(p.a.part + (size_t)ti.e * p.a.k * p.N, p.N, ti.m0, ti.n0, mrows, ncols, t);
      return;
    }
    const int wm0 = Cfg::wave_m(threadIdx.x >> 6) * (Cfg::BM / Cfg::WM);
    const int c0 = ti.n0 + t.wave_n() * (Cfg::BN / Cfg::WN);
    char* st = epi - Cfg::STAGE_BYTES + (threadIdx.x >> 6) * 4096;
#pragma unroll
    for (int i = 0; i < Cfg::RM; ++i) {
      const int m0 = wm0 + 32 * i;
      if (m0 >= mrows) continue;
      auto pack = [&](int j, u32x2(&v)[4]) {
#pragma unroll
        for (int g = 0; g < 4; ++g)
          v[g] = pack_bf16x4(t.acc[i][j][4 * g], t.acc[i][j][4 * g + 1], t.acc[i][j][4 * g + 2], t.acc[i][j][4 * g + 3]);
      };
#pragma unroll
      for (int j = 0; j < Cfg::RN; j += 2) {
        const int col = c0 + 32 * j;
        if (col >= p.N) continue;
        u32x2 v[4];
        pack(j, v);
        stage_block32(st, 0, v);
        pack(j + 1, v);
        stage_block32(st, 1, v);
        store_staged_cols(st, p.dW + (size_t)(ti.m0 + m0) * p.N, p.N, mrows - m0, col, p.N);
      }
    }
  }
};

// ---------------------------------------------------------------- dP and db
// A workgroup takes 256 columns (32 threads of 8) of `rows` rows; dP is formed where the
// product has an activation, and the column sums of the rows in fp32, from the values before
// their rounding.  grid: `blocks` column blocks of the (gate's) columns for each row chunk.
// dP is rounded to bf16, what the products' instruction takes: in two bf16 parts dX and dW
// would be twice the work.  They are 2.3e-3 off the gradients in 64 bits so (1003 rows of 904 x
// 1528, silu), 1.7e-3 without an activation.
template <bool GATED>
__global__ __launch_bounds__(256) void linear_dp_kernel(const LinearBwdArgs a, int blocks, int rows, float* __restrict__ sums) {
  const int chunk = blockIdx.x / blocks, first = 256 * (blockIdx.x - chunk * blocks);
  const int c = threadIdx.x & 31, rl = threadIdx.x >> 5, col = first + 8 * c;
  const int n = a.n, N = GATED ? 2 * n : n;
  const int64_t t0 = (int64_t)chunk * rows;
  float s[GATED ? 2 : 1][8] = {};
  if (col < n)
#pragma unroll 2
    for (int r = rl; r < rows && t0 + r < a.T; r += 8) {
      const size_t t = t0 + r;
      const u32x4 y = *(const u32x4*)(a.dY + t * a.ldy + col);
      float d[8], e[8];
#pragma unroll
      for (int q = 0; q < 4; ++q) {
        d[2 * q] = bf_lo(y[q]);
        d[2 * q + 1] = bf_hi(y[q]);
      }
      if (a.dP) {
        const u32x4 h = *(const u32x4*)(a.H + t * N + col);
        u32x4 o;
        if constexpr (GATED) {
          const u32x4 u = *(const u32x4*)(a.H + t * N + n + col);
          u32x4 o2;
#pragma unroll
          for (int q = 0; q < 8; ++q) {
            const float g = q & 1 ? bf_hi(h[q / 2]) : bf_lo(h[q / 2]), up = q & 1 ? bf_hi(u[q / 2]) : bf_lo(u[q / 2]);
            float sg;
            const float sl = silu_sig(g, &sg);
            e[q] = d[q] * sl;
            d[q] = d[q] * up * sg * (1.f + g * (1.f - sg));
          }
#pragma unroll
          for (int q = 0; q < 4; ++q) o2[q] = pack_bf2(e[2 * q], e[2 * q + 1]);
          *(u32x4*)(a.dP + t * N + n + col) = o2;
        } else {
#pragma unroll
          for (int q = 0; q < 8; ++q) d[q] = act_grad(a.act, q & 1 ? bf_hi(h[q / 2]) : bf_lo(h[q / 2]), d[q]);
        }
#pragma unroll
        for (int q = 0; q < 4; ++q) o[q] = pack_bf2(d[2 * q], d[2 * q + 1]);
        *(u32x4*)(a.dP + t * N + col) = o;
      }
#pragma unroll
      for (int q = 0; q < 8; ++q) {
        s[0][q] += d[q];
        if constexpr (GATED) s[1][q] += e[q];
      }
    }
  if (!sums) return;
  __shared__ float lds[8][GATED ? 2 : 1][256];
#pragma unroll
  for (int h = 0; h < (GATED ? 2 : 1); ++h)
#pragma unroll
    for (int q = 0; q < 8; ++q) lds[rl][h][8 * c + q] = s[h][q];
  __syncthreads();
  const int out = first + threadIdx.x;
  if (out >= n) return;
#pragma unroll
  for (int h = 0; h < (GATED ? 2 : 1); ++h) {
    float v = 0.f;
#pragma unroll
    for (int r = 0; r < 8; ++r) v += lds[r][h][threadIdx.x];
    sums[(size_t)chunk * N + h * n + out] = v;
  }
}

// The last sums, in a fixed order: dW from its slabs (workgroups below `wgs`), db from its row
// chunks (the others: 32 columns each, eight threads of a column's chunks)
__global__ __launch_bounds__(256) void linear_sums_kernel(const float* __restrict__ slabs, int splits, int64_t MN,
                                                          uint16_t* __restrict__ dW, int wgs,
                                                          const float* __restrict__ sums, int chunks, int N,
                                                          float* __restrict__ db) {
  if ((int)blockIdx.x < wgs) {
    for (int64_t i = 4 * ((int64_t)blockIdx.x * 256 + threadIdx.x); i < MN; i += 4 * 256 * (int64_t)wgs) {
      f32x4 v = *(const f32x4*)(slabs + i);
#pragma unroll 4
      for (int s = 1; s < splits; ++s) {
        const f32x4 x = *(const f32x4*)(slabs + s * MN + i);
#pragma unroll
        for (int q = 0; q < 4; ++q) v[q] += x[q];
      }
      *(u32x2*)(dW + i) = pack_bf16x4(v[0], v[1], v[2], v[3]);
    }
    return;
  }
  __shared__ float lds[8][33];
  const int c = threadIdx.x & 31, r = threadIdx.x >> 5, col = ((int)blockIdx.x - wgs) * 32 + c;
  float v = 0.f;
  if (col < N)
#pragma unroll 8  // (loads in flight; added in their order)
    for (int q = r; q < chunks; q += 8) v += sums[(size_t)q * N + col];
  lds[r][c] = v;
  __syncthreads();
  if (r == 0 && col < N) {
#pragma unroll
    for (int q = 1; q < 8; ++q) v += lds[q][c];
    db[col] = v;
  }
}

// ---------------------------------------------------------------- host
using L256x256 = GemmCfg<256, 256, 4, 2, 2>;           // 64 x 128 a wave
using L256x128 = GemmCfg<256, 128, 4, 2, 3>;
using L128x128 = GemmCfg<128, 128, 4, 2, 2, kBK, 2>;   // two workgroups to a CU
using L128x128d = GemmCfg<128, 128, 4, 2, 4>;          // one, three stages ahead
using D256x256 = GemmCfg<256, 256, 2, 4, 2>;
using D128x128 = GemmCfg<128, 128, 4, 2, 2, kBK, 2>;
using D128x128d = GemmCfg<128, 128, 4, 2, 4>;

constexpr int kLinearMaxSlices = 16;
constexpr size_t kSlabBytes = (size_t)256 << 20;
constexpr int kCus = 256;  // (a size of workspaces: not the device's own count)

static int64_t ceil_div(int64_t a, int64_t b) { return (a + b - 1) / b; }
// rows of a workgroup of linear_dp_kernel: 64, fewer where that leaves CUs idle; but all of up to
// 16 rows, whose sums are then db itself (a step of one row, k = 1024, n = 1536, silu, with bias:
// 30.0 us, 26.7 so; 56 rows of k = 832, n = 1024 would take 36.7, not 29.2)
static int dp_rows(int T, int64_t N) {
  if (T <= 16) return 16;
  int rows = 64;
  while (rows > 8 && ceil_div(T, rows) * ceil_div(N, 256) < 4 * kCus) rows /= 2;
  return rows;
}

// Forward (and dX): M x N outputs over K.  few: streaming, with kb k blocks of a step and mb
// row blocks; else tiles of bm x bn.  slices: of K, whose partial sums are joined.  deep: three
// stages of loads ahead of the products, where a workgroup has its CU to itself.
struct LinearPlan { bool few; int kb, mb, bm, bn; bool deep; int slices, chunk; double cost; };

// Rounds over the CUs times a tile's time for a k step (a 256 x 256 tile's is 100 units of 14.6 ns:
// tiled_us), and what the join of slices costs: a launch, and its reading.
static LinearPlan tiled_plan(int64_t M, int64_t N, int64_t K, int most_slices = kLinearMaxSlices) {
  struct Shape { int bm, bn; bool deep; int slots, step; };
  static const Shape shapes[] = {{256, 256, false, kCus, 100}, {256, 128, false, kCus, 60}, {128, 128, false, 2 * kCus, 72},
                                 {128, 128, true, kCus, 36}};
  LinearPlan best{};
  for (const Shape& t : shapes) {
    const int64_t tiles = ceil_div(M, t.bm) * ceil_div(N, t.bn);
    for (int slices = 1; slices <= most_slices; slices *= 2) {
      if (slices > 1 && (K < 512 * slices || (int64_t)slices * M * N * 4 > (int64_t)kSlabBytes)) break;
      const int64_t steps = ceil_div(ceil_div(K, slices), kBK);
      double cost = ceil_div(tiles * slices, t.slots) * (double)t.step * (steps + 4);
      if (slices > 1) cost += 250 + slices * M * N * 4 / 70e3;
      if (best.cost == 0 || cost < 0.97 * best.cost)
        best = {false, 0, 0, t.bm, t.bn, t.deep, slices, slices == 1 ? (int)K : (int)(steps * kBK), cost};
    }
  }
  best.slices = (int)ceil_div(K, best.chunk);
  return best;
}
// The columns that whole rounds of 256 x 256 tiles take, where the others are better off in a
// launch of their own (T = 1777, k = 4096, n = 14336 gated: 784 tiles are 3 rounds and 16 more);
// 0: all in one.
static int64_t whole_rounds(int64_t M, int64_t N, int64_t K, const LinearPlan& all) {
  if (all.bn != 256 || all.slices > 1) return 0;
  const int64_t mt = ceil_div(M, 256), nt = ceil_div(N, 256), rounds = mt * nt / kCus;
  if (rounds == 0 || mt * nt % kCus == 0) return 0;
  const int64_t cols = rounds * kCus / mt * 256;
  if (cols == 0 || cols >= N) return 0;
  const LinearPlan rest = tiled_plan(M, N - cols, K, 1);  // (no partial sums for a part of the columns)
  return rounds * 100. * (ceil_div(K, kBK) + 4) + rest.cost + 200 < 0.97 * all.cost ? cols : 0;
}

// More than 16 rows streamed, in groups of 16 or 32 that each read the weights.  In us, fitted: a
// start; the larger of a workgroup's reading of its columns (a CU: 60 GB/s, 50 with two row
// blocks; 1.7 us at least), in rounds, and all reads (5.5 TB/s; a group's after the first are
// found nearer, at four times that); and the join.
static double join_us(int slices, int64_t T, int64_t N) { return slices > 1 ? 2.5 + 0.12 * slices + slices * T * N * 4 / 4e6 : 0; }
static void stream_plan(int T, int64_t k, int64_t N, LinearPlan& best) {
  for (int mb = 1; mb <= 2; ++mb) {
    const int64_t groups = ceil_div(T, 16 * mb), tiles = ceil_div(N, 128) * groups;
    const double reads = (1 + (groups - 1) / 4.) * k * N * 2 / 5.5e6;
    for (int slices = 1; slices <= kLinearMaxSlices; slices *= 2) {
      if (slices > 1 && k < 256 * slices) break;
      const int64_t chunk = ceil_div(ceil_div(k, slices), 128) * 128;
      const double rounds = ceil_div(tiles * slices, kCus) * std::max(1.7, chunk * (mb == 1 ? 4.3 : 5.3) / 1024);
      const double us = (mb == 1 ? 3.1 : 4.4) + std::max(rounds, reads) + join_us(slices, T, N);
      if (us < 0.97 * best.cost) best = {true, 1, mb, 0, 0, false, (int)ceil_div(k, chunk), (int)chunk, us};
    }
  }
}
// the same of a tiled plan, whose own cost compares tiles only
static double tiled_us(const LinearPlan& p, int64_t T, int64_t N) {
  const double join = p.slices > 1 ? 250 + p.slices * T * N * 4 / 70e3 : 0;
  return 2.4 + 0.0146 * (p.cost - join) + join_us(p.slices, T, N);
}
static LinearPlan forward_plan(int T, int k, int n, int act, int64_t ldx) {
  const int64_t N = act == MOE_ACT_SWIGLU ? 2 * (int64_t)n : n;
  const bool fits = (int64_t)k * N * 2 <= INT32_MAX && (T * ldx + k) * 2 <= INT32_MAX;
  if (T > 16 || !fits) {
    LinearPlan best = tiled_plan(T, N, k);
    // T = 45, k = 1000, n = 2824: 8.5 us, 13.0 in tiles; 256 rows 12.7 and 16.2, 512 22.5 and
    // 16.3; T = 512, k = 512, n = 512 5.4 and 10.6; T = 40, k = 4096, n = 14336 41 and 27
    best.cost = tiled_us(best, T, N);
    if (fits && T <= 1 << 14) stream_plan(T, k, N, best);
    return best;
  }
  // narrower tiles for fewer rows, while that gives up to a workgroup to two CUs
  int kb = 1;
  while (kb < 4 && 16 / (2 * kb) >= T && ceil_div(N, 128 / kb) < 128) kb *= 2;
  const int64_t tiles = ceil_div(N, 128 / kb);
  int slices = 1;
  // k slices where a workgroup would read more than 256 KB on its own
  while (2 * slices * tiles <= kCus && 2 * slices <= kLinearMaxSlices && (int64_t)(k / slices) * (256 / kb) > 256 * 1024) slices *= 2;
  const int chunk = (int)ceil_div(ceil_div(k, slices), 128) * 128;
  slices = (int)ceil_div(k, chunk);
  return {true, kb, 1, 0, 0, false, slices, chunk, 0};
}

static LinearPlan dx_plan(int T, int k, int64_t N) { return tiled_plan(T, k, N); }
struct DwPlan { int bm; bool deep; int splits, chunk; };
static DwPlan dw_plan(int T, int64_t k, int64_t N) {
  struct Shape { int bm; bool deep; int slots, step; };
  static const Shape shapes[] = {{256, false, kCus, 100}, {128, false, 2 * kCus, 72}, {128, true, kCus, 38}};
  DwPlan best{};
  double least = 0;
  for (const Shape& t : shapes) {
    const int64_t tiles = ceil_div(k, t.bm) * ceil_div(N, t.bm);
    for (int splits = 1; splits <= 2 * kLinearMaxSlices; ++splits) {
      if (splits > 1 && (T < 256 * splits || splits * k * N * 4 > (int64_t)kSlabBytes)) break;
      const int64_t steps = ceil_div(ceil_div(T, splits), kBK);
      double cost = ceil_div(tiles * splits, t.slots) * (double)t.step * (steps + 5);
      if (splits > 1) cost += 250 + splits * k * N * 4 / 70e3;
      if (least == 0 || cost < 0.97 * least) {
        best = {t.bm, t.deep, splits, splits == 1 ? T : (int)(steps * kBK)};
        least = cost;
      }
    }
  }
  best.splits = (int)ceil_div(T, best.chunk);
  return best;
}

size_t linear_fwd_part_bytes(int T, int k, int n, int act, int64_t ldx) {
  const LinearPlan p = forward_plan(T, k, n, act, ldx);
  return p.slices > 1 ? (size_t)p.slices * T * (act == MOE_ACT_SWIGLU ? 2 * (size_t)n : n) * 4 : 0;
}
size_t linear_dx_part_bytes(int T, int k, int64_t N) {
  const LinearPlan p = dx_plan(T, k, N);
  return p.slices > 1 ? (size_t)p.slices * T * k * 4 : 0;
}
size_t linear_dw_part_bytes(int T, int k, int64_t N) {
  const DwPlan p = dw_plan(T, k, N);
  return p.splits > 1 ? (size_t)p.splits * k * N * 4 : 0;
}
size_t linear_db_part_bytes(int T, int64_t N) { return (size_t)ceil_div(T, dp_rows(T, N)) * N * 4; }

template <bool GATED>
static hipError_t join(const LinearArgs& a, int slices, hipStream_t s) {
  linear_join_kernel<GATED><<<dim3(a.T, (unsigned)ceil_div(a.n, 1024)), 256, 0, s>>>(a, slices);
  return hipGetLastError();
}

template <bool GATED, int KB, int MB>
static hipError_t run_few(const LinearArgs& a, const LinearPlan& p, hipStream_t s) {
  constexpr int out = RowTile<KB>::COLS / (GATED ? 2 : 1);
  linear_few_kernel<GATED, KB, MB><<<dim3((unsigned)ceil_div(a.n, out), p.slices, (unsigned)ceil_div(a.T, RowTile<KB>::RT * MB)), kFewThreads, 0, s>>>(a,
                                                                                                           p.chunk);
  return hipGetLastError();
}
template <bool GATED>
static hipError_t few_rows(const LinearArgs& a, const LinearPlan& p, hipStream_t s) {
  hipError_t e;
  if (p.kb == 4)
    e = run_few<GATED, 4, 1>(a, p, s);
  else if (p.kb == 2)
    e = run_few<GATED, 2, 1>(a, p, s);
  else if (p.mb == 1)
    e = run_few<GATED, 1, 1>(a, p, s);
  else
    e = run_few<GATED, 1, 2>(a, p, s);
  return e == hipSuccess && p.slices > 1 ? join<GATED>(a, p.slices, s) : e;
}

// the tiled product of plan p; tail: K is no multiple of the stage depth
template <template <class, bool, bool> class Op>
static hipError_t run_tiles(const LinearArgs& a, const LinearPlan& p, int64_t N, bool tail, hipStream_t s) {
  const int tiles = (int)(p.slices * ceil_div(a.T, p.bm) * ceil_div(N, p.bn));
  auto go = [&](auto cfg) {
    using C = decltype(cfg);
    if (p.slices > 1)
      return tail ? run<Op<C, true, true>>({a, p.slices, p.chunk}, tiles, s) : run<Op<C, false, true>>({a, p.slices, p.chunk}, tiles, s);
    return tail ? run<Op<C, true, false>>({a, 1, p.chunk}, tiles, s) : run<Op<C, false, false>>({a, 1, p.chunk}, tiles, s);
  };
  if (p.bn == 256) return go(L256x256{});
  if (p.bm == 256) return go(L256x128{});
  return p.deep ? go(L128x128d{}) : go(L128x128{});
}
// all columns, or those of whole rounds and the others
template <template <class, bool, bool> class Op>
static hipError_t run_columns(LinearArgs a, int64_t N, int per_col, bool tail, hipStream_t s) {
  a.col0 = 0;
  a.cols = (int)(N / per_col);
  const LinearPlan all = tiled_plan(a.T, N, a.k);
  const int64_t cols = whole_rounds(a.T, N, a.k, all);
  if (cols == 0) return run_tiles<Op>(a, all, per_col * ceil_div(a.cols, all.bn / per_col) * (all.bn / per_col), tail, s);
  const int n = a.cols;
  a.cols = (int)(cols / per_col);
  const hipError_t e = run_tiles<Op>(a, all, cols, tail, s);
  if (e != hipSuccess) return e;
  a.col0 = a.cols;
  a.cols = n - a.col0;
  const LinearPlan rest = tiled_plan(a.T, N - cols, a.k, 1);
  return run_tiles<Op>(a, rest, per_col * ceil_div(a.cols, rest.bn / per_col) * (rest.bn / per_col), tail, s);
}
template <int ACT>
struct LinearOf {
  template <class C, bool TAIL, bool PART>
  using Op = OpLinear<C, PART && ACT != MOE_ACT_SWIGLU ? MOE_ACT_NONE : ACT, TAIL, PART>;
};

hipError_t launch_linear_fwd(const LinearArgs& a, hipStream_t s) {
  const bool gated = a.act == MOE_ACT_SWIGLU;
  const LinearPlan p = forward_plan(a.T, a.k, a.n, a.act, a.ldx);
  if (p.few) return gated ? few_rows<true>(a, p, s) : few_rows<false>(a, p, s);
  const bool tail = a.k % kBK != 0;
  const int per_col = gated ? 2 : 1;  // columns of W to an output column
  const int64_t N = (int64_t)per_col * a.n;
  hipError_t e;
  switch (a.act) {
    case MOE_ACT_RELU: e = run_columns<LinearOf<MOE_ACT_RELU>::Op>(a, N, per_col, tail, s); break;
    case MOE_ACT_SILU: e = run_columns<LinearOf<MOE_ACT_SILU>::Op>(a, N, per_col, tail, s); break;
    case MOE_ACT_GELU: e = run_columns<LinearOf<MOE_ACT_GELU>::Op>(a, N, per_col, tail, s); break;
    case MOE_ACT_SWIGLU: e = run_columns<LinearOf<MOE_ACT_SWIGLU>::Op>(a, N, per_col, tail, s); break;
    default: e = run_columns<LinearOf<MOE_ACT_NONE>::Op>(a, N, per_col, tail, s);
  }
  if (e != hipSuccess || p.slices == 1) return e;
  return gated ? join<true>(a, p.slices, s) : join<false>(a, p.slices, s);
}

hipError_t launch_linear_bwd(const LinearBwdArgs& a, hipStream_t s) {
  const bool gated = a.act == MOE_ACT_SWIGLU;
  const int64_t N = gated ? 2 * (int64_t)a.n : a.n;
  const int rows = dp_rows(a.T, N), chunks = (int)ceil_div(a.T, rows);
  if (a.dP || a.db) {
    const int blocks = (int)ceil_div(a.n, 256);
    float* sums = chunks == 1 ? a.db : a.db ? a.db_part : nullptr;
    if (gated)
      linear_dp_kernel<true><<<chunks * blocks, 256, 0, s>>>(a, blocks, rows, sums);
    else
      linear_dp_kernel<false><<<chunks * blocks, 256, 0, s>>>(a, blocks, rows, sums);
    const hipError_t e = hipGetLastError();
    if (e != hipSuccess) return e;
  }
  const uint16_t* dP = a.dP ? a.dP : a.dY;
  const int64_t ldp = a.dP ? N : a.ldy;
  if (a.dX) {
    const LinearPlan p = dx_plan(a.T, a.k, N);
    const LinearArgs x{dP, a.W, nullptr, a.G, nullptr, a.dX, a.dx_part, a.T, (int)N, a.k, MOE_ACT_NONE, ldp, a.ldx, a.ldx};
    hipError_t e = run_columns<OpLinearDX>(x, a.k, 1, N % kBK != 0, s);
    if (e == hipSuccess && p.slices > 1) e = join<false>(x, p.slices, s);
    if (e != hipSuccess) return e;
  }
  int splits = 1;
  if (a.dW) {
    const DwPlan p = dw_plan(a.T, a.k, N);
    splits = p.splits;
    const LinearArgs x{a.X, nullptr, nullptr, nullptr, nullptr, nullptr, a.dw_part, a.T, a.k, 0, 0, a.ldx, 0, 0};
    const int tiles = (int)(p.splits * ceil_div(a.k, p.bm) * ceil_div(N, p.bm));
    auto go = [&](auto cfg) {
      using C = decltype(cfg);
      return splits > 1 ? run<OpLinearDW<C, true>>({x, dP, ldp, a.dW, (int)N, splits, p.chunk}, tiles, s)
                        : run<OpLinearDW<C, false>>({x, dP, ldp, a.dW, (int)N, 1, p.chunk}, tiles, s);
    };
    const hipError_t e = p.bm == 256 ? go(D256x256{}) : p.deep ? go(D128x128d{}) : go(D128x128{});
    if (e != hipSuccess) return e;
  }
  const bool join_db = a.db && chunks > 1;
  if (splits > 1 || join_db) {
    const int64_t MN = (int64_t)a.k * N;
    const int wgs = splits > 1 ? (int)std::min<int64_t>(ceil_div(MN / 4, 256), 2048) : 0;
    const int cols = join_db ? (int)ceil_div(N, 32) : 0;
    linear_sums_kernel<<<wgs + cols, 256, 0, s>>>(a.dw_part, splits, MN, a.dW, wgs, a.db_part, chunks, (int)N, a.db);
    return hipGetLastError();
  }
  return hipSuccess;
}

}  // namespace smoe

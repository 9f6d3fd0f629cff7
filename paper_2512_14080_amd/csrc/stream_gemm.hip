// Grouped GEMMs over few rows per expert (decode and short prefill calls).
//
// With a handful of rows per expert the layer is bound by reading the expert
// weights once; the 256 x 256 tiles of gemm_core.h then run one latency-bound
// k loop per CU (T = 1, d = 1536, n = 256, E = 128, K = 8: 16 workgroups of 24
// dependent 64-deep steps, 26 us for 12.6 MB), and their M side stages 256 rows
// for the few that exist.  Here the weights stream straight into registers, and
// nothing but the final sum is shared between waves:
//   - A workgroup computes 128 columns of one expert for 16 MB rows; its KW
//     waves split the reduction (wave w takes steps w, w + KW, ... of 32 k), so
//     every wave is an independent stream of loads without barriers, and even
//     one row's weights are requested by many waves at once.
//   - Weights with k outer in memory (W1 and W2 in the forward): a lane loads
//     16 bytes (8 columns) of 8 consecutive k rows, whole 128- or 256-byte runs
//     per row, and transposes its 8 x 8 block with 32 v_perm_b32.  MFMA j
//     (16x16x32) then takes column 8 l + j of lane l: the columns of one MFMA
//     are 8 apart, which only permutes the accumulators, so a lane ends with
//     eight consecutive columns of four rows.
//   - The rows (k contiguous) are MFMA fragments as they lie in memory: 16
//     bytes per lane of a gathered row, no LDS.
//   - NBUF steps of loads are in flight per wave (8 KB of weights each).
//   - At the end the waves' accumulators meet in LDS, 16 rows at a time, and are
//     added in wave order by the epilogue.
#include <algorithm>

#include "fp8_block.h"
#include "launch.h"

namespace smoe {

// 8 rows (k) x 8 columns of bf16, one row per register quad -> per column the
// 8 k values (an MFMA operand)
__device__ __forceinline__ bf16x8 column_of(const u32x4 (&w)[8], int j) {
  const uint32_t sel = (j & 1) ? 0x07060302u : 0x05040100u;
  u32x4 f;
#pragma unroll
  for (int p = 0; p < 4; ++p) f[p] = __builtin_amdgcn_perm(w[2 * p + 1][j >> 1], w[2 * p][j >> 1], sel);
  return __builtin_bit_cast(bf16x8, f);
}

constexpr int kStreamCols = 128;  // columns of a workgroup
typedef f32x4 StreamPart[16][2][16];  // one wave's 16 x 128 partial: [row][half of 8 columns][lane column]

// the sum over the waves of four consecutive columns, 4 c4 .. 4 c4 + 3 of the tile
template <int KW>
__device__ __forceinline__ f32x4 stream_sum(const StreamPart* part, int row, int c4) {
  f32x4 s = part[0][row][c4 & 1][c4 >> 1];
#pragma unroll
  for (int w = 1; w < KW; ++w) {
    const f32x4 v = part[w][row][c4 & 1][c4 >> 1];
#pragma unroll
    for (int q = 0; q < 4; ++q) s[q] += v[q];
  }
  return s;
}

// The i-th further group (of `rows` rows; each expert's first is not counted, the
// others follow in expert order): its expert and first row.  False where there are
// no more than i.  Called by every thread of a workgroup of NT; lds: 18 words.
template <int NT>
__device__ __forceinline__ bool find_group(const int32_t* __restrict__ offsets, int E, int rows, int i, int* lds,
                                           int* expert, int* first_row) {
  constexpr int kOwn = 8;  // consecutive experts of a thread (E is a multiple of 8)
  if (i >= offsets[E] / rows) return false;  // (c rows have at most c / rows further groups)
  int* found = lds + 16;
  int base = 0;
  for (int e0 = 0; e0 < E; e0 += kOwn * NT) {
    const int e = e0 + kOwn * threadIdx.x;
    int n[kOwn], sum = 0;
    if (e < E) {
      int o[kOwn + 1];
#pragma unroll
      for (int q = 0; q <= kOwn; ++q) o[q] = offsets[e + q];
#pragma unroll
      for (int q = 0; q < kOwn; ++q) {
        n[q] = o[q + 1] > o[q] ? (o[q + 1] - o[q] - 1) / rows : 0;
        sum += n[q];
      }
    }
    int total;
    int at = base + block_excl_scan<NT>(sum, &total, lds);
    if (base + total > i) {  // here: one thread holds it
      if (at <= i && i < at + sum)
#pragma unroll
        for (int q = 0; q < kOwn; ++q) {
          if (at <= i && i < at + n[q]) {
            found[0] = e + q;
            found[1] = (i - at + 1) * rows;
          }
          at += n[q];
        }
      __syncthreads();
      *expert = __builtin_amdgcn_readfirstlane(found[0]);
      *first_row = __builtin_amdgcn_readfirstlane(found[1]);
      return true;
    }
    base += total;
  }
  return false;
}

// grid: x column tiles.  Router: y k slices, z groups of 16 MB rows.  Experts: y
// < E the first group of expert y, y >= E the experts' other groups, in expert
// order.  Most experts have one group, but with a skewed router a hot one has up
// to T rows; a workgroup past E finds its group in the sums of the experts'
// further groups (find_group), about 2 us beside the first groups' loads.
// (Eight workgroups per expert and tile that looped over its groups, most of them
// empty, ran a hot expert's groups one after the other: T = 1024, d = 1536, n =
// 256, E = 512, K = 8, Zipf 2: 207 us a forward call, now 134; balanced 291, 284.)
// Op supplies
//   EXPERTS: rows and groups by expert,
//   void rows(p, y, off, cnt): the rows [off, off + cnt),
//   int k0(p, y), int k(p, y): the reduction, a multiple of 32,
//   const uint16_t* x_row(p, row) (k contiguous from 0),
//   const uint16_t* w(p, y) with leading dimension ldw(p),
//   int col(p, tile, l): first of the eight columns of lane column l
//   template <int KW> void finish(p, y, tile, row0, rows, part): 16 rows
template <class Op, int MB, int KW, int NBUF, int OCC>
__global__ __launch_bounds__(64 * KW, OCC) void stream_gemm_kernel(const typename Op::Params p) {
  __shared__ StreamPart part[KW];
  const int tile = blockIdx.x;
  int e = blockIdx.y, m0 = blockIdx.z * 16 * MB;
  if constexpr (Op::EXPERTS)
    if (e >= p.E && !find_group<64 * KW>(p.offsets, p.E, 16 * MB, e - p.E, (int*)part, &e, &m0)) return;
  int off, cnt;
  Op::rows(p, e, off, cnt);
  if (m0 >= cnt) return;
  const int kbeg = Op::k0(p, e);
  const int lane = lane_id(), g = lane >> 4, l = lane & 15;
  const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  const int ns = (Op::k(p, e) / 32 - wave + KW - 1) / KW;  // this wave's steps
  const uint16_t* wbase = Op::w(p, e);
  const uint32_t ldw = Op::ldw(p);
  const uint32_t wcol = Op::col(p, tile, l);
  const uint16_t* xp[MB];
#pragma unroll
  for (int b = 0; b < MB; ++b) xp[b] = Op::x_row(p, off + min(m0 + 16 * b + l, cnt - 1)) + 8 * g;
  f32x4 acc[MB][8];
#pragma unroll
  for (int b = 0; b < MB; ++b)
#pragma unroll
    for (int j = 0; j < 8; ++j) acc[b][j] = f32x4{0.f, 0.f, 0.f, 0.f};
  u32x4 wv[NBUF][8];
  bf16x8 xv[NBUF][MB];
  // step s of this wave; a step past the end reads the step 0 addresses (cached, unused)
  auto load = [&](int buf, int s) {
    const uint32_t k = kbeg + 32 * (s < ns ? wave + KW * s : wave);
    const uint32_t o = (k + 8 * g) * ldw + wcol;
#pragma unroll
    for (int i = 0; i < 8; ++i) wv[buf][i] = *(const u32x4*)(wbase + (size_t)(o + i * ldw));
#pragma unroll
    for (int b = 0; b < MB; ++b) xv[buf][b] = *(const bf16x8*)(xp[b] + k);
  };
  if (ns > 0) {
#pragma unroll
    for (int q = 0; q < NBUF; ++q) load(q, q);
    for (int s = 0;; s += NBUF) {
#pragma unroll
      for (int q = 0; q < NBUF; ++q) {
#pragma unroll
        for (int j = 0; j < 8; ++j) {
          const bf16x8 wf = column_of(wv[q], j);
#pragma unroll
          for (int b = 0; b < MB; ++b)
            acc[b][j] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(xv[q][b], wf, acc[b][j], 0, 0, 0);
        }
        if (s + q + 1 >= ns) goto done;
        load(q, s + q + NBUF);
      }
    }
  done:;
  }
#pragma unroll
  for (int b = 0; b < MB; ++b) {
    if (m0 + 16 * b >= cnt) break;
    __syncthreads();  // the previous rows' sums have been read
#pragma unroll
    for (int r = 0; r < 4; ++r)
#pragma unroll
      for (int h = 0; h < 2; ++h)
        part[wave][4 * g + r][h][l] =
            f32x4{acc[b][4 * h][r], acc[b][4 * h + 1][r], acc[b][4 * h + 2][r], acc[b][4 * h + 3][r]};
    __syncthreads();
    Op::template finish<KW>(p, e, tile, off + m0 + 16 * b, min(16, cnt - m0 - 16 * b), part);
  }
}

// rows of the routing: expert y's
template <class Params>
__device__ __forceinline__ void expert_rows(const Params& p, int y, int& off, int& cnt) {
  off = p.offsets[y];
  cnt = p.offsets[y + 1] - off;
}

// H = gather(X) W1_e (+ b1_e), A = SwiGLU(H): 64 gate columns (lane columns
// 0..7) and the matching up columns (8..15)
struct StreamUp {
  using Params = UpArgs;
  static constexpr bool EXPERTS = true;
  static __device__ void rows(const Params& p, int y, int& off, int& cnt) { expert_rows(p, y, off, cnt); }
  static __device__ int k0(const Params&, int) { return 0; }
  static __device__ int k(const Params& p, int) { return p.d; }
  static __device__ const uint16_t* x_row(const Params& p, int row) { return p.X + (size_t)p.row_token[row] * p.d; }
  static __device__ const uint16_t* w(const Params& p, int e) { return p.W1 + (size_t)e * p.d * (2 * p.n); }
  static __device__ uint32_t ldw(const Params& p) { return 2 * p.n; }
  static __device__ uint32_t col(const Params& p, int tile, int l) {
    return (l < 8 ? 0 : p.n) + 64 * tile + 8 * (l & 7);
  }
  template <int KW>
  static __device__ void finish(const Params& p, int e, int tile, int row0, int rows, const StreamPart* part) {
    for (int i = threadIdx.x; i < 256; i += 64 * KW) {
      const int row = i >> 4, c4 = i & 15;
      if (row >= rows) break;
      f32x4 hg = stream_sum<KW>(part, row, c4), hu = stream_sum<KW>(part, row, c4 + 16);
      const int c = 64 * tile + 4 * c4;
      if (p.b1) {
        const float* b = p.b1 + (size_t)e * 2 * p.n + c;
        const f32x4 bg = *(const f32x4*)b, bu = *(const f32x4*)(b + p.n);
#pragma unroll
        for (int q = 0; q < 4; ++q) {
          hg[q] += bg[q];
          hu[q] += bu[q];
        }
      }
      float a[4];
#pragma unroll
      for (int q = 0; q < 4; ++q) {
        float sg;
        a[q] = silu_sig(hg[q], &sg) * hu[q];
      }
      uint16_t* h = p.H + (size_t)(row0 + row) * (2 * p.n) + c;
      *(u32x2*)h = pack_bf16x4(hg[0], hg[1], hg[2], hg[3]);
      *(u32x2*)(h + p.n) = pack_bf16x4(hu[0], hu[1], hu[2], hu[3]);
      *(u32x2*)(p.A + (size_t)(row0 + row) * p.n + c) = pack_bf16x4(a[0], a[1], a[2], a[3]);
    }
  }
};

// Y = A W2_e (+ b2_e); AGG: how Y leaves (0: Y rows expert-major; 1 and 2: the
// aggregation ablation's scatter to p.dst[row] and fp32 atomics, as OpDown)
template <int AGG>
struct StreamDown {
  using Params = DownArgs;
  static constexpr bool EXPERTS = true;
  static __device__ void rows(const Params& p, int y, int& off, int& cnt) { expert_rows(p, y, off, cnt); }
  static __device__ int k0(const Params&, int) { return 0; }
  static __device__ int k(const Params& p, int) { return p.n; }
  static __device__ const uint16_t* x_row(const Params& p, int row) { return p.A + (size_t)row * p.n; }
  static __device__ const uint16_t* w(const Params& p, int e) { return p.W2 + (size_t)e * p.n * p.d; }
  static __device__ uint32_t ldw(const Params& p) { return p.d; }
  static __device__ uint32_t col(const Params& p, int tile, int l) { return kStreamCols * tile + 8 * l; }
  template <int KW>
  static __device__ void finish(const Params& p, int e, int tile, int row0, int rows, const StreamPart* part) {
    for (int i = threadIdx.x; i < 512; i += 64 * KW) {
      const int row = i >> 5, c4 = i & 31;
      if (row >= rows) break;
      f32x4 y = stream_sum<KW>(part, row, c4);
      const int c = kStreamCols * tile + 4 * c4;
      if (p.b2) {
        const f32x4 b = *(const f32x4*)(p.b2 + (size_t)e * p.d + c);
#pragma unroll
        for (int q = 0; q < 4; ++q) y[q] += b[q];
      }
      const u32x2 v = pack_bf16x4(y[0], y[1], y[2], y[3]);
      const int r = row0 + row;
      if constexpr (AGG == 2) {
        float* o = p.O32 + (size_t)p.row_token[r] * p.d + c;
        const float s = p.row_w[r];
        unsafeAtomicAdd(o, s * bf_lo(v[0]));
        unsafeAtomicAdd(o + 1, s * bf_hi(v[0]));
        unsafeAtomicAdd(o + 2, s * bf_lo(v[1]));
        unsafeAtomicAdd(o + 3, s * bf_hi(v[1]));
      } else {
        *(u32x2*)(p.Y + (size_t)(AGG == 1 ? p.dst[r] : r) * p.d + c) = v;
      }
    }
  }
};

// Row blocks per workgroup.  (up + down) streaming / tiled, with mb = 1 | mb = 2, for
// balanced experts and for a router skewed by Zipf exponents 0.5 to 2 (the worst):
//                                            mean 2       8            12           16
//   d = 1024, n = 256, E = 64, K = 8         .84|.83      .91|.89      1.12|.92     1.20|.95
//     skewed                                 .81|.80      1.15|1.01    1.15|1.10    1.16|1.08
//   d = 1536, n = 256, E = 256, K = 8        .78|.79      .91|.86      .97|.89      1.20|.90
//     skewed                                 .85|.81      1.08|.97     1.17|.99     1.42|1.11
//   d = 1024, n = 128, E = 1024, K = 8       .74|.75      .80|.78      .88|.80      1.11|.84
//     skewed                                 .76|.79      1.24|1.01    1.41|1.08    1.65|1.22
//   d = 4096, n = 512, E = 128, K = 8        .90|.90      1.03|.95     1.10|.95     1.36|.97
//     skewed                                 .89|.93      1.10|1.03    1.21|1.07    1.26|1.09
//   d = 1024, n = 256, E = 16, K = 8         .61|.63      .59|.63      .67|.69      .69|.70
//     skewed                                 .66|.67      .62|.68      .72|.71      .75|.72
// An expert with more rows than a group has its weights read again per group, so
// two row blocks are the better ones from a few rows per expert on, skewed or not
// (with at most 16 tokens no expert fills a second).  Up to 12 rows per expert
// streaming is the faster one and a skewed router costs it little; up to 20 it
// depends on the skew, more so the more tokens a hot expert can have (T = 2048 in
// the third line: 69 us against 57).  Beyond, and for more tokens, the tiled GEMMs
// are taken, except where they have too few tiles for the CUs:
//   d = 1536, n = 1024, E = 16, K = 2, T = 256, mean 32   up 29 / 41   down 18 / 25
// A rounded routing's experts have no rows or m_tile and more, whatever the mean:
//   T = 512, d = 1536, n = 256, E = 256, K = 8 (mean 16), rounded up to 256:
//   forward call 1088 us streaming, 350 tiled; d = 4096, n = 512, up to 128: 2923, 826
static StreamShape stream_groups(const moe_dims& m, int capacity, int mb) {
  // further groups of at most `capacity` rows over experts of at most T
  const int64_t rows = 16 * mb, further = std::min(capacity / rows, m.E * ((m.T - 1) / rows));
  return m.E + further <= 65535 ? StreamShape{mb, (int)further} : StreamShape{0, 0};
}
StreamShape stream_shape(const moe_dims& m, int capacity, int m_tile, int64_t tiles_per_expert) {
  const StreamShape tiled{0, 0};
  if ((int64_t)m.d * 2 * m.n > INT32_MAX) return tiled;  // 32-bit offsets within an expert's weights
  const int64_t mean = std::max<int64_t>(((int64_t)m.T * m.K + m.E - 1) / m.E, m_tile);
  const bool few_tiles = m.E * tiles_per_expert < 192;
  int mb;
  if (m.T <= 16 || mean <= 2)
    mb = 1;
  else if (mean <= (few_tiles || m.T <= 2048 ? 20 : 12))
    mb = 2;
  else if (mean <= 64 && few_tiles)
    mb = 4;
  else
    return tiled;
  return stream_groups(m, capacity, mb);
}

// Partial router logits of k slice y: part[y][t][e] = sum over the slice of X W_r
struct StreamRouter {
  using Params = RouterPartArgs;
  static constexpr bool EXPERTS = false;
  static __device__ void rows(const Params& p, int, int& off, int& cnt) {
    off = 0;
    cnt = p.T;
  }
  static __device__ int k0(const Params& p, int y) { return y * p.slice; }
  static __device__ int k(const Params& p, int y) { return min(p.slice, p.d - y * p.slice); }
  static __device__ const uint16_t* x_row(const Params& p, int row) { return p.X + (size_t)row * p.d; }
  static __device__ const uint16_t* w(const Params& p, int) { return p.Wr; }
  static __device__ uint32_t ldw(const Params& p) { return p.E; }
  // (lane columns past E, a multiple of 8, re-read the last ones)
  static __device__ uint32_t col(const Params& p, int tile, int l) { return min(kStreamCols * tile + 8 * l, p.E - 8); }
  template <int KW>
  static __device__ void finish(const Params& p, int y, int tile, int row0, int rows, const StreamPart* part) {
    for (int i = threadIdx.x; i < 512; i += 64 * KW) {
      const int row = i >> 5, c4 = i & 31, c = kStreamCols * tile + 4 * c4;
      if (row >= rows) break;
      if (c < p.E) *(f32x4*)(p.part + ((size_t)y * p.T + row0 + row) * p.E + c) = stream_sum<KW>(part, row, c4);
    }
  }
};

// Waves and steps of loads in flight of the row blocks, within the registers (no
// spills): up to eight waves share the k / 32 steps.  From k = 768 on every wave has
// three or more; k = 256 is one step for each of eight waves, below 256 some of them
// have none, and a second buffer then re-reads the first step (cached, unused).  A
// short k (the down-projection of a narrow expert) has two waves with a step or two
// each (T = 65, d = 1664, n = 64, E = 312, K = 8: down 26 us with eight waves, six of
// them idle, 13 with two).
template <class Op>
static hipError_t run_stream(const typename Op::Params& p, dim3 grid, int mb, int k, hipStream_t s) {
  if (mb == 1 && k >= 768)
    stream_gemm_kernel<Op, 1, 8, 3, 2><<<grid, dim3(512), 0, s>>>(p);
  else if (mb == 1 && k > 128)
    stream_gemm_kernel<Op, 1, 8, 2, 4><<<grid, dim3(512), 0, s>>>(p);
  else if (mb == 1)
    stream_gemm_kernel<Op, 1, 2, 2, 3><<<grid, dim3(128), 0, s>>>(p);
  else if (mb == 2 && k <= 128)
    stream_gemm_kernel<Op, 2, 2, 1, 3><<<grid, dim3(128), 0, s>>>(p);
  else if (mb == 2)
    stream_gemm_kernel<Op, 2, 4, 2, 2><<<grid, dim3(256), 0, s>>>(p);
  else
    stream_gemm_kernel<Op, 4, 4, 1, 2><<<grid, dim3(256), 0, s>>>(p);
  return hipGetLastError();
}

static dim3 stream_grid(int tiles, int E, const StreamShape& t) { return dim3(tiles, E + t.further); }

hipError_t launch_stream_up(const UpArgs& a, const StreamShape& t, hipStream_t s) {
  return run_stream<StreamUp>(a, stream_grid(a.n / 64, a.E, t), t.mb, a.d, s);
}
hipError_t launch_stream_down(const DownArgs& a, int strategy, const StreamShape& t, hipStream_t s) {
  const dim3 grid = stream_grid(a.d / kStreamCols, a.E, t);
  if (strategy == MOE_AGG_SCATTER_SUM) return run_stream<StreamDown<1>>(a, grid, t.mb, a.n, s);
  if (strategy == MOE_AGG_ATOMIC_F32) return run_stream<StreamDown<2>>(a, grid, t.mb, a.n, s);
  return run_stream<StreamDown<0>>(a, grid, t.mb, a.n, s);
}

// Row blocks of the router's workgroups: one (16 tokens) while that gives up to
// two workgroups per CU, more as W_r would otherwise be re-read too often.
static int router_row_blocks(int T, int E, int* groups) {
  const int tiles = (E + kStreamCols - 1) / kStreamCols;
  for (int mb = 1;; mb *= 2) {
    *groups = (T + 16 * mb - 1) / (16 * mb);
    if (mb == 4 || tiles * *groups <= 512) return mb;
  }
}

int router_slices(int T, int d, int E, size_t part_bytes) {
  int groups;
  router_row_blocks(T, E, &groups);
  const int steps = d / 32, wgs = (E + kStreamCols - 1) / kStreamCols * groups;
  // about one workgroup per two CUs, two or more steps for each of eight waves
  const int64_t fit = part_bytes / ((size_t)T * E * 4);
  const int want = std::min({128 / wgs, steps / 16, (int)std::min<int64_t>(fit, 64)});
  if (want <= 1) return 1;
  const int per = (steps + want - 1) / want;  // steps of a slice
  return (steps + per - 1) / per;
}

hipError_t launch_router_part(const uint16_t* X, const uint16_t* Wr, float* part, int slices, int T, int d, int E,
                              hipStream_t s) {
  const int steps = d / 32, slice = 32 * ((steps + slices - 1) / slices);
  int groups;
  const int mb = router_row_blocks(T, E, &groups);
  const dim3 grid((E + kStreamCols - 1) / kStreamCols, slices, groups);
  return run_stream<StreamRouter>({X, Wr, part, T, d, E, slice}, grid, mb, slice, s);
}

// ---------------------------------------------------------------- 8-bit weights
// The same for the 8-bit forward.  MFMA 16x16x128 takes one block of 128 k at a time,
// so a wave's step is one block, with one scale byte of the weights and one of the
// row.  A workgroup computes 64 weight columns (8 KB of codes a step and wave); lane l
// loads, of weight column l % 16, the codes of k 16 (l / 16) + [0, 16) and the same 64
// further on: whole 64-byte runs of k per instruction.  The rows are quantised as they
// are loaded (each block by one wave of the workgroup, its largest |x| a maximum over
// the four lanes that share the row), so neither X nor A needs a launch or a buffer of
// codes of its own; A passes between the two products in fp32, and so does Y to its sum
// (T = 256 at d = 4096, n = 512, E = 128: 188.5 instead of 184.5 us a call and O 2.1e-3
// instead of 2.7e-3 off; the tiled projections, whose Y is large, keep bf16).  D = W x X: a lane ends
// with four consecutive columns of one row.  What keeps loads in flight is many waves,
// each with one step's: two steps in flight per wave cost registers, and with them
// waves (d = 4096, n = 512, E = 128, 256 tokens: up 127 -> 117 us, down 113 -> 73).
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

// grid: as stream_gemm_kernel's of the experts.  Op supplies
//   F32: whether rows come in fp32 (else bf16),
//   int blocks(p), k(p): blocks of the reduction, and its length,
//   const void* row(p, r), const uint8_t* w(p, e), const uint8_t* ws(p, e, tile, half),
//   uint32_t w_row(p, tile, c): offset of weight column c of the tile,
//   finish(p, e, tile, row0, rows, part)
// stream8_rows: rows [m0, cnt) of the expert's, at most 16 MB; xp: those that the lanes load.
// The 8-bit instruction adds its products to 1.3e-5 of the result, which moves some of
// A's codes to the other side of a step.  With few rows single ones show in O (one
// token, d = 1536, n = 256: O 2.7e-3 off, 1.7e-3 without): there the up-projection
// multiplies the same codes in bf16, which is exact but for fp32 sums, at 11.5 instead
// of 11.3 us a call.  With two row blocks it would cost 7 to 12%.
template <template <int> class OpT, int NJ, int MB, int KW>
__device__ __forceinline__ void stream8_rows(const QuantArgs& p, int tile, int e, int off, int cnt, int m0,
                                             const void* const (&xp)[MB], Stream8Part<NJ>* part) {
  using Op = OpT<NJ>;
  constexpr bool kInBf16 = MB == 1 && !Op::F32;
  const int lane = lane_id(), g = lane >> 4, l = lane & 15;
  const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  const uint8_t* wbase = Op::w(p, e);
  const uint8_t* ws0 = Op::ws(p, e, tile, 0);
  const uint8_t* ws1 = Op::ws(p, e, tile, 1);
  uint32_t wrow[NJ];
#pragma unroll
  for (int j = 0; j < NJ; ++j) wrow[j] = Op::w_row(p, tile, 16 * j + l) + 16 * g;
  f32x4 acc[MB][NJ];
#pragma unroll
  for (int b = 0; b < MB; ++b)
#pragma unroll
    for (int j = 0; j < NJ; ++j) acc[b][j] = f32x4{0.f, 0.f, 0.f, 0.f};
  const int blocks = Op::blocks(p);
  for (int kb = wave; kb < blocks; kb += KW) {
    const uint32_t k = kQBlock * kb;
    Weights8<NJ> wv;
    wv.load(wbase, wrow, k);
    const int sv[2] = {ws0[kb], ws1[kb]};
    RowBlock8<Op::F32> xv[MB];
#pragma unroll
    for (int b = 0; b < MB; ++b) xv[b].load(xp[b], k + 16 * g, (int)k + 64 < Op::k(p));
#pragma unroll
    for (int b = 0; b < MB; ++b) {
      int xs;
      const i32x8 x = xv[b].codes(&xs);
#pragma unroll
      for (int j = 0; j < NJ; ++j) {
        const int ws = sv[2 * j / NJ];
        if constexpr (kInBf16) {
          f32x4 y = f32x4{0.f, 0.f, 0.f, 0.f};
#pragma unroll
          for (int i = 0; i < 4; ++i)
            y = __builtin_amdgcn_mfma_f32_16x16x32_bf16(codes_bf16(wv.frag(j), i, 1.f), codes_bf16(x, i, 1.f), y, 0, 0, 0);
#pragma unroll
          for (int q = 0; q < 4; ++q) acc[b][j][q] += ldexpf(y[q], ws + xs - 254);
        } else {
          acc[b][j] = __builtin_amdgcn_mfma_scale_f32_16x16x128_f8f6f4(wv.frag(j), x, acc[b][j], 0, 0, 0, ws, 0, xs);
        }
      }
    }
  }
#pragma unroll
  for (int b = 0; b < MB; ++b) {
    if (m0 + 16 * b >= cnt) break;
    __syncthreads();  // the previous rows' sums have been read
#pragma unroll
    for (int j = 0; j < NJ; ++j) part[wave][l][4 * j + g] = acc[b][j];
    __syncthreads();
    Op::template finish<KW>(p, e, tile, off + m0 + 16 * b, min(16, cnt - m0 - 16 * b), part);
  }
}

template <template <int> class OpT, int NJ, int MB, int KW, int OCC>
__global__ __launch_bounds__(64 * KW, OCC) void stream8_gemm_kernel(const QuantArgs p) {
  __shared__ Stream8Part<NJ> part[KW];
  const int tile = blockIdx.x;
  int e = blockIdx.y, m0 = 0;
  if (e >= p.E && !find_group<64 * KW>(p.offsets, p.E, 16 * MB, e - p.E, (int*)part, &e, &m0)) return;
  const int off = p.offsets[e], cnt = p.offsets[e + 1] - off;
  if (m0 >= cnt) return;
  const void* xp[MB];
#pragma unroll
  for (int b = 0; b < MB; ++b) xp[b] = OpT<NJ>::row(p, off + min(m0 + 16 * b + (lane_id() & 15), cnt - 1));
  stream8_rows<OpT, NJ, MB, KW>(p, tile, e, off, cnt, m0, xp, part);
}

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

// 8 NJ gate columns and the matching up columns; A in fp32
template <int NJ>
struct Stream8Up {
  static constexpr bool F32 = false;
  static constexpr int kCols = 8 * NJ;
  static __device__ int blocks(const QuantArgs& p) { return p.d / kQBlock; }
  static __device__ int k(const QuantArgs& p) { return p.d; }
  static __device__ const void* row(const QuantArgs& p, int r) { return p.X + (size_t)p.row_token[r] * p.d; }
  static __device__ const uint8_t* w(const QuantArgs& p, int e) { return p.W1q + (size_t)e * w1q_bytes(p.d, p.n); }
  static __device__ const uint8_t* ws(const QuantArgs& p, int e, int tile, int half) {
    return p.W1s + (size_t)e * w1s_bytes(p.d, p.n) + (size_t)(2 * (kCols * tile / kQBlock) + half) * q_stride(p.d / kQBlock);
  }
  static __device__ uint32_t w_row(const QuantArgs& p, int tile, int c) {
    const int col = kCols * tile + c % kCols;
    return (uint32_t)(256 * (col / kQBlock) + w1q_row(col % kQBlock, c / kCols)) * p.d;
  }
  template <int KW>
  static __device__ void finish(const QuantArgs& p, int e, int tile, int row0, int rows, const Stream8Part<NJ>* part) {
    constexpr int C4 = kCols / 4;
    for (int i = threadIdx.x; i < 16 * C4; i += 64 * KW) {
      const int row = i / C4, c4 = i % C4;
      if (row >= rows) break;
      f32x4 hg = stream8_sum<KW, NJ>(part, row, c4), hu = stream8_sum<KW, NJ>(part, row, c4 + C4), a;
      const int c = kCols * tile + 4 * c4;
      const float* b1 = p.b1 ? p.b1 + (size_t)e * 2 * p.n + c : nullptr;
#pragma unroll
      for (int q = 0; q < 4; ++q) {
        if (b1) {
          hg[q] += b1[q];
          hu[q] += b1[p.n + q];
        }
        float sg;
        a[q] = silu_sig(hg[q], &sg) * hu[q];
      }
      *(f32x4*)(p.A32 + (size_t)(row0 + row) * p.n + c) = a;
    }
  }
};

template <int NJ>
struct Stream8Down {
  static constexpr bool F32 = true;
  static constexpr int kCols = 16 * NJ;
  static __device__ int blocks(const QuantArgs& p) { return q_blocks(p.n); }
  static __device__ int k(const QuantArgs& p) { return p.n; }
  static __device__ const void* row(const QuantArgs& p, int r) { return p.A32 + (size_t)r * p.n; }
  static __device__ const uint8_t* w(const QuantArgs& p, int e) { return p.W2q + (size_t)e * w2q_bytes(p.d, p.n); }
  static __device__ const uint8_t* ws(const QuantArgs& p, int e, int tile, int) {
    return p.W2s + (size_t)e * w2s_bytes(p.d, p.n) + (size_t)(kCols * tile / kQBlock) * q_stride(q_blocks(p.n));
  }
  static __device__ uint32_t w_row(const QuantArgs& p, int tile, int c) { return (uint32_t)(kCols * tile + c) * q_pad(p.n); }
  template <int KW>
  static __device__ void finish(const QuantArgs& p, int e, int tile, int row0, int rows, const Stream8Part<NJ>* part) {
    constexpr int C4 = kCols / 4;
    for (int i = threadIdx.x; i < 16 * C4; i += 64 * KW) {
      const int row = i / C4, c4 = i % C4;
      if (row >= rows) break;
      f32x4 y = stream8_sum<KW, NJ>(part, row, c4);
      const int c = kCols * tile + 4 * c4;
      if (p.b2) {
        const f32x4 b = *(const f32x4*)(p.b2 + (size_t)e * p.d + c);
#pragma unroll
        for (int q = 0; q < 4; ++q) y[q] += b[q];
      }
      *(f32x4*)(p.Y32 + (size_t)(row0 + row) * p.d + c) = y;
    }
  }
};

// Few tokens: a workgroup per row instead of one per expert, most of which have no
// rows (rows of the same expert read its weights again)
template <int NJ, int KW, int OCC>
__global__ __launch_bounds__(64 * KW, OCC) void stream8_row_up_kernel(const QuantArgs p) {
  __shared__ Stream8Part<NJ> part[KW];
  const int r = blockIdx.y, e = p.row_expert[r], t = p.row_token[r];  // (the grid is within the capacity)
  if (r >= p.offsets[p.E]) return;
  const void* xp[1] = {p.X + (size_t)t * p.d};
  stream8_rows<Stream8Up, NJ, 1, KW>(p, blockIdx.x, e, r, 1, 0, xp, part);
}

// and the down-projection by token, with the sum over the token's rows: a wave's step is
// one block of one row, its product weighted as it is added (Y stays in fp32)
template <int NJ, int KW, int OCC>
__global__ __launch_bounds__(64 * KW, OCC) void stream8_token_down_kernel(const QuantArgs p) {
  using Op = Stream8Down<NJ>;
  __shared__ f32x4 part[KW][4 * NJ];
  const int tile = blockIdx.x, t = blockIdx.y;
  const int lane = lane_id(), g = lane >> 4, l = lane & 15;
  const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  const int blocks = Op::blocks(p), j0 = p.tok_offsets[t], steps = (p.tok_offsets[t + 1] - j0) * blocks;
  uint32_t wrow[NJ];
#pragma unroll
  for (int j = 0; j < NJ; ++j) wrow[j] = Op::w_row(p, tile, 16 * j + l) + 16 * g;
  f32x4 acc[NJ];
#pragma unroll
  for (int j = 0; j < NJ; ++j) acc[j] = f32x4{0.f, 0.f, 0.f, 0.f};
  for (int i = wave; i < steps; i += KW) {
    const int kb = i % blocks, r = p.tok_rows[j0 + i / blocks], e = p.row_expert[r];
    const float s = p.row_w[r];
    const uint32_t k = kQBlock * kb;
    Weights8<NJ> wv;
    wv.load(Op::w(p, e), wrow, k);
    const int sv = Op::ws(p, e, tile, 0)[kb];
    RowBlock8<true> xv;
    xv.load(Op::row(p, r), k + 16 * g, (int)k + 64 < p.n);
    int xs;
    const i32x8 x = xv.codes(&xs);
#pragma unroll
    for (int j = 0; j < NJ; ++j) {
      f32x4 y = f32x4{0.f, 0.f, 0.f, 0.f};
      if (kb == 0 && p.b2) y = *(const f32x4*)(p.b2 + (size_t)e * p.d + Op::kCols * tile + 16 * j + 4 * g);
      y = __builtin_amdgcn_mfma_scale_f32_16x16x128_f8f6f4(wv.frag(j), x, y, 0, 0, 0, sv, 0, xs);
#pragma unroll
      for (int q = 0; q < 4; ++q) acc[j][q] += s * y[q];
    }
  }
  if (l == 0)  // (all 16 rows of the product are this one)
#pragma unroll
    for (int j = 0; j < NJ; ++j) part[wave][4 * j + g] = acc[j];
  __syncthreads();
  if (threadIdx.x < 4 * NJ) {
    f32x4 o = part[0][threadIdx.x];
#pragma unroll
    for (int w = 1; w < KW; ++w)
#pragma unroll
      for (int q = 0; q < 4; ++q) o[q] += part[w][threadIdx.x][q];
    *(u32x2*)(p.O + (size_t)t * p.d + Op::kCols * tile + 4 * threadIdx.x) = pack_bf16x4(o[0], o[1], o[2], o[3]);
  }
}

template <template <int> class Op, int NJ, int MB, int KW, int OCC>
static hipError_t run_stream8(const QuantArgs& p, const StreamShape& t, int cols, hipStream_t s) {
  stream8_gemm_kernel<Op, NJ, MB, KW, OCC><<<stream_grid(cols / Op<NJ>::kCols, p.E, t), dim3(64 * KW), 0, s>>>(p);
  return hipGetLastError();
}

// us of up / down by columns and waves of a workgroup (weights read at 5.0 to 5.6 TB/s
// in the large ones):
//   up                                       64, 4 waves   64, 8   128, 4   128, 8
//     d = 1536, n = 256, E = 128, T = 4       11.5          9.8     14.9     9.6
//     d = 1024, n = 256, E = 64, T = 64       9.2           10.3    10.9     10.4
//     d = 1536, n = 256, E = 128, T = 128     22.9          24.1    21.9     25.1
//     d = 4096, n = 512, E = 128, T = 256     117           119     112      125
//     d = 1536, n = 1024, E = 16, K = 2, T = 512     34.1   39.7     31.6
//   and one token (d = 1536, n = 256, 8 rows): 64 columns and 8 waves 8.4, 32 and 16 waves
//   6.4; d = 4096, n = 512: 19.6, 14.3; but d = 4096, n = 14336, 2 rows (the CUs are full): 40, 52
//   down, Y in fp32                          32, 2   32, 4   64, 2   64, 4   128, 1   128, 2   128, 4
//    16-row groups
//     d = 1536, n = 256, E = 128, T = 16      9.1     9.6     8.3     9.4     15.3     13.8     17.3
//     d = 768, n = 256, E = 8, T = 16         3.7     3.6     3.8     4.0     8.3      5.8      5.8
//     d = 896, n = 320, E = 8, T = 10         4.2     3.6     4.4     4.0     12.4     9.6      6.4
//     d = 1280, n = 1152, E = 8, T = 5        6.7     6.0     7.6     6.4     35.5     22.0     14.8
//     d = 1024, n = 1024, E = 16, T = 8       6.8     6.5     6.8     5.9     32.6     19.4     12.4
//     d = 4096, n = 14336, E = 8, T = 4       87.2    92.1    79.8    74.8    557      363      206
//     d = 4096, n = 512, E = 128, K = 8, T = 32     51.4    48.6    44.4    40.9    78.1   72.2     76.1
//    32-row groups
//     d = 1024, n = 256, E = 64, T = 64       8.6     9.2     7.2     8.0     8.2      7.2      7.7
//     d = 1536, n = 256, E = 128, T = 128     19.5    22.6    15.9    19.4    16.0     18.1     17.7
//     d = 2048, n = 128, E = 256, T = 128     23.6    38.0    20.2    30.8    17.4     20.5     29.0
//     d = 1024, n = 512, E = 16, T = 20       6.1     4.9     5.0     5.3     8.6      6.5      5.4
//     d = 768, n = 1024, E = 32, K = 2, T = 64      10.0    10.2    10.7    10.3    13.9   11.2     9.5
//     d = 2048, n = 1024, E = 32, T = 64      28.2    26.9    21.4    21.0    24.3     17.8     19.4
//     d = 4096, n = 512, E = 128, T = 256     106     109     73.6    73.6    67.1     64.9     65.7
//     d = 2048, n = 2048, E = 16, K = 1, T = 100    26.8    24.9    20.5    20.2    29.9   22.2     18.4
//     d = 4096, n = 4096, E = 16, K = 2, T = 64     93.5    89.6    73.0    66.8    73.9   70.7     62.6
//     d = 4096, n = 14336, E = 8, K = 2, T = 20     152     146     98.3    102     191    125      86.8
//   so: more waves over a long k, or where there are few workgroups; 64 columns of 16 rows
//   where they are a workgroup to a CU at least
hipError_t launch_stream8_up(const QuantArgs& a, const StreamShape& t, hipStream_t s) {
  if (t.mb == 1 && (int64_t)a.capacity * (a.n / 32) <= 128) return run_stream8<Stream8Up, 2, 1, 16, 4>(a, t, a.n, s);
  if (t.mb == 1) return run_stream8<Stream8Up, 4, 1, 8, 4>(a, t, a.n, s);
  return run_stream8<Stream8Up, 4, 2, 4, 4>(a, t, a.n, s);
}
hipError_t launch_stream8_down(const QuantArgs& a, const StreamShape& t, hipStream_t s) {
  const int blocks = q_blocks(a.n), groups = a.E * (a.d / kQBlock);
  if (t.mb == 1) {
    if (blocks <= 2) return run_stream8<Stream8Down, 2, 1, 2, 4>(a, t, a.d, s);
    if (2 * groups < 256) return run_stream8<Stream8Down, 2, 1, 4, 4>(a, t, a.d, s);
    return run_stream8<Stream8Down, 4, 1, 4, 4>(a, t, a.d, s);
  }
  if (blocks <= 2 && groups > 768) return run_stream8<Stream8Down, 8, 2, 1, 2>(a, t, a.d, s);
  if (blocks >= 16 || (blocks > 2 && groups <= 256)) return run_stream8<Stream8Down, 8, 2, 4, 2>(a, t, a.d, s);
  return run_stream8<Stream8Down, 8, 2, 2, 2>(a, t, a.d, s);
}

// Up to E / 2 rows of a token choice, and up to E where the rows' weights are at most 128
// MB, of tokens that make at most 1024 workgroups of 32 columns: by row and by token.  us a
// call, by expert (three launches) / so, by tokens; where rows repeat experts, their
// weights are read again:
//     T =                                1          2           4           8           12          16
//   d = 1536, n = 256, E = 128, K = 8    13.8/11.1  17.3/12.3   19.8/13.7   22.0/19.7   26.6/25.5   29.0/29.1
//   d = 1024, n = 256, E = 64, K = 8     10.9/10.3  12.9/10.6   15.0/11.8   16.7/14.2
//   d = 2048, n = 128, E = 256, K = 10   17.1/10.5              23.6/13.1               28.1/24.9   34.2/28.9
//     (25 tokens, 196 MB: 35.5/40.0)
//   d = 640, n = 768, E = 16, K = 2, 7 tokens: 13.6/12.0; d = 768, n = 512, E = 64, K = 2, 32: 20.3/20.6
//   d = 4096, n = 512, E = 128, K = 8    26.6/19.4  34.7/23.4   48.8/43.4   64.6/69.0   91/99       105/124
//   d = 2048, n = 1024, E = 32, K = 4    18.7/16.3  24.1/17.6   28.3/22.1   33.8/37.3
//   d = 4096, n = 14336, E = 8, K = 2    91.3/90.6  140/128     173/234
// Many workgroups of one or a few steps each lose what the third launch costs (T d / 32):
//   n = 64    d = 4096, E = 64, K = 4, 16 tokens (2048 of them): 19.6/21.8
//             d = 4096, E = 128: K = 8, 8 (1024): 26.6/20.1; K = 1, 64 (8192): 25.8/35.2
//             d = 4096, E = 256, K = 4, 32 (4096): 36.6/34.4; d = 1024, K = 8, 32 (1024): 19.6/18.7
//             d = 2048, E = 256: K = 8, 32 (2048): 26.5/30.1; K = 1, 128 (8192): 22.1/34.5
//             d = 1536, E = 128, K = 2, 64 (2048 and a half as many again): 15.0/20.3
//   n = 128   d = 2048, E = 64, K = 2, 16 (1024): 16.0/11.2; d = 1024, E = 128, K = 2, 64 (2048): 15.3/18.4
//             d = 4096, E = 256, K = 8, 16 (2048): 37.7/40.7
//   n = 256   d = 2048, E = 64, K = 1, 32 (2048): 20.5/18.6
//   n = 512   d = 2048, E = 64, K = 2, 16 (1024): 24.1/22.7; d = 4096, E = 128, K = 1, 64 (8192): 62/81
// Columns and waves as above; of the down-projection: 32 and 8 (16 waves: coarse 102
// instead of 91 a call; 64 columns and 16 or 4 waves: +2 to 25).
bool stream8_by_token(const moe_dims& m, const moe_routing& r) {
  const int64_t rows = (int64_t)m.T * m.K;
  return token_choice(r) && (int64_t)m.T * (m.d / 32) <= 1024 &&
         (2 * rows <= m.E || (rows <= m.E && rows * 3 * m.d * m.n <= 128 << 20));
}
hipError_t launch_stream8_row_up(const QuantArgs& a, int T, int K, hipStream_t s) {
  const int rows = std::min(T * K, a.capacity);
  if ((int64_t)rows * (a.n / 32) <= 128)
    stream8_row_up_kernel<2, 16, 4><<<dim3(a.n / 16, rows), 64 * 16, 0, s>>>(a);
  else
    stream8_row_up_kernel<4, 8, 4><<<dim3(a.n / 32, rows), 64 * 8, 0, s>>>(a);
  return hipGetLastError();
}
hipError_t launch_stream8_token_down(const QuantArgs& a, int T, hipStream_t s) {
  stream8_token_down_kernel<2, 8, 4><<<dim3(a.d / 32, T), 64 * 8, 0, s>>>(a);
  return hipGetLastError();
}

// One rule for both projections, since A passes between the two in one of two forms.
// us a call, streaming / tiled (128-row tiles, gemm_ops.hip), by rows per expert:
//                                  8          12         16         20
//   d = 768, n = 256, E = 128      25 / 27    26 / 28    29 / 28
//   d = 1024, n = 256, E = 64      20 / 24    22 / 25               24 / 25
//   d = 1536, n = 256, E = 512     131 / 130  142 / 133  152 / 134
//   d = 2048, n = 512, E = 64                 56 / 53    59 / 55    63 / 55
//   d = 4096, n = 256, E = 256                176 / 197  187 / 199  200 / 200
//   d = 4096, n = 512, E = 128     163 / 190  172 / 194  183 / 192  194 / 196
//   d = 4096, n = 1024, E = 64                176 / 187  183 / 187  195 / 189
//   d = 4096, n = 4096, E = 16                180 / 198  189 / 198  197 / 199
//   d = 4096, n = 14336, E = 8     288 / 293  303 / 294  320 / 296
StreamShape stream8_shape(const moe_dims& m, int capacity, int m_tile) {
  if (2 * (int64_t)m.d * q_pad(m.n) > INT32_MAX) return {0, 0};  // 32-bit offsets within an expert's codes
  const int64_t mean = std::max<int64_t>(((int64_t)m.T * m.K + m.E - 1) / m.E, m_tile);
  if (m.T <= 16 || mean <= 2) return stream_groups(m, capacity, 1);
  return mean <= (m.d >= 4096 && m.n <= 4096 ? 16 : 10) ? stream_groups(m, capacity, 2) : StreamShape{0, 0};
}

}  // namespace smoe

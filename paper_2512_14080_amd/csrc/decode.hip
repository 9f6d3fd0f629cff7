// The whole layer for a few tokens (T <= 64) in two launches.
//
//   1. Partial logits of the router's k slices, and the second launch's counters to zero.
//   2. Softmax, top-K, up-projection, down-projection and the weighted sum.
//
// With few tokens the layer is bound by one pass over the weights of the experts that
// the tokens pick, and beside that by the launches in a row: a dependent launch costs
// 3 to 6 us here, as much as one token's weights.  So the second launch is a work queue:
// its items, in order, are the up-projection tiles of every picked expert, the
// down-projection tiles, and the sums; a workgroup takes the next item by an atomic
// ticket, and an item that needs others waits for their counter.
//
// The waits end, whatever else runs on the GPU: an item only waits for items of lower
// tickets, a ticket is taken by a workgroup that runs already and that holds at most one
// ticket beyond the one it works on, and the lowest unfinished ticket waits for nothing
// that is unfinished.  No co-residency of the grid is assumed.
//
// Selection is the routing kernels' (wave_topk on the softmax of the summed partials):
// every workgroup forms it for itself from T x E logits in L2, which is cheaper than
// another dependent step, and all get the same from the same sums.
#include <algorithm>

#include "launch.h"
#include "stream_tile.h"
#include "wave_topk.h"

namespace smoe {

constexpr int kDecodeWaves = 8, kDecodeThreads = 64 * kDecodeWaves;

// ---------------------------------------------------------------- router
template <int KB, int MB>
__global__ __launch_bounds__(kDecodeThreads, 2) void decode_router_kernel(const DecodeArgs a, int slice, int counters) {
  using Tile = RowTile<KB>;
  __shared__ typename Tile::Part part[kDecodeWaves];
  const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  if (blockIdx.x == 0 && blockIdx.y == 0 && blockIdx.z == 0)
    for (int i = threadIdx.x; i < counters; i += kDecodeThreads) a.sync[i] = 0;
  const int c0 = Tile::COLS * blockIdx.x, t0 = Tile::RT * MB * blockIdx.z;
  const int kbeg = blockIdx.y * slice, kend = min(a.d, kbeg + slice);
  const Rsrc w = buffer_of(a.Wr, (uint32_t)a.d * a.E * 2), x = buffer_of(a.X, (uint32_t)a.T * a.d * 2);
  const int col = c0 + 8 * Tile::cg();
  uint32_t xoff[MB];
#pragma unroll
  for (int b = 0; b < MB; ++b) {
    const int t = t0 + Tile::RT * b + Tile::row();
    xoff[b] = t < a.T ? (uint32_t)t * a.d * 2 : kBufferOut;
  }
  f32x4 acc[MB][8];
  zero_acc(acc);
  stream_acc<KB, MB, 2, kDecodeWaves>(acc, w, a.E * 2, col < a.E ? col * 2 : kBufferOut, x, xoff, kbeg, kend, wave);
#pragma unroll
  for (int b = 0; b < MB; ++b) {
    if (t0 + Tile::RT * b >= a.T) break;
    __syncthreads();
    Tile::put(part[wave], acc[b]);
    __syncthreads();
    for (int i = threadIdx.x; i < Tile::RT * Tile::COLS / 4; i += kDecodeThreads) {
      const int row = i / (Tile::COLS / 4), c4 = i % (Tile::COLS / 4), t = t0 + Tile::RT * b + row, c = c0 + 4 * c4;
      if (t < a.T && c < a.E) *(f32x4*)(a.part + ((size_t)blockIdx.y * a.T + t) * a.E + c) = Tile::template sum<kDecodeWaves>(part, row, c4);
    }
  }
}

// ---------------------------------------------------------------- the selection
// LDS of a workgroup behind the partial sums
struct Picked {
  unsigned long long* word;  // [E] tokens of each expert, one bit each
  int* gexp;                 // [groups] the picked experts, ascending: a group each
  int* goff;                 // [groups + 1] their first entries in `rows`
  int* rows;                 // [T K] entries t K + j by group, by token within
  int* sel;                  // [T K] expert of entry t K + j
  int* group;                // [T K] its group
  float* w;                  // [T K] its weight
};
__host__ __device__ inline size_t picked_bytes(int T, int E, int K) {
  const int g = T * K < E ? T * K : E;
  return 8 * (size_t)E + 4 * (size_t)(2 * g + 1) + 16 * (size_t)T * K;
}
__device__ __forceinline__ Picked picked_at(char* lds, int T, int E, int K) {
  const int g = min(T * K, E), n = T * K;
  Picked p;
  p.word = (unsigned long long*)lds;
  p.gexp = (int*)(lds + 8 * (size_t)E);
  p.goff = p.gexp + g;
  p.rows = p.goff + g + 1;
  p.sel = p.rows + n;
  p.group = p.sel + n;
  p.w = (float*)(p.group + n);
  return p;
}

template <int EPL>
__device__ __forceinline__ void select_tokens(const DecodeArgs& a, const Picked& p) {
  const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), lane = lane_id();
  const size_t slab = (size_t)a.T * a.E;
  for (int t = wave; t < a.T; t += kDecodeWaves) {
    float v[EPL];
    const float* in = a.part + (size_t)t * a.E;
    for (int q0 = 0; q0 < a.slices; q0 += 4) {  // (four slabs' loads in flight, added in slice order)
      float x[4][EPL];
#pragma unroll
      for (int q = 0; q < 4; ++q)
#pragma unroll
        for (int j = 0; j < EPL; ++j) {
          const int e = lane + 64 * j;
          x[q][j] = q0 + q < a.slices && e < a.E ? in[(q0 + q) * slab + e] : 0.f;
        }
#pragma unroll
      for (int q = 0; q < 4; ++q)
#pragma unroll
        for (int j = 0; j < EPL; ++j) v[j] = q0 + q == 0 ? x[0][j] : v[j] + x[q][j];
    }
    float m = -INFINITY;
#pragma unroll
    for (int j = 0; j < EPL; ++j) {
      const int e = lane + 64 * j;
      v[j] = e < a.E ? v[j] + (a.bias ? a.bias[e] : 0.f) : -INFINITY;
      m = fmaxf(m, v[j]);
    }
    m = dpp_reduce(m, [](float x, float y) { return fmaxf(x, y); });
    float s = 0.f;
#pragma unroll
    for (int j = 0; j < EPL; ++j) {
      v[j] = lane + 64 * j < a.E ? expf(v[j] - m) : 0.f;
      s += v[j];
    }
    s = dpp_reduce(s, [](float x, float y) { return x + y; });
#pragma unroll
    for (int j = 0; j < EPL; ++j) v[j] = v[j] / s;
    wave_topk<EPL>(v, a.E, a.K, [&](int k, int e, float w) {
      p.sel[t * a.K + k] = e;
      p.w[t * a.K + k] = w;
      atomicOr(&p.word[e], 1ull << t);
      if (blockIdx.x == 0) {
        if (a.topk_idx) a.topk_idx[t * a.K + k] = e;
        if (a.topk_w) a.topk_w[t * a.K + k] = w;
      }
    });
  }
}

// the selection and the groups; returns how many there are
__device__ __forceinline__ int pick(const DecodeArgs& a, const Picked& p, int* scan_lds) {
  for (int e = threadIdx.x; e < a.E; e += kDecodeThreads) p.word[e] = 0ull;
  __syncthreads();
  if (a.E <= 64)
    select_tokens<1>(a, p);
  else if (a.E <= 128)
    select_tokens<2>(a, p);
  else if (a.E <= 256)
    select_tokens<4>(a, p);
  else if (a.E <= 512)
    select_tokens<8>(a, p);
  else
    select_tokens<16>(a, p);
  __syncthreads();
  int groups = 0, entries = 0;
  for (int e0 = 0; e0 < a.E; e0 += kDecodeThreads) {
    const int e = e0 + threadIdx.x;
    const int c = e < a.E ? __popcll(p.word[e]) : 0;
    int total;
    // (the picked experts before this one in the upper half, their entries in the lower)
    const int at = block_excl_scan<kDecodeThreads>(c ? c | 1 << 16 : 0, &total, scan_lds);
    if (c) {
      p.gexp[groups + (at >> 16)] = e;
      p.goff[groups + (at >> 16)] = entries + (at & 0xffff);
    }
    groups += total >> 16;
    entries += total & 0xffff;
  }
  if (threadIdx.x == 0) p.goff[groups] = entries;
  __syncthreads();
  for (int i = threadIdx.x; i < a.T * a.K; i += kDecodeThreads) {
    const int e = p.sel[i], t = i / a.K;
    int lo = 0, hi = groups;  // gexp[lo] <= e < gexp[hi]
    while (hi - lo > 1) {
      const int mid = (lo + hi) >> 1;
      if (p.gexp[mid] <= e) lo = mid; else hi = mid;
    }
    p.group[i] = lo;
    p.rows[p.goff[lo] + __popcll(p.word[e] & ((1ull << t) - 1))] = i;
  }
  __syncthreads();
  return groups;
}

// ---------------------------------------------------------------- counters
// sync: [0] the next ticket; from 32 on one word per group, of finished up-projection
// items; then one per column tile, of finished down-projection items
constexpr int kSyncUp = 32;
__device__ __forceinline__ int take_ticket(const DecodeArgs& a) {
  return __hip_atomic_fetch_add(a.sync, 1, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT);
}
// An item's stores, by every thread of the workgroup, before its counter
__device__ __forceinline__ void finish_item(int* counter) {
  asm volatile("s_waitcnt vmcnt(0)" ::: "memory");  // each wave's own are in L2
  __syncthreads();
  if (threadIdx.x == 0) __hip_atomic_fetch_add(counter, 1, __ATOMIC_RELEASE, __HIP_MEMORY_SCOPE_AGENT);
}
// One lane waits until the counter has reached `want`.  A call that shares its workspace with
// another one in flight, which is an error, may have lost counts: the wait is bounded
// (seconds), and false makes the outputs NaN.
constexpr int kMostPolls = 1 << 22;
__device__ __forceinline__ bool wait_counter(int* counter, int want) {
  for (int i = 0; i < kMostPolls; ++i) {
    if (__hip_atomic_load(counter, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT) >= want) return true;
    __builtin_amdgcn_s_sleep(2);
  }
  return false;
}

// ---------------------------------------------------------------- the layer
// KB, MB: rows of a group in MB blocks of 16 / KB
template <int KB, int MB>
struct Decode {
  using Tile = RowTile<KB>;
  static constexpr int RT = Tile::RT, CG = Tile::CG, COLS = Tile::COLS, C4 = COLS / 4;
  static constexpr int NBUF = MB == 1 ? 3 : MB == 2 ? 2 : 1;

  // up-projection: COLS / 2 gate columns and the matching up columns of a group's rows
  static __device__ void up(const DecodeArgs& a, const Picked& p, typename Tile::Part* part, int wave, int gi, int tile) {
    const int e = __builtin_amdgcn_readfirstlane(p.gexp[gi]), r0 = p.goff[gi];
    const int cnt = __builtin_amdgcn_readfirstlane(p.goff[gi + 1] - r0);
    const int n = a.n, N = 2 * n;
    const Rsrc w = buffer_of(a.W1 + (size_t)e * a.d * N, (uint32_t)a.d * N * 2), x = buffer_of(a.X, (uint32_t)a.T * a.d * 2);
    const int c = tile * (COLS / 2) + 8 * (Tile::cg() & (CG / 2 - 1));
    const uint32_t wcol = c < n ? 2 * (c + (Tile::cg() >= CG / 2 ? n : 0)) : kBufferOut;
    auto run = [&](auto blocks) {
      constexpr int B = decltype(blocks)::value;
      uint32_t xoff[B];
#pragma unroll
      for (int b = 0; b < B; ++b) {
        const int r = RT * b + Tile::row();
        xoff[b] = r < cnt ? (uint32_t)(p.rows[r0 + r] / a.K) * a.d * 2 : kBufferOut;
      }
      f32x4 acc[B][8];
      zero_acc(acc);
      stream_acc<KB, B, NBUF, kDecodeWaves>(acc, w, N * 2, wcol, x, xoff, 0, a.d, wave);
#pragma unroll
      for (int b = 0; b < B; ++b) {
        if (RT * b >= cnt) break;
        __syncthreads();
        Tile::put(part[wave], acc[b]);
        __syncthreads();
        for (int i = threadIdx.x; i < RT * C4 / 2; i += kDecodeThreads) {
          const int row = i / (C4 / 2), c4 = i % (C4 / 2), col = tile * (COLS / 2) + 4 * c4;
          if (RT * b + row >= cnt || col >= n) continue;
          f32x4 hg = Tile::template sum<kDecodeWaves>(part, row, c4);
          f32x4 hu = Tile::template sum<kDecodeWaves>(part, row, c4 + C4 / 2);
          if (a.b1) {
            const float* bias = a.b1 + (size_t)e * N + col;
            const f32x4 bg = *(const f32x4*)bias, bu = *(const f32x4*)(bias + n);
#pragma unroll
            for (int q = 0; q < 4; ++q) {
              hg[q] += bg[q];
              hu[q] += bu[q];
            }
          }
          float v[4];
#pragma unroll
          for (int q = 0; q < 4; ++q) {
            float sg;
            v[q] = silu_sig(hg[q], &sg) * hu[q];
          }
          // (A to bf16, the type of the product that follows, as in the layer's forward)
          *(u32x2*)(a.A + (size_t)p.rows[r0 + RT * b + row] * n + col) = pack_bf16x4(v[0], v[1], v[2], v[3]);
        }
      }
    };
    if constexpr (MB >= 4)
      if (cnt > 2 * RT) return run(std::integral_constant<int, 4>{});
    if constexpr (MB >= 2)
      if (cnt > RT) return run(std::integral_constant<int, 2>{});
    run(std::integral_constant<int, 1>{});
  }

  // down-projection of a group's rows: Y in fp32
  static __device__ void down(const DecodeArgs& a, const Picked& p, typename Tile::Part* part, int wave, int gi, int tile) {
    const int e = __builtin_amdgcn_readfirstlane(p.gexp[gi]), r0 = p.goff[gi];
    const int cnt = __builtin_amdgcn_readfirstlane(p.goff[gi + 1] - r0);
    const int n = a.n, d = a.d;
    const Rsrc w = buffer_of(a.W2 + (size_t)e * n * d, (uint32_t)n * d * 2), x = buffer_of(a.A, (uint32_t)a.T * a.K * n * 2);
    const uint32_t wcol = 2 * (tile * COLS + 8 * Tile::cg());
    auto run = [&](auto blocks) {
      constexpr int B = decltype(blocks)::value;
      uint32_t xoff[B];
#pragma unroll
      for (int b = 0; b < B; ++b) {
        const int r = RT * b + Tile::row();
        xoff[b] = r < cnt ? (uint32_t)p.rows[r0 + r] * n * 2 : kBufferOut;
      }
      f32x4 acc[B][8];
      zero_acc(acc);
      stream_acc<KB, B, NBUF, kDecodeWaves>(acc, w, d * 2, wcol, x, xoff, 0, n, wave);
#pragma unroll
      for (int b = 0; b < B; ++b) {
        if (RT * b >= cnt) break;
        __syncthreads();
        Tile::put(part[wave], acc[b]);
        __syncthreads();
        for (int i = threadIdx.x; i < RT * C4; i += kDecodeThreads) {
          const int row = i / C4, c4 = i % C4, col = tile * COLS + 4 * c4;
          if (RT * b + row >= cnt) continue;
          f32x4 y = Tile::template sum<kDecodeWaves>(part, row, c4);
          if (a.b2) {
            const f32x4 bias = *(const f32x4*)(a.b2 + (size_t)e * d + col);
#pragma unroll
            for (int q = 0; q < 4; ++q) y[q] += bias[q];
          }
          *(f32x4*)(a.Y + (size_t)p.rows[r0 + RT * b + row] * d + col) = y;
        }
      }
    };
    if constexpr (MB >= 4)
      if (cnt > 2 * RT) return run(std::integral_constant<int, 4>{});
    if constexpr (MB >= 2)
      if (cnt > RT) return run(std::integral_constant<int, 2>{});
    run(std::integral_constant<int, 1>{});
  }

  // O = R + sum of s Y over each token's entries, the columns of one down-projection tile
  static __device__ void sum_tokens(const DecodeArgs& a, const Picked& p, int tile, int t0, int tokens, bool ok) {
    for (int i = threadIdx.x; i < tokens * C4; i += kDecodeThreads) {
      const int t = t0 + i / C4, col = tile * COLS + 4 * (i % C4);
      if (t >= a.T) break;
      f32x4 o = f32x4{0.f, 0.f, 0.f, 0.f};
      for (int j = 0; j < a.K; ++j) {
        const f32x4 y = *(const f32x4*)(a.Y + (size_t)(t * a.K + j) * a.d + col);
        const float w = p.w[t * a.K + j];
#pragma unroll
        for (int q = 0; q < 4; ++q) o[q] += w * y[q];
      }
      if (a.R) {
        const u32x2 r = *(const u32x2*)(a.R + (size_t)t * a.d + col);
        o[0] += bf_lo(r[0]);
        o[1] += bf_hi(r[0]);
        o[2] += bf_lo(r[1]);
        o[3] += bf_hi(r[1]);
      }
      if (!ok) o = f32x4{NAN, NAN, NAN, NAN};
      *(u32x2*)(a.O + (size_t)t * a.d + col) = pack_bf16x4(o[0], o[1], o[2], o[3]);
    }
  }
};

constexpr int kSumTokens = 16;  // tokens of one item of the sums

template <int KB, int MB>
__global__ __launch_bounds__(kDecodeThreads, 2) void decode_kernel(const DecodeArgs a) {
  using D = Decode<KB, MB>;
  extern __shared__ __attribute__((aligned(16))) char dyn[];  // picked_bytes
  __shared__ typename D::Tile::Part part[kDecodeWaves];
  __shared__ int sh[2];
  __shared__ int scan_lds[kDecodeWaves];
  const Picked p = picked_at(dyn, a.T, a.E, a.K);
  const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  if (threadIdx.x == 0) sh[0] = take_ticket(a);
  const int groups = __builtin_amdgcn_readfirstlane(pick(a, p, scan_lds));
  const int up_tiles = (a.n + D::COLS / 2 - 1) / (D::COLS / 2), down_tiles = a.d / D::COLS;
  const int ups = groups * up_tiles, downs = groups * down_tiles;
  const int sums = down_tiles * ((a.T + kSumTokens - 1) / kSumTokens);
  int* up_done = a.sync + kSyncUp;
  int* down_done = up_done + min(a.T * a.K, a.E);
  bool ok = true;  // (of the waits so far)
  for (;;) {
    int item = __builtin_amdgcn_readfirstlane(sh[0]);
    if (item >= ups + downs + sums) break;
    int next = 0;
    if (threadIdx.x == 0) next = take_ticket(a);
    int* counter = nullptr;
    int* awaited = nullptr;
    int want = 0;
    if (item >= ups + downs) {
      awaited = down_done + (item - ups - downs) % down_tiles;
      want = groups;
    } else if (item >= ups) {
      awaited = up_done + (item - ups) / down_tiles;
      want = up_tiles;
    }
    if (awaited) {
      if (threadIdx.x == 0) {
        sh[1] = wait_counter(awaited, want);
        __builtin_amdgcn_fence(__ATOMIC_ACQUIRE, "agent");
      }
      __syncthreads();
      ok = ok && sh[1];
    }
    if (item < ups) {
      D::up(a, p, part, wave, item / up_tiles, item % up_tiles);
      counter = up_done + item / up_tiles;
    } else if (item < ups + downs) {
      item -= ups;
      D::down(a, p, part, wave, item / down_tiles, item % down_tiles);
      counter = down_done + item % down_tiles;
    } else {
      item -= ups + downs;
      D::sum_tokens(a, p, item % down_tiles, item / down_tiles * kSumTokens, kSumTokens, ok);
    }
    if (counter && ok) finish_item(counter);  // (what gave up is not counted, so that nothing is summed from it)
    __syncthreads();
    if (threadIdx.x == 0) sh[0] = next;
    __syncthreads();
  }
}

// ---------------------------------------------------------------- host
int decode_slices(int T, int d, int E) {
  // about 64 workgroups, of two steps or more for each wave
  const int tiles = (E + 127) / 128 * ((T + 15) / 16);
  const int want = std::max(1, std::min(64 / tiles, d / (2 * 32 * kDecodeWaves)));
  const int per = (d / 32 + want - 1) / want;
  return (d / 32 + per - 1) / per;
}
size_t decode_sync_words(int T, int d, int E, int K) { return kSyncUp + std::min(T * K, E) + d / 32; }

template <int KB, int MB>
static hipError_t run_router(const DecodeArgs& a, hipStream_t s) {
  using Tile = RowTile<KB>;
  const int per = (a.d / 32 + a.slices - 1) / a.slices;
  const dim3 grid((a.E + Tile::COLS - 1) / Tile::COLS, a.slices, (a.T + Tile::RT * MB - 1) / (Tile::RT * MB));
  decode_router_kernel<KB, MB><<<grid, kDecodeThreads, 0, s>>>(a, 32 * per, (int)decode_sync_words(a.T, a.d, a.E, a.K));
  return hipGetLastError();
}

template <int KB, int MB>
static hipError_t run_decode(const DecodeArgs& a, hipStream_t s) {
  using D = Decode<KB, MB>;
  const int64_t groups = std::min(a.T * a.K, a.E);
  const int64_t items = groups * ((a.n + D::COLS / 2 - 1) / (D::COLS / 2) + a.d / D::COLS);
  decode_kernel<KB, MB><<<(int)std::min<int64_t>(items, 256), kDecodeThreads, picked_bytes(a.T, a.E, a.K), s>>>(a);
  return hipGetLastError();
}

hipError_t launch_decode(const DecodeArgs& a, hipStream_t s) {
  const hipError_t e = run_router<1, 1>(a, s);
  if (e != hipSuccess) return e;
  if (a.T <= 4) return run_decode<2, 1>(a, s);
  if (a.T <= 16) return run_decode<1, 1>(a, s);
  if (a.T <= 32) return run_decode<1, 2>(a, s);
  return run_decode<1, 4>(a, s);
}

}  // namespace smoe

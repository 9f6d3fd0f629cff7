// The whole layer for a few tokens (T <= 64) in two launches.
//
//   1. Partial logits of the router's k slices, and the second launch's counters to zero.
//   2. Softmax, top-K, up-projection, down-projection and the weighted sum.
//
// With few tokens the layer is bound by one pass over the weights of the experts that
// the tokens pick, and beside that by the steps in a row: an empty launch behind another
// costs 2.4 us here, and a step's first loads and last sums as much again, while one token's
// weights are read in 3 us.  So the second launch is a work queue: its items, in order, are
// the selection of more than 8 tokens, the up-projection tiles of every picked expert, the
// down-projection tiles, and the sums; a workgroup takes the next item by an atomic ticket,
// and an item that needs others waits for their counter.  What one item leaves for another
// goes past the caches (shared loads and stores): the counter's hop takes 1 us, where a
// write-back of the L2 by every workgroup took 3.2 and an invalidation 1.8.
//
// The waits end, whatever else runs on the GPU: an item only waits for items of lower
// tickets, a ticket is taken by a workgroup that runs already and that holds at most one
// ticket beyond the one it works on, and the lowest unfinished ticket waits for nothing
// that is unfinished.  No co-residency of the grid is assumed.
//
// Selection is the routing kernels' (the K best of the softmax of the summed partials).  Up
// to 8 tokens every workgroup forms it for itself from T x E logits in L2, which is cheaper
// than another dependent step, and all get the same from the same sums.
//
// Measured, as the whole call: one token of d 1536, n 256, E 128, K 8 19 us; 7 tokens of
// d 1024, n 256, E 64, K 8 27.5 us; 64 of d 4096, n 512, E 128, K 8 (1.6 GB of weights) 291 us,
// 5.4 TB/s.
#include <algorithm>

#include "decode_queue.h"
#include "launch.h"
#include "stream8_tile.h"
#include "stream_tile.h"
#include "topk_net.h"

namespace smoe {

constexpr int kDecodeWaves = 8, kDecodeThreads = 64 * kDecodeWaves;

// ---------------------------------------------------------------- router
// grid: column tiles, k slices, groups of 16 rows
__global__ __launch_bounds__(kDecodeThreads, 2) void decode_router_kernel(const DecodeArgs a, int slice, int counters) {
  using Tile = RowTile<1>;
  __shared__ typename Tile::Part part[kDecodeWaves];
  const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), lane = lane_id();
  for (int i = ((blockIdx.z * gridDim.y + blockIdx.y) * gridDim.x + blockIdx.x) * kDecodeThreads + threadIdx.x; i < counters;
       i += gridDim.x * gridDim.y * gridDim.z * kDecodeThreads)
    a.sync[i] = 0;
  const int c0 = Tile::COLS * blockIdx.x, t0 = Tile::RT * blockIdx.z;
  const int kbeg = blockIdx.y * slice, kend = min(a.d, kbeg + slice);
  const Rsrc w = buffer_of(a.Wr, (uint32_t)a.d * a.E * 2), x = buffer_of(a.X, (uint32_t)a.T * a.d * 2);
  const int col = c0 + 8 * Tile::cg(lane), r = t0 + Tile::row(lane);
  const uint32_t xoff[1] = {r < a.T ? (uint32_t)r * a.d * 2 : kBufferOut};
  f32x4 acc[1][8];
  zero_acc(acc);
  RowStream<1, 2> stream;
  stream.prime(w, a.E * 2, col < a.E ? col * 2 : kBufferOut, kbeg, kend, wave, kDecodeWaves, lane);
  stream.template add<false>(acc, x, xoff);
  Tile::put(part[wave], acc[0], lane);
  __syncthreads();
  for (int i = threadIdx.x; i < Tile::RT * Tile::COLS / 4; i += kDecodeThreads) {
    const int row = i / (Tile::COLS / 4), c4 = i % (Tile::COLS / 4), t = t0 + row, c = c0 + 4 * c4;
    if (t < a.T && c < a.E) *(f32x4*)(a.part + ((size_t)blockIdx.y * a.T + t) * a.E + c) = Tile::template sum<kDecodeWaves>(part, row, c4);
  }
}

// ---------------------------------------------------------------- the selection
// LDS of a workgroup behind the partial sums
struct Picked {
  unsigned long long* word;  // [E] tokens of each expert, one bit each
  int* first;                // [E] the first entry of a picked expert
  int* gexp;                 // [groups] the picked experts, ascending: a group each
  int* goff;                 // [groups + 1] their first entries in `rows`
  int* rows;                 // [T K] entries t K + j by group, by token within (one word more)
  int* sel;                  // [T K] expert of entry t K + j
  float* w;                  // [T K] its weight
  uint32_t* keys;            // [T][64 or 128] where waves share a token: its scores' images
};
// waves that share a token, whose experts are then placed by counting (place_experts)
__host__ __device__ inline int decode_share(int T, int E) { return E > 128 || T > 4 ? 1 : T == 1 ? 8 : T == 2 ? 4 : 2; }
__host__ __device__ inline size_t picked_bytes(int T, int E, int K) {
  const int g = T * K < E ? T * K : E;
  const size_t keys = decode_share(T, E) > 1 ? (E <= 64 ? 256 : 512) * (size_t)T : 0;
  return (12 * (size_t)E + 4 * (size_t)(2 * g + 2) + 12 * (size_t)T * K + 15) / 16 * 16 + keys;
}
__device__ __forceinline__ Picked picked_at(char* lds, int T, int E, int K) {
  const int g = min(T * K, E), n = T * K;
  Picked p;
  p.word = (unsigned long long*)lds;
  p.first = (int*)(lds + 8 * (size_t)E);
  p.gexp = p.first + E;
  p.goff = p.gexp + g;
  p.rows = p.goff + g + 1;
  p.sel = p.rows + n + 1;
  p.w = (float*)(p.sel + n);
  p.keys = (uint32_t*)(lds + (12 * (size_t)E + 4 * (size_t)(2 * g + 2) + 12 * (size_t)n + 15) / 16 * 16);
  return p;
}

// An expert's place is the count of those before it, of N: the waves of a token take N / WPT
// experts each, and the lanes of an expert a part of the keys each.  (4 tokens of d 1024, n 256,
// E 64, K 8 24.3 us, 26 with K rounds of an arg-max in one wave; by one wave for a token it loses:
// 16 tokens 36.0, with the arg-max 35.0.)
template <int N, int WPT>
__device__ __forceinline__ void place_experts(const DecodeArgs& a, const Picked& p, const uint32_t* keys, int t, int part) {
  constexpr int MINE = N / WPT, LANES = kWave / MINE, KEYS = N / LANES;
  static_assert(MINE <= kWave && KEYS >= 4);
  const int lane = lane_id(), e = MINE * part + lane / LANES, first = lane % LANES * KEYS;
  const uint32_t key = keys[e];
  int before = 0;
#pragma unroll 8
  for (int i = 0; i < KEYS; i += 4) {
    const u32x4 k = *(const u32x4*)(keys + first + i);
#pragma unroll
    for (int q = 0; q < 4; ++q) before += k[q] > key || (k[q] == key && first + i + q < e);
  }
#pragma unroll
  for (int i = 1; i < LANES; i *= 2) before += __shfl_xor(before, i, kWave);
  // (past E the keys are 0, and behind every expert's)
  if (lane % LANES == 0 && e < a.E && before < a.K) {
    p.sel[t * a.K + before] = e;
    p.w[t * a.K + before] = topk_value(key);
  }
}

// selection of token t by wave `part` of its `wpt`
template <int EPL>
__device__ __forceinline__ void select_token(const DecodeArgs& a, const Picked& p, int t, int part, int wpt) {
  const int lane = lane_id();
  const uint32_t slab = (uint32_t)a.T * a.E;
  const Rsrc in = buffer_of(a.part, a.slices * slab * 4);
  float v[EPL];
  for (int q0 = 0; q0 < a.slices; q0 += 4) {  // (four slabs' loads in flight, added in slice order; zero past the last)
    float x[4][EPL];
#pragma unroll
    for (int q = 0; q < 4; ++q)
#pragma unroll
      for (int j = 0; j < EPL; ++j) {
        const int e = lane + 64 * j;
        x[q][j] = __int_as_float(__builtin_amdgcn_raw_buffer_load_b32(
            in, e < a.E ? (int)(((q0 + q) * slab + t * a.E + e) * 4) : (int)kBufferOut, 0, 0));
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
  // the order-preserving images of the scores (the routing kernels' order, NaN included)
  uint32_t key[EPL];
#pragma unroll
  for (int j = 0; j < EPL; ++j) key[j] = lane + 64 * j < a.E ? topk_key(v[j] / s) : 0u;
  if constexpr (EPL <= 2)
    if (wpt > 1) {
      // (every wave of the token has all its keys, and writes them for itself: the same values)
      constexpr int N = 64 * EPL;
      uint32_t* keys = p.keys + t * N;
      for (int j = 0; j < EPL; ++j) keys[lane + 64 * j] = key[j];
      __builtin_amdgcn_wave_barrier();
      if (wpt == 8)
        place_experts<N, 8>(a, p, keys, t, part);
      else if (wpt == 4)
        place_experts<N, 4>(a, p, keys, t, part);
      else
        place_experts<N, 2>(a, p, keys, t, part);
      return;
    }
  // K rounds of an arg-max, in a loop that is not unrolled: its scalars would not fit
  uint32_t taken = 0;
#pragma unroll 1
  for (int k = 0; k < a.K; ++k) {
    uint32_t best = 0;
    int at = INT32_MAX;  // the lane's best, the lowest expert among equals
#pragma unroll
    for (int j = 0; j < EPL; ++j) {
      const int e = lane + 64 * j;
      if (e < a.E && !((taken >> j) & 1u) && (at == INT32_MAX || key[j] > best)) {
        best = key[j];
        at = e;
      }
    }
    const uint32_t top = dpp_reduce(best, [](uint32_t x, uint32_t y) { return x > y ? x : y; });
    int e = INT32_MAX;
    if constexpr (EPL <= 2) {
#pragma unroll
      for (int j = EPL - 1; j >= 0; --j) {
        const uint64_t hit = __ballot(best == top && at >> 6 == j);
        e = hit ? 64 * j + __ffsll((unsigned long long)hit) - 1 : e;
      }
    } else {
      e = dpp_reduce(best == top ? at : INT32_MAX, [](int x, int y) { return x < y ? x : y; });
    }
    if (lane == (e & 63)) taken |= 1u << (e >> 6);
    if (lane == 0) {
      p.sel[t * a.K + k] = e;
      p.w[t * a.K + k] = topk_value(top);
    }
  }
}
__device__ __forceinline__ void select_token_of(const DecodeArgs& a, const Picked& p, int t, int part, int wpt) {
  if (a.E <= 64)
    select_token<1>(a, p, t, part, wpt);
  else if (a.E <= 128)
    select_token<2>(a, p, t, part, wpt);
  else if (a.E <= 256)
    select_token<4>(a, p, t, part, wpt);
  else if (a.E <= 512)
    select_token<8>(a, p, t, part, wpt);
  else
    select_token<16>(a, p, t, part, wpt);
}

// a token's weights: its selected scores over their sum, in the order of the selection.  One
// wave; `out`: to the caller's arrays; `all`: to every workgroup's too
__device__ __forceinline__ void weigh_token(const DecodeArgs& a, const Picked& p, int t, bool out, bool all) {
  const int lane = lane_id(), i = t * a.K + lane;
  const float x = lane < a.K ? p.w[i] : 0.f;
  float sum = 0.f;
  for (int k = 0; k < a.K; ++k) sum += __int_as_float(__builtin_amdgcn_readlane(__float_as_int(x), k));
  if (lane >= a.K) return;
  const int e = expert_within((uint32_t)p.sel[i], a.E);
  const float w = x / sum;
  p.sel[i] = e;
  p.w[i] = w;
  if (all) store8_shared(buffer_of(a.picked, (uint32_t)a.T * a.K * 8), i * 8, u32x2{(uint32_t)e, __float_as_uint(w)});
  if (out && a.topk_idx) a.topk_idx[i] = e;
  if (out && a.topk_w) a.topk_w[i] = w;
}

// the selection, by every workgroup for itself
__device__ __forceinline__ void select_all(const DecodeArgs& a, const Picked& p) {
  const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  const bool out = blockIdx.x == 0;
  const int wpt = decode_share(a.T, a.E);
  if (wpt > 1) {
    const int t = wave / wpt;
    if (t < a.T) select_token_of(a, p, t, wave % wpt, wpt);
    __syncthreads();
    if (wave < a.T) weigh_token(a, p, wave, out, false);  // (the weights are read past other barriers)
  } else {
    for (int t = wave; t < a.T; t += kDecodeWaves) {
      select_token_of(a, p, t, 0, 1);
      weigh_token(a, p, t, out, false);
    }
    __syncthreads();
  }
}
// the same of one item's tokens, for all
__device__ __forceinline__ void select_some(const DecodeArgs& a, const Picked& p, int item) {
  const int t = item * kDecodeWaves + __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  if (t >= a.T) return;
  select_token_of(a, p, t, 0, 1);
  weigh_token(a, p, t, true, true);
}
__device__ __forceinline__ void read_selection(const DecodeArgs& a, const Picked& p, bool ok) {
  for (int i = threadIdx.x; i < a.T * a.K; i += kDecodeThreads) {
    const uint64_t v = __hip_atomic_load((uint64_t*)a.picked + i, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT);
    p.sel[i] = ok ? expert_within((uint32_t)v, a.E) : i % a.K;  // (a selection even where the wait gave up)
    p.w[i] = __uint_as_float((uint32_t)(v >> 32));
  }
  __syncthreads();
}

// One token's groups are its entries (written ahead of the selection's barrier)
__device__ __forceinline__ void one_token(const DecodeArgs& a, Picked& p) {
  p.gexp = p.sel;
  if (threadIdx.x <= a.K) p.goff[threadIdx.x] = p.rows[threadIdx.x] = threadIdx.x;
}
// the groups of a selection; returns how many there are
__device__ __forceinline__ int form_groups(const DecodeArgs& a, const Picked& p, int* scan_lds) {
  const int n = a.T * a.K;
  if (a.T == 1) return n;  // (each entry its own: one_token)
  for (int e = threadIdx.x; e < a.E; e += kDecodeThreads) p.word[e] = 0ull;
  __syncthreads();
  for (int i = threadIdx.x; i < n; i += kDecodeThreads) atomicOr(&p.word[p.sel[i]], 1ull << (i / a.K));
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
      p.goff[groups + (at >> 16)] = p.first[e] = entries + (at & 0xffff);
    }
    groups += total >> 16;
    entries += total & 0xffff;
  }
  if (threadIdx.x == 0) p.goff[groups] = entries;
  __syncthreads();
  for (int i = threadIdx.x; i < n; i += kDecodeThreads) {
    const int e = p.sel[i];
    p.rows[p.first[e] + __popcll(p.word[e] & ((1ull << (i / a.K)) - 1))] = i;
  }
  __syncthreads();
  return groups;
}

// ---------------------------------------------------------------- counters
// sync, in lines of 128 bytes of their own (the polls and counts of one line wait for each
// other: eight counters in one line made a hop 3.5 us, apart they take 1): the ticket,
// eight counters of all finished up-projection items, one of selection items, one per group,
// one per column tile of finished down-projection items
constexpr int kLine = 32;
__device__ __forceinline__ int* ups_counter(const DecodeArgs& a, int i) { return a.sync + (1 + (i & 7)) * kLine; }
__device__ __forceinline__ int* select_counter(const DecodeArgs& a) { return a.sync + 9 * kLine; }
__device__ __forceinline__ int* group_counter(const DecodeArgs& a, int g) { return a.sync + (10 + g) * kLine; }
__device__ __forceinline__ int* tile_counter(const DecodeArgs& a, int t) {
  return a.sync + (10 + min(a.T * a.K, a.E) + t) * kLine;
}
__device__ __forceinline__ int take_ticket(const DecodeArgs& a) {
  return __hip_atomic_fetch_add(a.sync, 1, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT);
}
// An item's stores (shared ones), by every thread of the workgroup, before its counter.  LOADS:
// so many loads of the wave's are younger than its stores and may be under way still.
template <int LOADS>
__device__ __forceinline__ void finish_item(int* counter) {
  asm volatile("s_waitcnt vmcnt(%0)" ::"n"(LOADS) : "memory");  // each wave's own have arrived
  __syncthreads();
  if (threadIdx.x == 0) __hip_atomic_fetch_add(counter, 1, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT);
}
// Wave 0 waits until the lanes' counters (lane i's where it has one) add up to `want`; then
// the workgroup goes on.  A call that shares its workspace with another one in flight,
// which is an error, may have lost counts, or take the other's for its own: the wait is bounded
// (seconds), and false makes what the workgroup writes of O NaN.  `so_far`: no wait before
// gave up (then this one does not wait either).
constexpr int kMostPolls = 1 << 22;
template <class Counter>
__device__ __forceinline__ bool await(Counter counter, int want, int* sh, bool so_far = true) {
  if (threadIdx.x < kWave) {
    int* c = counter(lane_id());
    bool ok = false;
    for (int i = 0; i < (so_far ? kMostPolls : 1) && !ok; ++i) {
      if (i) __builtin_amdgcn_s_sleep(1);
      const int n = c ? __hip_atomic_load(c, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT) : 0;
      ok = dpp_reduce(n, [](int x, int y) { return x + y; }) >= want;
    }
    if (threadIdx.x == 0) *sh = ok;
  }
  __syncthreads();  // (the loads behind it are shared ones, which no cache answers from before)
  return so_far && *sh;
}

// ---------------------------------------------------------------- the layer
__device__ __forceinline__ void write_o(const DecodeArgs& a, int t, int col, f32x4 o, u32x2 r, bool ok) {
  if (a.R) {
    o[0] += bf_lo(r[0]);
    o[1] += bf_hi(r[0]);
    o[2] += bf_lo(r[1]);
    o[3] += bf_hi(r[1]);
  }
  if (!ok) o = f32x4{NAN, NAN, NAN, NAN};
  *(u32x2*)(a.O + (size_t)t * a.d + col) = pack_bf16x4(o[0], o[1], o[2], o[3]);
}

// O = R + sum of s Y over each token's entries, the columns of one down-projection item
__device__ __forceinline__ void sum_tokens(const DecodeArgs& a, const Picked& p, int cols, int tile, int t0, int tokens, bool ok) {
  const int C4 = cols / 4;
  const Rsrc y = buffer_of(a.Y, (uint32_t)a.T * a.K * a.d * 4);
  for (int i = threadIdx.x; i < tokens * C4; i += kDecodeThreads) {
    const int t = t0 + i / C4, col = tile * cols + 4 * (i % C4);
    if (t >= a.T) break;
    if (col >= a.d) continue;
    u32x2 res = {0, 0};
    if (a.R) res = *(const u32x2*)(a.R + (size_t)t * a.d + col);
    f32x4 o = f32x4{0.f, 0.f, 0.f, 0.f};
#pragma unroll 4
    for (int j = 0; j < a.K; ++j) {
      const f32x4 v = __builtin_bit_cast(f32x4, load16<true>(y, (uint32_t)((t * a.K + j) * a.d + col) * 4));
      const float w = p.w[t * a.K + j];
#pragma unroll
      for (int q = 0; q < 4; ++q) o[q] += w * v[q];
    }
    write_o(a, t, col, o, res, ok);
  }
}

// a token's A from the slices of H, added in slice order: put(place in [K][n], four values)
template <class Put>
__device__ __forceinline__ void token_rows(const DecodeArgs& a, const Picked& p, int t, Put put) {
  const int n = a.n, P = a.T * a.K, N = 2 * n;
  const Rsrc h = buffer_of(a.H32, (uint32_t)a.ks * P * N * 4);
  for (int i = threadIdx.x; i < a.K * n / 4; i += kDecodeThreads) {
    const int j = i / (n / 4), c = 4 * (i % (n / 4));
    f32x4 hg = f32x4{0.f, 0.f, 0.f, 0.f}, hu = hg;
    if (a.b1) {
      const float* b1 = a.b1 + (size_t)p.sel[t * a.K + j] * N + c;
      hg = *(const f32x4*)b1;
      hu = *(const f32x4*)(b1 + n);
    }
#pragma unroll 4
    for (int q = 0; q < a.ks; ++q) {
      const uint32_t o = (uint32_t)((q * P + t * a.K + j) * N + c) * 4;
      const f32x4 vg = __builtin_bit_cast(f32x4, load16<true>(h, o)), vu = __builtin_bit_cast(f32x4, load16<true>(h, o + 4 * n));
#pragma unroll
      for (int r = 0; r < 4; ++r) {
        hg[r] += vg[r];
        hu[r] += vu[r];
      }
    }
    float v[4];
#pragma unroll
    for (int r = 0; r < 4; ++r) {
      float sg;
      v[r] = silu_sig(hg[r], &sg) * hu[r];
    }
    put(j * n + c, v);
  }
}

// Y of rows first .. first + rows of an item, from the column tiles (C4 times four columns) of
// its waves' shares
template <int C4, class Item, class Sum>
__device__ __forceinline__ void store_y(const DecodeArgs& a, const Picked& p, const Item& t, int first, int rows, Sum sum) {
  const int shares = kDecodeWaves / a.kw, per_row = C4 * shares;
  for (int i = threadIdx.x; i < rows * per_row; i += kDecodeThreads) {
    const int row = i / per_row, c = i % per_row, col = 4 * (t.tile * per_row + c);
    if (col >= a.d) continue;
    f32x4 y = sum(c / C4, row, c % C4);
    if (a.b2) {
      const f32x4 bias = *(const f32x4*)(a.b2 + (size_t)t.e * a.d + col);
#pragma unroll
      for (int q = 0; q < 4; ++q) y[q] += bias[q];
    }
    store16_shared(buffer_of(a.Y, (uint32_t)a.T * a.K * a.d * 4), (uint32_t)(p.rows[t.r0 + first + row] * a.d + col) * 4,
                   __builtin_bit_cast(u32x4, y));
  }
}

// KB, MB: rows of a group in MB blocks of 16 / KB
template <int KB, int MB>
struct Decode {
  using Tile = RowTile<KB>;
  static constexpr int RT = Tile::RT, CG = Tile::CG, COLS = Tile::COLS, C4 = COLS / 4;
  // steps in flight of a wave, within the registers
  static constexpr int NBUF = 2;
  using Stream = RowStream<KB, NBUF>;
  using Part = typename Tile::Part;
  static constexpr int UP_COLS = COLS / 2, DOWN_COLS = COLS, MAX_ROWS = RT * MB;
  static size_t stage_bytes(int) { return 0; }

  // An item of a group: the up-projection of COLS / 2 gate columns and the matching up columns
  // (a.ks > 1: of a slice of k), or the down-projection of COLS columns for every a.kw waves
  struct Item {
    int gi, tile, slice, e, r0, cnt;  // (cnt: rows left, of which a pass takes RT MB)
  };
  template <bool UP>
  static __device__ __forceinline__ Item item_of(const DecodeArgs& a, const Picked& p, int i, int tiles) {
    Item t;
    t.slice = UP ? i % a.ks : 0;
    if (UP) i /= a.ks;
    t.gi = i / tiles;
    t.tile = i % tiles;
    t.e = expert_within(__builtin_amdgcn_readfirstlane(p.gexp[t.gi]), a.E);  // (of one token: ahead of weigh_token's)
    t.r0 = __builtin_amdgcn_readfirstlane(p.goff[t.gi]);
    t.cnt = __builtin_amdgcn_readfirstlane(p.goff[t.gi + 1]) - t.r0;
    return t;
  }
  template <bool UP>
  static __device__ __forceinline__ void prime(const DecodeArgs& a, const Item& t, Stream& stream, int wave) {
    const int n = a.n, d = a.d, lane = opaque_lane();
    const uint32_t bytes = (uint32_t)n * d * 2;
    if constexpr (UP) {
      const int c = t.tile * (COLS / 2) + 8 * (Tile::cg(lane) & (CG / 2 - 1));
      stream.prime(buffer_of(a.W1 + (size_t)t.e * n * d * 2, 2 * bytes), n * 4,
                   c < n ? 2 * (c + (Tile::cg(lane) >= CG / 2 ? n : 0)) : kBufferOut, t.slice * a.kslice,
                   min(d, (t.slice + 1) * a.kslice), wave, kDecodeWaves, lane);
    } else {
      const int c = COLS * (t.tile * (kDecodeWaves / a.kw) + wave / a.kw) + 8 * Tile::cg(lane);
      stream.prime(buffer_of(a.W2 + (size_t)t.e * n * d, bytes), d * 2, c < d ? 2 * c : kBufferOut, 0, n, wave % a.kw, a.kw, lane);
    }
  }
  // the rest of the product of a primed item, into A (or the slices of H) or Y
  // (before(): called by every thread ahead of the first barrier)
  template <bool UP, class Before>
  static __device__ __forceinline__ void run(const DecodeArgs& a, const Picked& p, const Item& t, Stream& stream, Part* part,
                                             char*, int wave, Before before) {
    const int n = a.n, d = a.d, N = 2 * n, P = a.T * a.K, lane = opaque_lane();
    {
      constexpr int B = MB;  // (a path of its own for fewer rows spilled)
      uint32_t xoff[B];
      f32x4 acc[B][8];
      zero_acc(acc);
#pragma unroll
      for (int b = 0; b < B; ++b) {
        const int r = RT * b + Tile::row(lane);
        const int i = r < t.cnt ? p.rows[t.r0 + r] : -1;
        xoff[b] = i < 0 ? kBufferOut : UP ? (uint32_t)(i / a.K) * d * 2 : (uint32_t)i * n * 2;
      }
      stream.template add<!UP>(acc, UP ? buffer_of(a.X, (uint32_t)a.T * d * 2) : buffer_of(a.A, (uint32_t)P * n * 2), xoff);
      before();
#pragma unroll
      for (int b = 0; b < B; ++b) {
        if (RT * b >= t.cnt) break;
        if (b) __syncthreads();
        Tile::put(part[wave], acc[b], lane);
        __syncthreads();
        const int rows = min(RT, t.cnt - RT * b);
        if (UP && a.ks == 1) {
          for (int i = threadIdx.x; i < rows * (C4 / 2); i += kDecodeThreads) {
            const int row = i / (C4 / 2), c4 = i % (C4 / 2), col = t.tile * (COLS / 2) + 4 * c4;
            if (col >= n) continue;
            f32x4 hg = Tile::template sum<kDecodeWaves>(part, row, c4);
            f32x4 hu = Tile::template sum<kDecodeWaves>(part, row, c4 + C4 / 2);
            if (a.b1) {
              const float* bias = a.b1 + (size_t)t.e * N + col;
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
            // (A to bf16, the type of the product that follows, as in the layer's forward: its
            // instruction takes no fp32, and A in two bf16 parts would double the products.  O is
            // then 2.3e-3 off, 1.7e-3 without: 16 tokens of d 4096, n 14336, E 8, K 2)
            store8_shared(buffer_of(a.A, (uint32_t)P * n * 2), (uint32_t)(p.rows[t.r0 + RT * b + row] * n + col) * 2,
                          pack_bf16x4(v[0], v[1], v[2], v[3]));
          }
          continue;
        }
        if constexpr (UP) {
          for (int i = threadIdx.x; i < rows * C4; i += kDecodeThreads) {
            const int row = i / C4, c4 = i % C4, r = p.rows[t.r0 + RT * b + row];
            const f32x4 y = Tile::template sum<kDecodeWaves>(part, row, c4);
            const int col = t.tile * (COLS / 2) + 4 * (c4 % (C4 / 2));
            if (col < n)
              store16_shared(buffer_of(a.H32, (uint32_t)a.ks * P * N * 4),
                             (uint32_t)((t.slice * P + r) * N + col + (c4 < C4 / 2 ? 0 : n)) * 4, __builtin_bit_cast(u32x4, y));
          }
          continue;
        }
        store_y<C4>(a, p, t, RT * b, rows, [&](int sub, int row, int c4) { return Tile::sum_of(part + sub * a.kw, a.kw, row, c4); });
      }
    }
  }

  // down-projection by token, with its sum: the token's K experts are one reduction of
  // K n, a wave's step 32 KB k of one expert, whose product is weighted as it is added
  template <class Wait>
  static __device__ __forceinline__ void token_down(const DecodeArgs& a, const Picked& p, typename Tile::Part* part,
                                                    char* lds, int wave, int t, int tile, Wait wait) {
    constexpr int NB = 2;
    uint16_t* rows = (uint16_t*)lds;  // [K][n] with slices of H
    const int n = a.n, d = a.d, spe = (n + Tile::KSTEP - 1) / Tile::KSTEP, steps = a.K * spe, lane = opaque_lane();
    const uint32_t wcol = 2 * (tile * COLS + 8 * Tile::cg(lane));
    u32x4 wv[NB][8];
    bf16x8 xv[NB];
    auto entry = [&](int s) { return t * a.K + min(wave + kDecodeWaves * s, steps - 1) / spe; };
    auto first_k = [&](int s) { return min(wave + kDecodeWaves * s, steps - 1) % spe * Tile::KSTEP + Tile::k0(lane); };
    auto load_w = [&](int buf, int s) {
      const int e = expert_within(__builtin_amdgcn_readfirstlane(p.sel[entry(s)]), a.E), k = first_k(s);
      const Rsrc w = buffer_of(a.W2 + (size_t)e * n * d, (uint32_t)n * d * 2);
      const uint32_t o = wave + kDecodeWaves * s < steps && k < n ? wcol + (uint32_t)k * d * 2 : kBufferOut;
#pragma unroll
      for (int i = 0; i < 8; ++i) wv[buf][i] = load16(w, o + i * d * 2);
    };
    auto load_x = [&](int buf, int s) {
      const int k = first_k(s);
      if (a.ks > 1)
        xv[buf] = __builtin_bit_cast(bf16x8, k < n ? *(const u32x4*)(rows + (entry(s) - t * a.K) * n + k) : u32x4{0, 0, 0, 0});
      else
        xv[buf] = __builtin_bit_cast(bf16x8, load16<true>(buffer_of(a.A, (uint32_t)a.T * a.K * n * 2),
                                                          k < n ? (uint32_t)(entry(s) * n + k) * 2 : kBufferOut));
    };
#pragma unroll
    for (int q = 0; q < NB; ++q) load_w(q, q);
    // what else the end needs
    const int col = tile * COLS + 4 * threadIdx.x;
    u32x2 res = {0, 0};
    f32x4 bias = f32x4{0.f, 0.f, 0.f, 0.f};
    if (threadIdx.x < C4) {
      if (a.R) res = *(const u32x2*)(a.R + (size_t)t * d + col);
      if (a.b2)
        for (int j = 0; j < a.K; ++j) {
          const f32x4 v = *(const f32x4*)(a.b2 + (size_t)p.sel[t * a.K + j] * d + col);
#pragma unroll
          for (int q = 0; q < 4; ++q) bias[q] += p.w[t * a.K + j] * v[q];
        }
    }
    wait();
    if (a.ks > 1) {
      // (A to bf16, as in run)
      token_rows(a, p, t, [&](int i, const float(&v)[4]) { *(u32x2*)(rows + i) = pack_bf16x4(v[0], v[1], v[2], v[3]); });
      __syncthreads();
    }
#pragma unroll
    for (int q = 0; q < NB; ++q) load_x(q, q);
    f32x4 acc[8];
#pragma unroll
    for (int j = 0; j < 8; ++j) acc[j] = f32x4{0.f, 0.f, 0.f, 0.f};
    const int ns = (steps - wave + kDecodeWaves - 1) / kDecodeWaves;
    auto run = [&]() __attribute__((always_inline)) {
      if (ns <= 0) return;
      for (int s = 0;; s += NB) {
#pragma unroll
        for (int q = 0; q < NB; ++q) {
          const float sw = p.w[entry(s + q)];
#pragma unroll
          for (int j = 0; j < 8; ++j) {
            const f32x4 y = __builtin_amdgcn_mfma_f32_16x16x32_bf16(xv[q], column_of8(wv[q], j), f32x4{0.f, 0.f, 0.f, 0.f}, 0, 0, 0);
#pragma unroll
            for (int r = 0; r < 4; ++r) acc[j][r] += sw * y[r];
          }
          if (s + q + 1 >= ns) return;
          load_w(q, s + q + NB);
          load_x(q, s + q + NB);
        }
      }
    };
    run();
    // (every row of the product's k block is this token)
    Tile::put(part[wave], acc, lane);
    __syncthreads();
    if (threadIdx.x < C4 * kDecodeWaves) {  // lanes of four columns, one for each wave's sums
      static_assert(C4 * kDecodeWaves <= kWave);
      const int c4 = threadIdx.x % C4, w = threadIdx.x / C4;
      f32x4 o = f32x4{0.f, 0.f, 0.f, 0.f};
#pragma unroll
      for (int b = 0; b < KB; ++b) {
        const f32x4 v = part[w][b][0][c4 & 1][c4 >> 1];
#pragma unroll
        for (int q = 0; q < 4; ++q) o[q] += v[q];
      }
#pragma unroll
      for (int q = 0; q < 4; ++q) {
#pragma unroll
        for (int i = C4; i < C4 * kDecodeWaves; i *= 2) o[q] += __shfl_xor(o[q], i, kWave);
        o[q] += bias[q];
      }
      if (threadIdx.x < C4) write_o(a, t, col, o, res, wait.ok());
    }
  }
};

// The same with 8-bit weights (stream8_tile.h): a wave's step is one block of 128 k of 64 weight
// columns, in the up-projection 32 gate columns and the matching up ones.  Rows are quantised
// as they are loaded, X from bf16 and A from fp32.  The up-projection's codes are multiplied
// in bf16 (exact products), with fp32 sums: the 8-bit instruction's are 1.3e-5 of the result
// off, which moves A's codes, and now and then a whole block's scale, to the other side of a
// step (6 tokens of d 1536, n 256, E 128, K 8: one token's O 7e-3 off, so 1.7e-3).  It costs
// 2%, since the weights bound it (32 tokens of a 30B-shaped layer: 148 us, 151 so).  The
// down-projection's sums are the 8-bit instruction's, as moe_fwd_quant's: no code follows
// that they could move, and 1.3e-5 is far below O's own rounding.  MB = 2 is for groups of
// more than 16 rows.
template <int MB, int NJ>
struct Decode8 {
  static constexpr int NBUF = 1, UP_COLS = 8 * NJ, DOWN_COLS = 16 * NJ, MAX_ROWS = 16 * MB;
  static size_t stage_bytes(int n) { return (size_t)q_blocks(n) * MB * kStageBlock; }
  typedef Stream8Part<NJ> Part;
  using Item = typename Decode<1, 1>::Item;
  struct Stream {
    Rsrc w;
    const uint8_t* ws[2];
    uint32_t row[NJ];
    // This wave's first block, the end, from a block to the next, and its steps, which begin
    // at step `rot`: where rows are 4 KB apart, one block of them all lies in few memory channels,
    // and items that all began there would ask the same ones (32 tokens of a 30B-shaped layer:
    // 162 us, 151 so; 64 184 and 170)
    int kb, end, step, ns, rot;
    __device__ __forceinline__ void turn(int by) {
      ns = max((end - kb + step - 1) / step, 1);
      rot = by % ns;
    }
    __device__ __forceinline__ int block(int s) const {  // (past the end: the last one again, unused)
      const int i = min(s, ns - 1) + rot;
      return min(kb + step * (i >= ns ? i - ns : i), end - 1);
    }
    u32x4 wv[NBUF][NJ][2];
    int sv[NBUF][2];
    __device__ __forceinline__ void load(int buf, int s) {
      const int b = block(s);
#pragma unroll
      for (int j = 0; j < NJ; ++j) {
        wv[buf][j][0] = load16(w, row[j] + kQBlock * b);
        wv[buf][j][1] = load16(w, row[j] + kQBlock * b + 64);
      }
      sv[buf][0] = ws[0][b];
      sv[buf][1] = ws[1][b];
    }
    __device__ __forceinline__ i32x8 frag(int buf, int j) const {
      const u32x4 lo = wv[buf][j][0], hi = wv[buf][j][1];
      return i32x8{(int)lo[0], (int)lo[1], (int)lo[2], (int)lo[3], (int)hi[0], (int)hi[1], (int)hi[2], (int)hi[3]};
    }
  };
  template <bool UP>
  static __device__ __forceinline__ Item item_of(const DecodeArgs& a, const Picked& p, int i, int tiles) {
    return Decode<1, 1>::template item_of<UP>(a, p, i, tiles);
  }
  template <bool UP>
  static __device__ __forceinline__ void prime(const DecodeArgs& a, const Item& t, Stream& s, int wave) {
    const int lane = opaque_lane(), g = lane >> 4, l = lane & 15, d = a.d, n = a.n;
    int c0 = 0;
    if constexpr (UP) {
      s.w = buffer_of(a.W1q + (size_t)t.e * w1q_bytes(d, n), (uint32_t)w1q_bytes(d, n));
      const uint8_t* ws = a.W1s + (size_t)t.e * w1s_bytes(d, n) + (size_t)(2 * (UP_COLS * t.tile / kQBlock)) * q_stride(d / kQBlock);
      s.ws[0] = ws;
      s.ws[1] = ws + q_stride(d / kQBlock);
      s.kb = t.slice * (a.kslice / kQBlock) + wave;
      s.end = min(d, (t.slice + 1) * a.kslice) / kQBlock;
      s.step = kDecodeWaves;
      s.turn(t.tile);
    } else {
      s.w = buffer_of(a.W2q + (size_t)t.e * w2q_bytes(d, n), (uint32_t)w2q_bytes(d, n));
      // (past the last column: the last tile's again, not stored)
      c0 = min(DOWN_COLS * (t.tile * (kDecodeWaves / a.kw) + wave / a.kw), d - DOWN_COLS);
      s.ws[0] = s.ws[1] = a.W2s + (size_t)t.e * w2s_bytes(d, n) + (size_t)(c0 / kQBlock) * q_stride(q_blocks(n));
      s.kb = wave % a.kw;
      s.step = a.kw;
      s.end = q_blocks(n);
      s.turn(t.tile);
    }
#pragma unroll
    for (int j = 0; j < NJ; ++j) {
      const int c = 16 * j + l, col = UP_COLS * t.tile + c % UP_COLS;
      s.row[j] = 16 * g + (UP ? (uint32_t)(256 * (col / kQBlock) + w1q_row(col % kQBlock, c / UP_COLS)) * d
                                : (uint32_t)(c0 + c) * q_pad(n));
    }
#pragma unroll
    for (int q = 0; q < NBUF; ++q) s.load(q, q);
  }
  // the values of a row's block of 128 that a lane holds: 16 from k on and 16 from k + 64 on
  template <bool F32>
  static __device__ __forceinline__ void load_row(RowBlock8<F32>& x, Rsrc r, uint32_t off, int k, int len) {
    constexpr int N = RowBlock8<F32>::N, ES = F32 ? 4 : 2;
#pragma unroll
    for (int i = 0; i < N; ++i) {
      const int kk = k + (i >= N / 2 ? 64 : 0);
      x.v[i] = load16<F32>(r, kk < len ? off + (uint32_t)kk * ES + 16 * (i % (N / 2)) : kBufferOut);
    }
  }
  // The rows of a step: quantised from what was loaded for it, or (F32, where column tiles share
  // them) codes in LDS, a kStageBlock for each block and row block.
  static constexpr int kStageBlock = kWave * 36;
  template <bool F32, bool STAGED, class Row>
  static __device__ __forceinline__ void add(Stream& s, f32x4 (&acc)[MB][NJ], const char* stage, int lane, Row row) {
    const int ns = s.ns;
    if (s.kb >= s.end) return;
    RowBlock8<F32> xv[STAGED ? 1 : NBUF][MB];
    auto load_x = [&](int q, int i) {
      if constexpr (!STAGED)
#pragma unroll
        for (int b = 0; b < MB; ++b) row(xv[q][b], b, s.block(i));
    };
#pragma unroll
    for (int q = 0; q < NBUF; ++q) load_x(q, q);
    for (int i = 0;; i += NBUF) {
#pragma unroll
      for (int q = 0; q < NBUF; ++q) {
#pragma unroll
        for (int b = 0; b < MB; ++b) {
          int xs;
          i32x8 x;
          if constexpr (STAGED) {
            const char* at = stage + (s.block(i + q) * MB + b) * kStageBlock;
            const u32x4 lo = *(const u32x4*)(at + 16 * lane), hi = *(const u32x4*)(at + 16 * (kWave + lane));
            x = i32x8{(int)lo[0], (int)lo[1], (int)lo[2], (int)lo[3], (int)hi[0], (int)hi[1], (int)hi[2], (int)hi[3]};
            xs = *(const int*)(at + 32 * kWave + 4 * lane);
          } else {
            x = xv[q][b].codes(&xs);
          }
#pragma unroll
          for (int j = 0; j < NJ; ++j) {
            const int ws = s.sv[q][2 * j / NJ];
            if constexpr (!F32) {
              f32x4 y = f32x4{0.f, 0.f, 0.f, 0.f};
#pragma unroll
              for (int h = 0; h < 4; ++h)
                y = __builtin_amdgcn_mfma_f32_16x16x32_bf16(codes_bf16(s.frag(q, j), h, 1.f), codes_bf16(x, h, 1.f), y, 0, 0, 0);
#pragma unroll
              for (int h = 0; h < 4; ++h) acc[b][j][h] += ldexpf(y[h], ws + xs - 254);
            } else {
              acc[b][j] = __builtin_amdgcn_mfma_scale_f32_16x16x128_f8f6f4(s.frag(q, j), x, acc[b][j], 0, 0, 0, ws, 0, xs);
            }
          }
        }
        if (i + q + 1 >= ns) return;
        __builtin_amdgcn_sched_barrier(0);  // (not ahead of the products: it would take registers of their own)
        s.load(q, i + q + NBUF);
        load_x(q, i + q + NBUF);
        __builtin_amdgcn_sched_barrier(0);
      }
    }
  }
  template <bool UP, class Before>
  static __device__ __forceinline__ void run(const DecodeArgs& a, const Picked& p, const Item& t, Stream& s, Part* part,
                                             char* stage, int wave, Before before) {
    const int cnt = min(t.cnt, MAX_ROWS);
    const int n = a.n, d = a.d, N = 2 * n, P = a.T * a.K, lane = opaque_lane(), g = lane >> 4, l = lane & 15;
    uint32_t xoff[MB];
    f32x4 acc[MB][NJ];
#pragma unroll
    for (int b = 0; b < MB; ++b) {
      // (a lane past the rows reads the last one's again)
      const int i = p.rows[t.r0 + min(16 * b + l, cnt - 1)];
      xoff[b] = UP ? (uint32_t)(i / a.K) * d * 2 : (uint32_t)i * n * 4;
#pragma unroll
      for (int j = 0; j < NJ; ++j) acc[b][j] = f32x4{0.f, 0.f, 0.f, 0.f};
    }
    const Rsrc r = UP ? buffer_of(a.X, (uint32_t)a.T * d * 2) : buffer_of(a.A32, (uint32_t)P * n * 4);
    auto row = [&](RowBlock8<!UP>& x, int b, int kb) { load_row(x, r, xoff[b], kQBlock * kb + 16 * g, UP ? d : n); };
    if constexpr (UP) {
      add<false, false>(s, acc, nullptr, lane, row);
    } else if (a.kw == kDecodeWaves) {
      add<true, false>(s, acc, nullptr, lane, row);
    } else {
      // (a wave for each block; 64 tokens of d 4096, n 1792, E 16, K 2 114 us without, 105 so; of
      // n 512, E 128, K 8 172.6 and 170.1)
      for (int kb = wave; kb < q_blocks(n); kb += kDecodeWaves)
#pragma unroll
        for (int b = 0; b < MB; ++b) {
          RowBlock8<true> x;
          row(x, b, kb);
          int xs;
          const i32x8 c = x.codes(&xs);
          char* at = stage + (kb * MB + b) * kStageBlock;
          *(u32x4*)(at + 16 * lane) = u32x4{(uint32_t)c[0], (uint32_t)c[1], (uint32_t)c[2], (uint32_t)c[3]};
          *(u32x4*)(at + 16 * (kWave + lane)) = u32x4{(uint32_t)c[4], (uint32_t)c[5], (uint32_t)c[6], (uint32_t)c[7]};
          *(int*)(at + 32 * kWave + 4 * lane) = xs;
        }
      __syncthreads();
      add<true, true>(s, acc, stage, lane, row);
    }
    before();
#pragma unroll
    for (int b = 0; b < MB; ++b) {
      if (16 * b >= cnt) break;
      if (b) __syncthreads();
#pragma unroll
      for (int j = 0; j < NJ; ++j) part[wave][l][4 * j + g] = acc[b][j];
      __syncthreads();
      const int rows = min(16, cnt - 16 * b);
      constexpr int C4 = 4 * NJ;
      if (UP && a.ks == 1) {
        for (int i = threadIdx.x; i < rows * (C4 / 2); i += kDecodeThreads) {
          const int row = i / (C4 / 2), c4 = i % (C4 / 2), col = UP_COLS * t.tile + 4 * c4;
          f32x4 hg = stream8_sum<kDecodeWaves, NJ>(part, row, c4), hu = stream8_sum<kDecodeWaves, NJ>(part, row, c4 + C4 / 2), v;
          const float* b1 = a.b1 ? a.b1 + (size_t)t.e * N + col : nullptr;
#pragma unroll
          for (int q = 0; q < 4; ++q) {
            if (b1) {
              hg[q] += b1[q];
              hu[q] += b1[n + q];
            }
            float sg;
            v[q] = silu_sig(hg[q], &sg) * hu[q];
          }
          store16_shared(buffer_of(a.A32, (uint32_t)P * n * 4), (uint32_t)(p.rows[t.r0 + 16 * b + row] * n + col) * 4,
                         __builtin_bit_cast(u32x4, v));
        }
        continue;
      }
      if constexpr (UP) {
        for (int i = threadIdx.x; i < rows * C4; i += kDecodeThreads) {
          const int row = i / C4, c4 = i % C4, r = p.rows[t.r0 + 16 * b + row];
          const f32x4 y = stream8_sum<kDecodeWaves, NJ>(part, row, c4);
          const int col = UP_COLS * t.tile + 4 * (c4 % (C4 / 2));
          store16_shared(buffer_of(a.H32, (uint32_t)a.ks * P * N * 4),
                         (uint32_t)((t.slice * P + r) * N + col + (c4 < C4 / 2 ? 0 : n)) * 4, __builtin_bit_cast(u32x4, y));
        }
        continue;
      }
      store_y<C4>(a, p, t, 16 * b, rows, [&](int sub, int row, int c4) {
        f32x4 y = part[sub * a.kw][row][c4];
        for (int w = 1; w < a.kw; ++w)
#pragma unroll
          for (int q = 0; q < 4; ++q) y[q] += part[sub * a.kw + w][row][c4][q];
        return y;
      });
    }
  }

  // by token: 32 columns, a wave's step one block of one entry, weighted as it is added
  struct Token {
    static constexpr int COLS = 32, C4 = COLS / 4;
    typedef f32x4 Part[C4];
    template <class Wait>
    static __device__ __forceinline__ void token_down(const DecodeArgs& a, const Picked& p, Part* part, char* lds, int wave, int t,
                                                      int tile, Wait wait) {
      constexpr int NB = 2, J = 2;
      const int n = a.n, d = a.d, blocks = q_blocks(n), steps = a.K * blocks, ns = (steps - wave + kDecodeWaves - 1) / kDecodeWaves;
      const int lane = opaque_lane(), g = lane >> 4, l = lane & 15;
      float* rows = (float*)lds;  // [K][n] with slices of H
      u32x4 wv[NB][J][2];
      int sv[NB];
      auto at = [&](int s) { return min(wave + kDecodeWaves * s, steps - 1); };
      auto load_w = [&](int q, int s) {
        const int i = at(s), kb = i % blocks, e = expert_within(__builtin_amdgcn_readfirstlane(p.sel[t * a.K + i / blocks]), a.E);
        const uint8_t* w = a.W2q + (size_t)e * w2q_bytes(d, n) + 16 * g + kQBlock * kb;
#pragma unroll
        for (int j = 0; j < J; ++j) {
          const uint8_t* row = w + (size_t)(COLS * tile + 16 * j + l) * q_pad(n);
          wv[q][j][0] = *(const u32x4*)row;
          wv[q][j][1] = *(const u32x4*)(row + 64);
        }
        sv[q] = (a.W2s + (size_t)e * w2s_bytes(d, n) + (size_t)(COLS * tile / kQBlock) * q_stride(blocks))[kb];
      };
#pragma unroll
      for (int q = 0; q < NB; ++q) load_w(q, q);
      // what else the end needs
      const int col = tile * COLS + 4 * threadIdx.x;
      u32x2 res = {0, 0};
      f32x4 bias = f32x4{0.f, 0.f, 0.f, 0.f};
      if (threadIdx.x < C4) {
        if (a.R) res = *(const u32x2*)(a.R + (size_t)t * d + col);
        if (a.b2)
          for (int j = 0; j < a.K; ++j) {
            const f32x4 v = *(const f32x4*)(a.b2 + (size_t)p.sel[t * a.K + j] * d + col);
#pragma unroll
            for (int q = 0; q < 4; ++q) bias[q] += p.w[t * a.K + j] * v[q];
          }
      }
      wait();
      if (a.ks > 1) {
        token_rows(a, p, t, [&](int i, const float(&v)[4]) { *(f32x4*)(rows + i) = f32x4{v[0], v[1], v[2], v[3]}; });
        __syncthreads();
      }
      f32x4 acc[J];
#pragma unroll
      for (int j = 0; j < J; ++j) acc[j] = f32x4{0.f, 0.f, 0.f, 0.f};
      const Rsrc x = buffer_of(a.A32, (uint32_t)a.T * a.K * n * 4);
      auto run = [&]() __attribute__((always_inline)) {
        if (ns <= 0) return;
        for (int s = 0;; s += NB) {
#pragma unroll
          for (int q = 0; q < NB; ++q) {
            const int i = at(s + q), kb = i % blocks, j0 = i / blocks, k = kQBlock * kb + 16 * g;
            RowBlock8<true> xv;
            if (a.ks > 1) {
#pragma unroll
              for (int h = 0; h < 8; ++h) {
                const int kk = k + (h >= 4 ? 64 : 0);
                xv.v[h] = kk < n ? *(const u32x4*)(rows + j0 * n + kk + 4 * (h % 4)) : u32x4{0, 0, 0, 0};
              }
            } else {
              load_row(xv, x, (uint32_t)(t * a.K + j0) * n * 4, k, n);
            }
            int xs;
            const i32x8 c = xv.codes(&xs);
            const float sw = p.w[t * a.K + j0];
#pragma unroll
            for (int j = 0; j < J; ++j) {
              const u32x4 lo = wv[q][j][0], hi = wv[q][j][1];
              const i32x8 wf = {(int)lo[0], (int)lo[1], (int)lo[2], (int)lo[3], (int)hi[0], (int)hi[1], (int)hi[2], (int)hi[3]};
              const f32x4 y = __builtin_amdgcn_mfma_scale_f32_16x16x128_f8f6f4(wf, c, f32x4{0.f, 0.f, 0.f, 0.f}, 0, 0, 0, sv[q], 0, xs);
#pragma unroll
              for (int r = 0; r < 4; ++r) acc[j][r] += sw * y[r];
            }
            if (s + q + 1 >= ns) return;
            load_w(q, s + q + NB);
          }
        }
      };
      run();
      if (l == 0)  // (all 16 rows of the product are this one)
#pragma unroll
        for (int j = 0; j < J; ++j) part[wave][4 * j + g] = acc[j];
      __syncthreads();
      if (threadIdx.x < C4 * kDecodeWaves) {
        const int c4 = threadIdx.x % C4, w = threadIdx.x / C4;
        f32x4 o = part[w][c4];
#pragma unroll
        for (int q = 0; q < 4; ++q) {
#pragma unroll
          for (int i = C4; i < C4 * kDecodeWaves; i *= 2) o[q] += __shfl_xor(o[q], i, kWave);
          o[q] += bias[q];
        }
        if (threadIdx.x < C4) write_o(a, t, col, o, res, wait.ok());
      }
    }
  };
};

// tokens of one item of the sums
__host__ __device__ inline int sum_tokens_of(int cols) { return 4096 / cols; }

// D: Decode or Decode8; TD: its down-projection by token
template <class D, class TD, bool BY_TOKEN>
__global__ __launch_bounds__(kDecodeThreads, 2) void decode_kernel(const DecodeArgs a) {
  extern __shared__ __attribute__((aligned(16))) char dyn[];  // picked_bytes, and a token's rows
  __shared__ typename D::Part part[kDecodeWaves];
  static_assert(sizeof(typename TD::Part) <= sizeof(typename D::Part), "the partial sums' area");
  __shared__ int sh[2];
  __shared__ int scan_lds[kDecodeWaves];
  Picked p = picked_at(dyn, a.T, a.E, a.K);
  if (a.T == 1) one_token(a, p);
  const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  if (threadIdx.x == kDecodeThreads - 1) sh[0] = take_ticket(a);  // (asked for ahead of the selection)
  // Up to 8 tokens every workgroup selects for itself.  More are the queue's first items, of 8
  // tokens each (a wave takes 3.8 us for one, and 64 would take 30).
  bool ok = true;  // (the waits so far)
  const int selects = a.T <= kDecodeWaves ? 0 : (a.T + kDecodeWaves - 1) / kDecodeWaves;
  int item;
  if (selects == 0) {
    select_all(a, p);
    item = next_item(-1, __builtin_amdgcn_readfirstlane(sh[0]));
  } else {
    __syncthreads();
    for (item = -1;;) {
      item = next_item(item, __builtin_amdgcn_readfirstlane(sh[0]));
      if (item >= selects) break;
      select_some(a, p, item);
      finish_item<0>(select_counter(a));
      if (threadIdx.x == 0) sh[0] = take_ticket(a);
      __syncthreads();
    }
    item -= selects;
    ok = await([&](int l) { return l == 0 ? select_counter(a) : nullptr; }, selects, sh + 1);
    read_selection(a, p, ok);
  }
  const int groups = __builtin_amdgcn_readfirstlane(form_groups(a, p, scan_lds));
  const int up_tiles = (a.n + D::UP_COLS - 1) / D::UP_COLS, down_cols = BY_TOKEN ? TD::COLS : D::DOWN_COLS * (kDecodeWaves / a.kw);
  const int down_tiles = (a.d + down_cols - 1) / down_cols, sum_rows = sum_tokens_of(down_cols);
  const int per_group = up_tiles * a.ks, ups = groups * per_group, downs = (BY_TOKEN ? a.T : groups) * down_tiles;
  const int sums = BY_TOKEN ? 0 : down_tiles * ((a.T + sum_rows - 1) / sum_rows);
  const int total = ups + downs + sums;
  // Where every item has a workgroup, no one asks for a second ticket (each costs 11 ns of all
  // the others' time).  Else the next ticket is asked for before an item's work, and the next
  // item's first weights between this one's stores and its count.
  const bool more = selects || total > (int)gridDim.x;
  const int last = BY_TOKEN ? ups : ups + downs;  // of the items of groups
  // the items [.., end) of one kind, from item - from on
  auto kind = [&](auto up_c, int from, int end) __attribute__((always_inline)) {
    constexpr bool UP = decltype(up_c)::value;
    if (item >= end) return;
    typename D::Stream stream;
    typename D::Item t = D::template item_of<UP>(a, p, item - from, UP ? up_tiles : down_tiles);
    D::template prime<UP>(a, t, stream, wave);
    for (;;) {
      int next = 0;
      if (more && threadIdx.x == 0) next = take_ticket(a);
      int* counter = !UP ? tile_counter(a, t.tile) : BY_TOKEN ? ups_counter(a, item) : group_counter(a, t.gi);
      if constexpr (!UP) ok = await([&](int l) { return l == 0 ? group_counter(a, t.gi) : nullptr; }, per_group, sh + 1, ok);
      while (t.cnt > D::MAX_ROWS) {  // (more rows than a pass takes: the weights again)
        D::template run<UP>(a, p, t, stream, part, dyn + picked_bytes(a.T, a.E, a.K), wave, []() {});
        t.r0 += D::MAX_ROWS;
        t.cnt -= D::MAX_ROWS;
        D::template prime<UP>(a, t, stream, wave);
        __syncthreads();
      }
      D::template run<UP>(a, p, t, stream, part, dyn + picked_bytes(a.T, a.E, a.K), wave, [&]() {
        if (more && threadIdx.x == 0) sh[0] = next;
      });
      item = more ? next_item(item + selects, __builtin_amdgcn_readfirstlane(sh[0])) - selects : total;
      asm volatile("" ::: "memory");
      if (!ok) counter = a.sync + 1;  // (no one's: what gave up is not counted, so that nothing is summed from it)
      if (item >= end) {
        finish_item<0>(counter);
        return;
      }
      t = D::template item_of<UP>(a, p, item - from, UP ? up_tiles : down_tiles);
      D::template prime<UP>(a, t, stream, wave);
      finish_item<8 * D::NBUF>(counter);
    }
  };
  kind(std::true_type{}, 0, ups);
  if constexpr (!BY_TOKEN) kind(std::false_type{}, ups, last);
  while (item < total) {
    const int i = item - last, tile = i % down_tiles;
    if constexpr (BY_TOKEN) {
      // (all up-projections: the token's own are seldom done much earlier)
      struct {
        const DecodeArgs& a; int ups; int* sh; bool* all;
        __device__ __forceinline__ void operator()() const {
          *all = await([&](int l) { return l < 8 ? ups_counter(a, l) : nullptr; }, ups, sh, *all);
        }
        __device__ bool ok() const { return *all; }
      } wait{a, ups, sh + 1, &ok};
      TD::token_down(a, p, (typename TD::Part*)part, dyn + picked_bytes(a.T, a.E, a.K), wave, i / down_tiles, tile, wait);
    } else {
      ok = await([&](int l) { return l == 0 ? tile_counter(a, tile) : nullptr; }, groups, sh + 1, ok);
      sum_tokens(a, p, down_cols, tile, i / down_tiles * sum_rows, sum_rows, ok);
    }
    if (!more) break;
    if (threadIdx.x == 0) sh[0] = take_ticket(a);
    __syncthreads();
    item = next_item(item + selects, __builtin_amdgcn_readfirstlane(sh[0])) - selects;
    __syncthreads();  // (sh and the partial sums are free again)
  }
}

// ---------------------------------------------------------------- host
int decode_slices(int T, int d, int E) {
  // up to about 64 workgroups, of a step or more for each wave
  const int tiles = (E + 127) / 128 * ((T + 15) / 16);
  const int want = std::max(1, std::min(64 / tiles, d / (32 * kDecodeWaves)));
  const int per = (d / 32 + want - 1) / want;
  return (d / 32 + per - 1) / per;
}
size_t decode_sync_words(int T, int d, int E, int K) { return (size_t)kLine * (10 + std::min(T * K, E) + d / 32); }
// whether the down-projection goes by token: where few entries repeat experts, whose weights are
// then read again, and the items leave CUs for the up-projection's (two tokens of d 1536, n 256,
// E 128, K 8 25.4 us, by group 27.1; four 35.4, 33.0).  decode_ks: the slices of k
static bool decode_by_token(int T, int d, int E, int K) { return T == 1 || (2 * T * K <= E && T * (d / 32) <= 160); }
int decode_ks(int T, int d, int n, int E, int K, bool q8) {
  if (!decode_by_token(T, d, E, K) || K * n > 8192) return 1;
  // about a workgroup to a CU with the down-projection's, and a step for each wave at least
  const int items = T * K * ((n + 63) / 64) * (q8 ? 2 : 1), rest = std::max(128, 256 - T * (d / 32));
  return std::max(1, std::min({rest / items, q8 ? (d + 1023) / 1024 : d / 256, 8}));
}

static hipError_t run_router(const DecodeArgs& a, hipStream_t s) {
  using Tile = RowTile<1>;
  const int per = (a.d / 32 + a.slices - 1) / a.slices;
  const dim3 grid((a.E + Tile::COLS - 1) / Tile::COLS, a.slices, (a.T + Tile::RT - 1) / Tile::RT);
  decode_router_kernel<<<grid, kDecodeThreads, 0, s>>>(a, 32 * per, (int)decode_sync_words(a.T, a.d, a.E, a.K));
  return hipGetLastError();
}

template <class D, class TD, bool BY_TOKEN>
static hipError_t run_decode(const DecodeArgs& a, hipStream_t s) {
  const int down_cols = BY_TOKEN ? TD::COLS : D::DOWN_COLS * (kDecodeWaves / a.kw), sum_rows = sum_tokens_of(down_cols);
  const int64_t groups = std::min(a.T * a.K, a.E), down_tiles = (a.d + down_cols - 1) / down_cols;
  int64_t items = groups * ((a.n + D::UP_COLS - 1) / D::UP_COLS) * a.ks;
  items += BY_TOKEN ? a.T * down_tiles : (groups + (a.T + sum_rows - 1) / sum_rows) * down_tiles;
  size_t lds = picked_bytes(a.T, a.E, a.K);  // and a token's rows, or the codes of an item's
  if (a.ks > 1)
    lds += (a.W1q ? 4 : 2) * (size_t)a.K * a.n;
  else if (!BY_TOKEN && a.kw < kDecodeWaves)
    lds += D::stage_bytes(a.n);
  decode_kernel<D, TD, BY_TOKEN><<<(int)std::min<int64_t>(items, 256), kDecodeThreads, lds, s>>>(a);
  return hipGetLastError();
}

hipError_t launch_decode(DecodeArgs a, hipStream_t s) {
  const bool q8 = a.W1q != nullptr, by_token = decode_by_token(a.T, a.d, a.E, a.K);
  const int unit = q8 ? kQBlock : 32;  // of a slice
  a.slices = decode_slices(a.T, a.d, a.E);
  a.ks = decode_ks(a.T, a.d, a.n, a.E, a.K, q8);
  a.kslice = (a.d / unit + a.ks - 1) / a.ks * unit;
  // waves of a down-projection column tile: two steps each, where there are as many
  const int steps = q8 ? q_blocks(a.n) : a.n / 32;
  a.kw = 1;
  // (8-bit: one step each, while the items are fewer than two to a CU: 9 tokens of d 1536, n 256,
  // E 128, K 8 46.3 us, 38.8 so; in 16 bits 46.9 and 47.5, and 7 tokens of the 1B layer 27.2 and 29.2)
  const int64_t groups = std::min(a.T * a.K, a.E);
  while (2 * a.kw <= kDecodeWaves &&
         (4 * a.kw <= steps || (q8 && 2 * a.kw <= steps && groups * a.d * a.kw < 512 * 64 * kDecodeWaves)))
    a.kw *= 2;
  const hipError_t e = run_router(a, s);
  if (e != hipSuccess) return e;
  // one row block where a group seldom has more than its 16 rows
  const bool one = a.T <= 16 || a.T * a.K <= 6 * a.E;
  using Q1 = Decode8<1, 4>;
  using B1 = Decode<1, 1>;
  using BT = Decode<4, 1>;
  if (q8) {
    if (by_token) return run_decode<Q1, Q1::Token, true>(a, s);
    // smaller tiles for few items (8 tokens of d 1024, n 256, E 64, K 8 27.2 us, 27.7 in the
    // larger; 16 of d 1536, n 256, E 128, K 8 45.5 and 42.5)
    if (a.T * a.K <= 64) return run_decode<Q1, Q1::Token, false>(a, s);
    return one ? run_decode<Decode8<1, 8>, Q1::Token, false>(a, s) : run_decode<Decode8<2, 4>, Q1::Token, false>(a, s);
  }
  if (by_token) return run_decode<B1, BT, true>(a, s);
  return one ? run_decode<B1, BT, false>(a, s) : run_decode<Decode<1, 2>, BT, false>(a, s);
}

}  // namespace smoe

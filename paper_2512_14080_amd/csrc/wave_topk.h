// The top K of one token by a wave, shared by the routing kernels and the layer for a
// few tokens.
#pragma once
#include "device_common.h"
#include "topk_net.h"

namespace smoe {

// The top K of one token, a wave per token (value j of lane l is expert 64 j +
// l), ordered by (value desc, expert asc): put(k, e, w) is called once for each
// of the K positions, by some lane, with w the value over the selected values'
// sum (added in ascending expert order).
//
// Small K: K rounds of a wave-wide arg-max (six dependent DPP steps each).
// Larger K, EPL <= 16 (beyond, the masks would not fit the scalar registers): a
// select over the bits of the 32-bit keys, most significant first, on ballots.  The
// candidates with the bit set replace the candidates if they are as many as still
// wanted, else they are selected and the others stay; it stops once the candidates
// are exactly as many as wanted, after about half of the bits.  Equal keys at the
// end go to the lowest experts (lowest j, then lowest lane).  Scalar masks and
// counts, one vector compare per bit, whatever K.  us of the top-K launch, rounds /
// bits:
//   T = 4096, E = 64     K = 1 6.7 / 7.3    4 7.5 / 7.9    6 8.2 / 8.5    8 9.3 / 8.7    16 12.0 / 9.3
//   T = 16, E = 64             7.3 / 8.8      9.0 / 8.5      9.7 / 8.6     11.1 / 9.2      14.1 / 10.2
//   T = 4096, E = 256          8.1 / 11.5     9.9 / 13.0    11.7 / 13.2    13.3 / 13.8     20.1 / 15.0
//   T = 4096, E = 1024        11.9 / 29.5    20.2 / 32.3    26.0 / 33.2    31.1 / 35.8     52.7 / 41.9
//   T = 16384, E = 512        19.4 / 47.4    36.6 / 55.3    48.0 / 57.7    58.8 / 61.2    103.5 / 67.1
template <int EPL>
constexpr int kBitSelectK = EPL == 1 ? 6 : EPL <= 4 ? 8 : EPL <= 16 ? 9 : 17;
template <int EPL, class Put>
__device__ __forceinline__ void wave_topk(const float (&v)[EPL], int E, int K, Put put) {
  static_assert(EPL >= 1 && EPL <= 64, "the taken mask holds one bit per value of a lane");
  const int lane = lane_id();
  float denom = 0.f;
  bool bits = false;
  if constexpr (kBitSelectK<EPL> <= 16) bits = K >= kBitSelectK<EPL>;
  if (bits) {
    uint32_t key[EPL];
    int rank[EPL];
    uint64_t alive[EPL], sel[EPL];
#pragma unroll
    for (int j = 0; j < EPL; ++j) {
      key[j] = topk_key(v[j]);
      rank[j] = 0;
      alive[j] = __ballot(lane + 64 * j < E);
      sel[j] = 0;
    }
    int na = E, need = K;
    for (int b = 31; b >= 0 && na > need; --b) {
      const uint32_t bit = 1u << b;
      uint64_t one[EPL];
      int c = 0;
#pragma unroll
      for (int j = 0; j < EPL; ++j) {
        one[j] = __ballot((key[j] & bit) != 0) & alive[j];
        c += __popcll(one[j]);
      }
      const bool more = c >= need;
#pragma unroll
      for (int j = 0; j < EPL; ++j) {
        sel[j] |= more ? 0ull : one[j];
        alive[j] = more ? one[j] : alive[j] & ~one[j];
      }
      na = more ? c : na - c;
      need = more ? need : need - c;
    }
    const bool ties = na > need;  // equal keys: the lowest experts
#pragma unroll
    for (int j = 0; j < EPL; ++j) {
      uint64_t a = alive[j];
      if (ties) {
        for (int drop = __popcll(a) - need; drop > 0; --drop) a &= ~(1ull << (63 - __clzll(a)));
        need -= __popcll(a);
      }
      sel[j] |= a;
    }
#pragma unroll
    for (int j = 0; j < EPL; ++j) {
      for (uint64_t m = sel[j]; m; m &= m - 1) {
        const int l = __ffsll((unsigned long long)m) - 1;
        denom += __int_as_float(__builtin_amdgcn_readlane(__float_as_int(v[j]), l));
        const uint32_t k = (uint32_t)__builtin_amdgcn_readlane((int)key[j], l);
        const int e = 64 * j + l;
#pragma unroll
        for (int i = 0; i < EPL; ++i) rank[i] += k > key[i] || (k == key[i] && e < lane + 64 * i);
      }
    }
#pragma unroll
    for (int j = 0; j < EPL; ++j)
      if ((sel[j] >> lane) & 1ull) put(rank[j], lane + 64 * j, topk_value(key[j]) / denom);
  } else {
    uint64_t taken = 0;  // bit j: value j of this lane is selected
    int sel_e[16];
    float sel_v[16];
#pragma unroll
    for (int k = 0; k < 16; ++k) {
      sel_e[k] = 0;
      sel_v[k] = 0.f;
      if (k < K) {
        uint32_t best = 0;
        int bj = -1;  // j of this lane's best candidate (the lowest j on equal keys)
#pragma unroll
        for (int j = 0; j < EPL; ++j) {
          const int e = lane + 64 * j;
          if (e < E && !((taken >> j) & 1ull)) {
            const uint32_t c = topk_key(v[j]);
            if (bj < 0 || c > best) {
              best = c;
              bj = j;
            }
          }
        }
        const uint32_t m = dpp_reduce(bj >= 0 ? best : 0u, [](uint32_t a, uint32_t b) { return a > b ? a : b; });
        int be = 0x7fffffff;
#pragma unroll
        for (int j = 0; j < EPL; ++j) {
          const uint64_t hit = __ballot(bj == j && best == m);
          if (hit && be == 0x7fffffff) be = __ffsll((unsigned long long)hit) - 1 + 64 * j;
        }
        if (be != 0x7fffffff && (be & 63) == lane) taken |= 1ull << (be >> 6);
        sel_e[k] = be;
        sel_v[k] = topk_value(m);
      }
    }
#pragma unroll
    for (int j = 0; j < EPL; ++j) {
      uint64_t sel = __ballot((taken >> j) & 1ull);
      while (sel) {
        const int l = __ffsll((unsigned long long)sel) - 1;
        denom += __int_as_float(__builtin_amdgcn_readlane(__float_as_int(v[j]), l));
        sel &= sel - 1;
      }
    }
#pragma unroll
    for (int k = 0; k < 16; ++k)
      if (k < K && lane == k) put(k, sel_e[k], sel_v[k] / denom);
  }
}

}  // namespace smoe

// C ABI of the MoE layer: host-side validation, routing/workspace layout and
// the launch sequence of each entry point.  No entry point allocates device
// memory or synchronises the stream.
#include <hip/hip_runtime.h>

#include <cstdarg>
#include <cstdio>
#include <initializer_list>
#include <mutex>
#include <string>
#include <vector>

#include "fp8_block.h"
#include "launch.h"

namespace {

thread_local std::string g_last_error;

int fail(int code, const char* fmt, ...) {
  char buf[512];
  va_list ap;
  va_start(ap, fmt);
  vsnprintf(buf, sizeof(buf), fmt, ap);
  va_end(ap);
  g_last_error = buf;
  return code;
}

int hip_fail(hipError_t e, const char* where) {
  return fail(MOE_ERR_HIP, "%s: %s", where, hipGetErrorString(e));
}

constexpr size_t kAlign = 256;
size_t align_up(size_t x) { return (x + kAlign - 1) / kAlign * kAlign; }

bool aligned(const void* p, size_t a) { return (reinterpret_cast<uintptr_t>(p) % a) == 0; }

int check_dims(const moe_dims& m) {
  if (m.T < 1) return fail(MOE_ERR_INVALID_ARG, "T must be >= 1 (got %d)", m.T);
  if (m.d < 128 || m.d % 128) return fail(MOE_ERR_UNSUPPORTED, "d must be a positive multiple of 128 (got %d)", m.d);
  if (m.n < 64 || m.n % 64) return fail(MOE_ERR_UNSUPPORTED, "n must be a positive multiple of 64 (got %d)", m.n);
  if (m.E < 8 || m.E % 8 || m.E > 4096)
    return fail(MOE_ERR_UNSUPPORTED, "E must be a multiple of 8 in [8, 4096] (got %d)", m.E);
  if (m.K < 1 || m.K > 16 || m.K > m.E)
    return fail(MOE_ERR_UNSUPPORTED, "K must be in [1, min(E, 16)] (got K=%d, E=%d)", m.K, m.E);
  if ((int64_t)m.T * m.E > (int64_t)INT32_MAX)
    return fail(MOE_ERR_UNSUPPORTED, "T*E must fit in int32 (got %lld)", (long long)m.T * m.E);
  return MOE_OK;
}

#define CHECK_PTR(p, a)                                                                                   \
  do {                                                                                                    \
    if (!(p)) return fail(MOE_ERR_INVALID_ARG, "%s must not be null", #p);                                \
    if (!aligned((p), (a))) return fail(MOE_ERR_INVALID_ARG, "%s must be %d-byte aligned", #p, (int)(a)); \
  } while (0)

int check_routing(const moe_dims& m, const moe_routing* r, int64_t min_capacity, const char* name) {
  if (!r) return fail(MOE_ERR_INVALID_ARG, "%s must not be null", name);
  if (r->words != (m.T + 63) / 64)
    return fail(MOE_ERR_INVALID_ARG, "%s->words must be ceil(T/64) = %d (got %d)", name, (m.T + 63) / 64, r->words);
  if ((int64_t)r->capacity < min_capacity)
    return fail(MOE_ERR_CAPACITY, "%s->capacity %d < required %lld", name, r->capacity, (long long)min_capacity);
  const void* req[] = {r->scores, r->mask, r->mask_prefix, r->counts, r->offsets, r->row_token, r->row_expert,
                       r->row_w, r->tok_offsets, r->tok_rows, r->tok_count, r->tok_denom, r->round_dir, r->scratch,
                       r->status};
  for (const void* p : req)
    if (!p) return fail(MOE_ERR_INVALID_ARG, "%s has a null array (initialise it with moe_routing_init)", name);
  return MOE_OK;
}

// the consumers of a routing (moe_fwd, moe_bwd) need its complete metadata
int check_built(const moe_routing* r, const char* name) {
  if (r->state != MOE_ROUTING_STATE_BUILT)
    return fail(MOE_ERR_INVALID_ARG,
                "%s is not a complete routing (state %d; moe_route without MOE_ROUTE_COUNTS_ONLY or "
                "moe_round_tokens builds one)",
                name, r->state);
  return MOE_OK;
}

bool valid_m_tile(int m) { return m >= 8 && m <= 256 && (m & (m - 1)) == 0; }

// ---------------------------------------------------------------- static workspace
// The forward workspace of moe_fwd_static: a file-scope device array that
// each GPU holds from the library's load to the end of the process.  In host
// code `scratch` only names the host-side stand-in of the symbol; its device
// address comes from hipGetSymbolAddress, once per device, with that device
// current, and only that address is ever handed to a kernel.
constexpr size_t kStaticWsBytes = (size_t)64 << 20;
static __device__ __align__(256) char scratch[kStaticWsBytes];
constexpr int kMaxDevices = 64;
std::mutex g_scratch_mu;
void* g_scratch_ptr[kMaxDevices] = {};

int static_ws(void** out) {
  int dev = 0;
  hipError_t e = hipGetDevice(&dev);
  if (e != hipSuccess) return hip_fail(e, "hipGetDevice");
  if (dev < 0 || dev >= kMaxDevices) return fail(MOE_ERR_UNSUPPORTED, "device %d beyond %d", dev, kMaxDevices);
  std::lock_guard<std::mutex> lk(g_scratch_mu);
  if (!g_scratch_ptr[dev]) {
    void* p = nullptr;
    e = hipGetSymbolAddress(&p, HIP_SYMBOL(scratch));
    if (e != hipSuccess) return hip_fail(e, "hipGetSymbolAddress(scratch)");
    if (!p) return fail(MOE_ERR_HIP, "hipGetSymbolAddress(scratch) returned null");
    g_scratch_ptr[dev] = p;
  }
  *out = g_scratch_ptr[dev];
  return MOE_OK;
}

// ---------------------------------------------------------------- timing
std::mutex g_prof_mu;
int g_prof_class = -1;
std::vector<std::pair<hipEvent_t, hipEvent_t>> g_prof_events;  // recorded pairs
std::vector<std::pair<hipEvent_t, hipEvent_t>> g_prof_pool;     // free pairs

// ---------------------------------------------------------------- workspaces
struct FwdWs {
  uint16_t* A;
  uint16_t* Y;
  int32_t* mtiles;
};
struct BwdWs {
  int32_t* mtiles;
  uint16_t* dH;
  uint16_t* Ap;
  uint16_t* dXt;
  float* dS;
  float* dS_part;
  uint16_t* dL;
  uint16_t* WrT;
  float* dWr_part;
  float* dbias_part;
  int32_t* klist2;  // k-chunk lists of the weight gradients
  int32_t* klist1;
  float* dw2_part;  // fp32 partials of row-chunked experts
  float* dw1_part;
  uint16_t* b2s;    // expert-bias dS term: b2^T as bf16 high/low parts [d][2E]
  float* bq;        // and <dO_t, b2_e> in those two parts [T][2E]
  float* colsum_part;  // per m-tile column sums of the expert-bias gradients
};

size_t carve(char* base, size_t off, size_t bytes, void** out) {
  if (out) *out = base ? base + off : nullptr;
  return align_up(off + bytes);
}

size_t fwd_layout(const moe_dims& m, int64_t cap, char* base, FwdWs* w) {
  size_t off = 0;
  off = carve(base, off, (size_t)cap * m.n * 2, w ? (void**)&w->A : nullptr);
  off = carve(base, off, (size_t)cap * m.d * 2, w ? (void**)&w->Y : nullptr);
  off = carve(base, off, smoe::mtiles_bytes(cap, m.E), w ? (void**)&w->mtiles : nullptr);
  return off;
}

// the aggregation ablation: the forward workspace, then the token-major slot
// of every row and an fp32 O
size_t abl_layout(const moe_dims& m, int64_t cap, char* base, FwdWs* w, int32_t** dst, float** O32) {
  size_t off = fwd_layout(m, cap, base, w);
  off = carve(base, off, (size_t)cap * 4, (void**)dst);
  off = carve(base, off, (size_t)m.T * m.d * 4, (void**)O32);
  return off;
}

size_t bwd_layout(const moe_dims& m, int64_t cap, char* base, BwdWs* w) {
  // (the narrowest tiles' dS parts: which are taken depends on the device's CUs,
  // which the size must not)
  const int nnt = smoe::dh_max_n_tiles(m.n);
  const int splits = smoe::dwr_splits(m.T, m.d, m.E, false);
  size_t off = 0;
  off = carve(base, off, smoe::mtiles_bytes(cap, m.E), w ? (void**)&w->mtiles : nullptr);
  off = carve(base, off, (size_t)cap * 2 * m.n * 2, w ? (void**)&w->dH : nullptr);
  off = carve(base, off, (size_t)cap * m.n * 2, w ? (void**)&w->Ap : nullptr);
  off = carve(base, off, (size_t)cap * m.d * 2, w ? (void**)&w->dXt : nullptr);
  off = carve(base, off, (size_t)cap * 4, w ? (void**)&w->dS : nullptr);
  off = carve(base, off, nnt > 1 ? (size_t)cap * nnt * 4 : 0, w ? (void**)&w->dS_part : nullptr);
  off = carve(base, off, (size_t)m.T * m.E * 2, w ? (void**)&w->dL : nullptr);
  off = carve(base, off, (size_t)m.E * m.d * 2, w ? (void**)&w->WrT : nullptr);
  off = carve(base, off, (size_t)splits * m.d * m.E * 4, w ? (void**)&w->dWr_part : nullptr);
  off = carve(base, off, (size_t)splits * m.E * 4, w ? (void**)&w->dbias_part : nullptr);
  off = carve(base, off, smoe::kchunks_bytes(m.E), w ? (void**)&w->klist2 : nullptr);
  off = carve(base, off, smoe::kchunks_bytes(m.E), w ? (void**)&w->klist1 : nullptr);
  off = carve(base, off, smoe::dw_part_bytes(m.T, (int64_t)m.n * m.d), w ? (void**)&w->dw2_part : nullptr);
  off = carve(base, off, smoe::dw_part_bytes(m.T, (int64_t)m.d * 2 * m.n), w ? (void**)&w->dw1_part : nullptr);
  off = carve(base, off, (size_t)m.d * 2 * m.E * 2, w ? (void**)&w->b2s : nullptr);
  off = carve(base, off, (size_t)m.T * 2 * m.E * 4, w ? (void**)&w->bq : nullptr);
  off = carve(base, off, smoe::colsum_part_bytes(cap, m.E, m.d, m.n), w ? (void**)&w->colsum_part : nullptr);
  return off;
}

// moe_bwd_ckpt: the backward workspace, then X in bf16 (where the kept one is used)
size_t bwd_ckpt_layout(const moe_dims& m, int64_t cap, char* base, BwdWs* w, uint16_t** X) {
  size_t off = bwd_layout(m, cap, base, w);
  off = carve(base, off, (size_t)m.T * m.d * 2, (void**)X);
  return off;
}

// moe_fwd_quant: X and A in 8-bit blocks (X's in the checkpoint where it is kept), or
// A in fp32 where the streaming projections may run, with or without a rounding
struct QuantWs {
  uint8_t* X8;
  uint8_t* Xs;
  float* A32;
  uint8_t* A8;
  uint8_t* As;
  uint16_t* Y;
  float* Y32;
  int32_t* mtiles256;
  int32_t* mtiles128;
};
size_t quant_layout(const moe_dims& m, int64_t cap, char* base, QuantWs* w) {
  const int np = smoe::q_pad(m.n);
  // (a rounding raises the mean rows of an expert, above 2 at the least: the wider of the
  // two row groups, which may fit a grid where the narrow ones of 2 rows do not)
  const bool streams = smoe::stream8_shape(m, (int)cap, 0).mb || smoe::stream8_shape(m, (int)cap, 3).mb;
  size_t off = 0;
  off = carve(base, off, (size_t)m.T * m.d, w ? (void**)&w->X8 : nullptr);
  off = carve(base, off, (size_t)m.T * smoe::q_stride(m.d / smoe::kQBlock), w ? (void**)&w->Xs : nullptr);
  off = carve(base, off, streams ? (size_t)cap * m.n * 4 : 0, w ? (void**)&w->A32 : nullptr);
  off = carve(base, off, (size_t)cap * np, w ? (void**)&w->A8 : nullptr);
  off = carve(base, off, (size_t)cap * smoe::q_stride(smoe::q_blocks(m.n)), w ? (void**)&w->As : nullptr);
  off = carve(base, off, (size_t)cap * m.d * (streams ? 4 : 2), w ? (void**)&w->Y : nullptr);
  if (w) w->Y32 = (float*)w->Y;
  off = carve(base, off, smoe::mtiles_bytes(cap, m.E, 256), w ? (void**)&w->mtiles256 : nullptr);
  off = carve(base, off, smoe::mtiles_bytes(cap, m.E, 128), w ? (void**)&w->mtiles128 : nullptr);
  return off;
}

// moe_decode and moe_decode_quant: the counters, partial logits, the selection, A (in fp32 for
// the 8-bit one), Y and the slices of H
struct DecodeWs {
  int32_t* sync;
  float* part;
  uint32_t* picked;
  void* A;
  float* Y;
  float* H32;
};
size_t decode_layout(const moe_dims& m, bool q8, char* base, DecodeWs* w) {
  const size_t P = (size_t)m.T * m.K;
  size_t off = 0;
  off = carve(base, off, smoe::decode_sync_words(m.T, m.d, m.E, m.K) * 4, w ? (void**)&w->sync : nullptr);
  off = carve(base, off, (size_t)smoe::decode_slices(m.T, m.d, m.E) * m.T * m.E * 4, w ? (void**)&w->part : nullptr);
  off = carve(base, off, P * 8, w ? (void**)&w->picked : nullptr);
  off = carve(base, off, P * m.n * (q8 ? 4 : 2), w ? &w->A : nullptr);
  off = carve(base, off, P * m.d * 4, w ? (void**)&w->Y : nullptr);
  const int ks = smoe::decode_ks(m.T, m.d, m.n, m.E, m.K, q8);
  off = carve(base, off, ks > 1 ? ks * P * m.n * 8 : 0, w ? (void**)&w->H32 : nullptr);
  return off;
}

int check_decode(const moe_dims& m) {
  int rc = check_dims(m);
  if (rc) return rc;
  if (m.T > smoe::kDecodeTokens)
    return fail(MOE_ERR_UNSUPPORTED, "T must be at most %d (got %d): moe_route and moe_fwd take more", smoe::kDecodeTokens, m.T);
  if (m.E > smoe::kDecodeExperts) return fail(MOE_ERR_UNSUPPORTED, "E must be at most %d (got %d)", smoe::kDecodeExperts, m.E);
  // (32-bit byte offsets within an expert's weights, W_r and the rows)
  const int64_t most = INT32_MAX;
  if (4 * (int64_t)m.d * m.n > most || 2 * (int64_t)m.d * m.E > most || 2 * (int64_t)m.T * m.d > most || 8 * (int64_t)m.T * m.K * m.n > most || 4 * (int64_t)m.T * m.K * m.d > most)
    return fail(MOE_ERR_UNSUPPORTED, "d = %d, n = %d: an expert's projection, W_r and the rows must be below 2^31 bytes each", m.d, m.n);
  return MOE_OK;
}

size_t qexperts_layout(const moe_dims& m, char* base, moe_qexperts* q) {
  size_t off = 0;
  off = carve(base, off, m.E * smoe::w1q_bytes(m.d, m.n), q ? (void**)&q->W1 : nullptr);
  off = carve(base, off, m.E * smoe::w1s_bytes(m.d, m.n), q ? (void**)&q->W1s : nullptr);
  off = carve(base, off, m.E * smoe::w2q_bytes(m.d, m.n), q ? (void**)&q->W2 : nullptr);
  off = carve(base, off, m.E * smoe::w2s_bytes(m.d, m.n), q ? (void**)&q->W2s : nullptr);
  return off;
}

size_t ckpt_layout(const moe_dims& m, int64_t cap, int flags, char* base, moe_ckpt* c) {
  const bool x = flags & MOE_CKPT_X;
  size_t off = 0;
  off = carve(base, off, (size_t)cap * 2 * m.n, c ? (void**)&c->H : nullptr);
  off = carve(base, off, (size_t)cap * smoe::h8_stride(m.n), c ? (void**)&c->Hs : nullptr);
  off = carve(base, off, x ? (size_t)m.T * m.d : 0, c ? (void**)&c->X : nullptr);
  off = carve(base, off, x ? (size_t)m.T * smoe::q_stride(m.d / smoe::kQBlock) : 0, c ? (void**)&c->Xs : nullptr);
  if (c && !x) c->X = c->Xs = nullptr;
  return off;
}

int check_qexperts(const moe_dims& m, const moe_qexperts* q, bool written) {
  if (!q) return fail(MOE_ERR_INVALID_ARG, "the 8-bit weights must not be null");
  if (!q->W1 || !q->W1s || !q->W2 || !q->W2s)
    return fail(MOE_ERR_INVALID_ARG, "the 8-bit weights have a null array (initialise them with moe_qexperts_init)");
  if (q->d != m.d || q->n != m.n || q->E != m.E)
    return fail(MOE_ERR_INVALID_ARG, "the 8-bit weights are of d = %d, n = %d, E = %d, not of the call's %d, %d, %d", q->d,
                q->n, q->E, m.d, m.n, m.E);
  if (written && q->state != MOE_HELD_WRITTEN)
    return fail(MOE_ERR_INVALID_ARG, "the 8-bit weights are not written (moe_quantize_experts does it)");
  return MOE_OK;
}

int check_ckpt(const moe_dims& m, const moe_routing* r, const moe_ckpt* c, bool written) {
  if (!c) return fail(MOE_ERR_INVALID_ARG, "the checkpoint must not be null");
  if (!c->H || !c->Hs || !c->X != !c->Xs)
    return fail(MOE_ERR_INVALID_ARG, "the checkpoint has a null array (initialise it with moe_ckpt_init)");
  if (c->T != m.T || c->d != m.d || c->n != m.n || c->capacity != r->capacity)
    return fail(MOE_ERR_INVALID_ARG,
                "the checkpoint is of T = %d, d = %d, n = %d, capacity %d, not of the call's %d, %d, %d, %d", c->T, c->d,
                c->n, c->capacity, m.T, m.d, m.n, r->capacity);
  if (written && c->state != MOE_HELD_WRITTEN)
    return fail(MOE_ERR_INVALID_ARG, "the checkpoint is not written (moe_fwd_ckpt or moe_fwd_quant does it)");
  return MOE_OK;
}

// byte offset of the rounding selection's lists in the routing scratch
size_t round_lists_offset(const moe_dims& m) {
  const int W = (m.T + 63) / 64;
  return ((size_t)(m.E + 64 + 2 * (W + 1)) * 4 + 255) / 256 * 256;
}

size_t routing_layout(const moe_dims& m, int64_t cap, int flags, char* base, moe_routing* r) {
  const int W = (m.T + 63) / 64;
  const size_t TE = (size_t)m.T * m.E, EW = (size_t)m.E * W, TK = (size_t)m.T * m.K;
  moe_routing tmp;
  moe_routing* o = r ? r : &tmp;
  size_t off = 0;
  auto take = [&](size_t bytes, void** p) { off = carve(base, off, bytes, p); };
  void* p;
  take((flags & MOE_ROUTING_LOGITS) ? TE * 4 : 0, &p);
  o->logits = (flags & MOE_ROUTING_LOGITS) ? (float*)p : nullptr;
  take(TE * 4, &p);
  o->scores = (float*)p;
  take((flags & MOE_ROUTING_SCORES_T) ? TE * 4 : 0, &p);
  o->scores_t = (flags & MOE_ROUTING_SCORES_T) ? (float*)p : nullptr;
  take(TK * 4, &p);
  o->topk_idx = (int32_t*)p;
  take(TK * 4, &p);
  o->topk_w = (float*)p;
  take(EW * 8, &p);
  o->mask = (uint64_t*)p;
  take(EW * 4, &p);
  o->mask_prefix = (int32_t*)p;
  take((size_t)m.E * 4, &p);
  o->counts = (int32_t*)p;
  take((size_t)(m.E + 1) * 4, &p);
  o->offsets = (int32_t*)p;
  take((size_t)cap * 4, &p);
  o->row_token = (int32_t*)p;
  take((size_t)cap * 4, &p);
  o->row_expert = (int32_t*)p;
  take((size_t)cap * 4, &p);
  o->row_w = (float*)p;
  take((size_t)(m.T + 1) * 4, &p);
  o->tok_offsets = (int32_t*)p;
  take((size_t)cap * 4, &p);
  o->tok_rows = (int32_t*)p;
  take((size_t)m.T * 4, &p);
  o->tok_count = (int32_t*)p;
  take((size_t)m.T * 4, &p);
  o->tok_denom = (float*)p;
  take((size_t)m.E * 4, &p);
  o->round_dir = (int32_t*)p;
  // rounding needs [E], then per-word token sums and bases, then the
  // selection's lists
  take(round_lists_offset(m) + smoe::round_scratch_bytes(m.T, m.E), &p);
  o->scratch = (int32_t*)p;
  take(4, &p);
  o->status = (int32_t*)p;
  o->capacity = (int32_t)cap;
  o->words = W;
  o->state = MOE_ROUTING_STATE_EMPTY;
  o->reserved = 0;
  return off;
}

// the projections, streaming (few rows per expert) or tiled
struct Projections {
  smoe::StreamShape up, down;  // mb = 0: tiled
  Projections(const moe_dims& m, const moe_routing& r)
      : up(smoe::stream_shape(m, r.capacity, smoe::rounding_tile(r), (2 * m.n + 255) / 256)),
        down(smoe::stream_shape(m, r.capacity, smoe::rounding_tile(r), (m.d + 255) / 256)) {}
  hipError_t lists(const int32_t* offsets, int E, int32_t* mtiles, hipStream_t s) const {
    return up.mb && down.mb ? hipSuccess : smoe::launch_mtiles(offsets, E, mtiles, s);
  }
  hipError_t run_up(const smoe::UpArgs& a, hipStream_t s) const {
    return up.mb ? smoe::launch_stream_up(a, up, s) : smoe::launch_up(a, s);
  }
  hipError_t run_down(const smoe::DownArgs& a, int strategy, hipStream_t s) const {
    return down.mb ? smoe::launch_stream_down(a, strategy, down, s) : smoe::launch_down_ablation(a, strategy, s);
  }
};

#define HIP_TRY(expr, where)                          \
  do {                                                \
    hipError_t _e = (expr);                           \
    if (_e != hipSuccess) return hip_fail(_e, where); \
  } while (0)

#define LAUNCH(kc, expr, where)          \
  do {                                   \
    smoe::prof_begin((kc), stream);      \
    hipError_t _e = (expr);              \
    smoe::prof_end((kc), stream);        \
    if (_e != hipSuccess) return hip_fail(_e, where); \
  } while (0)

}  // namespace

namespace smoe {

void prof_begin(int kc, hipStream_t s) {
  std::lock_guard<std::mutex> lk(g_prof_mu);
  if (kc != g_prof_class) return;
  std::pair<hipEvent_t, hipEvent_t> ev;
  if (!g_prof_pool.empty()) {
    ev = g_prof_pool.back();
    g_prof_pool.pop_back();
  } else {
    if (hipEventCreate(&ev.first) != hipSuccess || hipEventCreate(&ev.second) != hipSuccess) return;
  }
  (void)hipEventRecord(ev.first, s);
  g_prof_events.push_back(ev);
}

void prof_end(int kc, hipStream_t s) {
  std::lock_guard<std::mutex> lk(g_prof_mu);
  if (kc != g_prof_class || g_prof_events.empty()) return;
  (void)hipEventRecord(g_prof_events.back().second, s);
}

}  // namespace smoe

extern "C" {

const char* moe_strerror(int code) {
  switch (code) {
    case MOE_OK: return "success";
    case MOE_ERR_INVALID_ARG: return "invalid argument";
    case MOE_ERR_UNSUPPORTED: return "unsupported shape";
    case MOE_ERR_CAPACITY: return "routing capacity too small";
    case MOE_ERR_WORKSPACE: return "workspace too small";
    case MOE_ERR_HIP: return "HIP runtime error";
    default: return "unknown error";
  }
}

const char* moe_last_error(void) { return g_last_error.c_str(); }

size_t moe_routing_bytes(moe_dims dims, int32_t capacity, int flags) {
  if (check_dims(dims) != MOE_OK || capacity < 0) return 0;
  return routing_layout(dims, capacity, flags, nullptr, nullptr);
}

int moe_routing_init(moe_dims dims, int32_t capacity, int flags, void* buf, size_t bytes, moe_routing* r) {
  int rc = check_dims(dims);
  if (rc) return rc;
  if (!r) return fail(MOE_ERR_INVALID_ARG, "r must not be null");
  CHECK_PTR(buf, kAlign);
  if (capacity < dims.T * dims.K)
    return fail(MOE_ERR_CAPACITY, "capacity %d < T*K = %d", capacity, dims.T * dims.K);
  const size_t need = routing_layout(dims, capacity, flags, nullptr, nullptr);
  if (bytes < need) return fail(MOE_ERR_INVALID_ARG, "routing buffer of %zu bytes < required %zu", bytes, need);
  routing_layout(dims, capacity, flags, (char*)buf, r);
  return MOE_OK;
}

int32_t moe_round_capacity(moe_dims dims, int32_t m_tile) {
  if (check_dims(dims) != MOE_OK || !valid_m_tile(m_tile)) return -1;
  const int64_t a = (int64_t)dims.T * dims.E;
  const int64_t b = (int64_t)dims.T * dims.K + (int64_t)dims.E * (m_tile - 1);
  const int64_t c = a < b ? a : b;
  return c > INT32_MAX ? -1 : (int32_t)c;
}

size_t moe_workspace_bytes(moe_dims dims, int32_t capacity, int which) {
  if (check_dims(dims) != MOE_OK || capacity < 0) return 0;
  if (which == MOE_WS_FWD) return fwd_layout(dims, capacity, nullptr, nullptr);
  if (which == MOE_WS_BWD) return bwd_layout(dims, capacity, nullptr, nullptr);
  if (which == MOE_WS_FWD_AGG_ABLATION) {
    int32_t* dst;
    float* o32;
    return abl_layout(dims, capacity, nullptr, nullptr, &dst, &o32);
  }
  if (which == MOE_WS_FWD_QUANT) return quant_layout(dims, capacity, nullptr, nullptr);
  if (which == MOE_WS_FWD_CKPT) return fwd_layout(dims, capacity, nullptr, nullptr);
  if (which == MOE_WS_BWD_CKPT) return bwd_ckpt_layout(dims, capacity, nullptr, nullptr, nullptr);
  if (which == MOE_WS_DECODE) return check_decode(dims) == MOE_OK ? decode_layout(dims, false, nullptr, nullptr) : 0;
  if (which == MOE_WS_DECODE_QUANT) return check_decode(dims) == MOE_OK ? decode_layout(dims, true, nullptr, nullptr) : 0;
  return 0;
}

int moe_route(moe_dims m, const moe_bf16* X, const moe_bf16* Wr, const float* bias, int flags, moe_routing* r,
              void* stream_) {
  int rc = check_dims(m);
  if (rc) return rc;
  rc = check_routing(m, r, (int64_t)m.T * m.K, "r");
  if (rc) return rc;
  if (!r->topk_idx || !r->topk_w) return fail(MOE_ERR_INVALID_ARG, "r->topk_idx and r->topk_w must not be null");
  const bool scores_in = flags & MOE_ROUTE_SCORES_IN;
  if (!scores_in) {
    CHECK_PTR(X, 16);
    CHECK_PTR(Wr, 16);
  }
  if (bias && !aligned(bias, 4)) return fail(MOE_ERR_INVALID_ARG, "bias must be 4-byte aligned");
  if ((flags & MOE_ROUTE_WRITE_LOGITS) && !r->logits)
    return fail(MOE_ERR_INVALID_ARG, "MOE_ROUTE_WRITE_LOGITS needs r->logits");
  if ((flags & MOE_ROUTE_WRITE_SCORES_T) && !r->scores_t)
    return fail(MOE_ERR_INVALID_ARG, "MOE_ROUTE_WRITE_SCORES_T needs r->scores_t");
  if (flags & ~(MOE_ROUTE_SCORES_IN | MOE_ROUTE_WRITE_LOGITS | MOE_ROUTE_WRITE_SCORES_T | MOE_ROUTE_COUNTS_ONLY |
                MOE_ROUTE_SEPARATE_TOPK))
    return fail(MOE_ERR_INVALID_ARG, "unknown flags 0x%x", flags);
  hipStream_t stream = (hipStream_t)stream_;
  float* scores_t = (flags & MOE_ROUTE_WRITE_SCORES_T) ? r->scores_t : nullptr;
  const float* in = r->scores;
  const bool counts_only = (flags & MOE_ROUTE_COUNTS_ONLY) != 0;
  r->state = MOE_ROUTING_STATE_EMPTY;  // until the metadata launch is enqueued
  r->reserved = 0;
  const bool fused = !scores_in && !(flags & MOE_ROUTE_SEPARATE_TOPK) && smoe::router_topk_fusable(m.E, m.K);
  if (smoe::route_few(m, counts_only, scores_in, fused)) {
    // few tokens: partial logits of the router's k slices in the routing's
    // scratch (one slice: in r->scores, which the softmax then overwrites)
    float* logits = !scores_in && (flags & MOE_ROUTE_WRITE_LOGITS) ? r->logits : nullptr;
    const int slices = scores_in ? 1 : smoe::router_slices(m.T, m.d, m.E, smoe::round_scratch_bytes(m.T, m.E));
    float* part = slices > 1 ? (float*)((char*)r->scratch + round_lists_offset(m)) : r->scores;
    auto gemm = [&]() { return smoe::launch_router_part(X, Wr, part, slices, m.T, m.d, m.E, stream); };
    auto topk = [&]() {
      return smoe::launch_topk_few(part, slices, scores_in ? nullptr : bias, logits, scores_t, *r, m.T, m.E, m.K,
                                   scores_in ? 0 : 1, counts_only, stream);
    };
    if (fused) {
      LAUNCH(MOE_KC_ROUTER_TOPK,
             [&]() {
               const hipError_t e = gemm();
               return e == hipSuccess ? topk() : e;
             }(),
             "router gemm with softmax/top-K");
    } else {
      if (!scores_in) LAUNCH(MOE_KC_ROUTER_GEMM, gemm(), "router gemm");
      LAUNCH(MOE_KC_TOPK, topk(), "softmax/top-K");
    }
    if (m.T > smoe::kFewOneGroup)
      LAUNCH(MOE_KC_META, smoe::launch_tc_metadata_few(*r, m.T, m.E, m.K, counts_only, stream), "routing metadata");
    r->state = counts_only ? MOE_ROUTING_STATE_COUNTS : MOE_ROUTING_STATE_BUILT;
    return MOE_OK;
  }
  if (fused) {
    float* logits = (flags & MOE_ROUTE_WRITE_LOGITS) ? r->logits : nullptr;
    smoe::RouterTopkArgs a{X, Wr, bias, logits, r->scores, scores_t, r->topk_idx, r->topk_w, r->mask,
                           m.T, m.d, m.E, m.K, r->words};
    LAUNCH(MOE_KC_ROUTER_TOPK, smoe::launch_router_topk(a, stream), "router gemm with softmax/top-K");
  } else {
    if (!scores_in) {
      float* logits = (flags & MOE_ROUTE_WRITE_LOGITS) ? r->logits : r->scores;
      smoe::RouterGemmArgs a{X, Wr, bias, logits, m.T, m.d, m.E};
      LAUNCH(MOE_KC_ROUTER_GEMM, smoe::launch_router_gemm(a, stream), "router gemm");
      in = logits;
    }
    LAUNCH(MOE_KC_TOPK,
           smoe::launch_topk_route(in, r->scores, scores_t, r->topk_idx, r->topk_w, r->mask, m.T, m.E, m.K,
                                   r->words, scores_in ? 0 : 1, stream),
           "softmax/top-K");
  }
  LAUNCH(MOE_KC_META, smoe::launch_tc_metadata(*r, m.T, m.E, m.K, counts_only, stream), "routing metadata");
  r->state = counts_only ? MOE_ROUTING_STATE_COUNTS : MOE_ROUTING_STATE_BUILT;
  return MOE_OK;
}

int moe_round_tokens(moe_dims m, int32_t m_tile, int mode, const float* u, const moe_routing* tc, moe_routing* tr,
                     void* stream_) {
  int rc = check_dims(m);
  if (rc) return rc;
  if (!valid_m_tile(m_tile))
    return fail(MOE_ERR_INVALID_ARG, "m_tile must be a power of two in [8, 256] (got %d)", m_tile);
  if (mode < MOE_ROUND_NEAREST || mode > MOE_ROUND_STOCHASTIC)
    return fail(MOE_ERR_INVALID_ARG, "unknown rounding mode %d", mode);
  if (mode == MOE_ROUND_STOCHASTIC) CHECK_PTR(u, 4);
  rc = check_routing(m, tc, (int64_t)m.T * m.K, "tc");
  if (rc) return rc;
  if (!tc->scores_t) return fail(MOE_ERR_INVALID_ARG, "tc->scores_t must be written (MOE_ROUTE_WRITE_SCORES_T)");
  if (tc->state < MOE_ROUTING_STATE_COUNTS)
    return fail(MOE_ERR_INVALID_ARG, "tc has no counts yet (state %d): run moe_route on it first", tc->state);
  rc = check_routing(m, tr, moe_round_capacity(m, m_tile), "tr");
  if (rc) return rc;
  if (tr == tc || tr->mask == tc->mask) return fail(MOE_ERR_INVALID_ARG, "tr must not alias tc");
  hipStream_t stream = (hipStream_t)stream_;
  tr->state = MOE_ROUTING_STATE_EMPTY;
  tr->reserved = smoe::rounding_word(m_tile, mode);
  smoe::prof_begin(MOE_KC_ROUND, stream);
  bool counted = false;
  uint64_t* list = (uint64_t*)((char*)tr->scratch + round_lists_offset(m));
  hipError_t e = smoe::launch_round(*tc, *tr, u, m.T, m.E, m_tile, mode, list, &counted, stream);
  if (e == hipSuccess) e = smoe::launch_metadata(*tr, tc->scores_t, m.T, m.E, counted, stream);
  smoe::prof_end(MOE_KC_ROUND, stream);
  if (e != hipSuccess) return hip_fail(e, "token rounding");
  tr->state = MOE_ROUTING_STATE_BUILT;
  return MOE_OK;
}

int check_expert_bias(const moe_expert_bias* eb) {
  if (!eb) return MOE_OK;
  const void* p[] = {eb->b1, eb->b2, eb->db1, eb->db2};
  const char* name[] = {"eb->b1", "eb->b2", "eb->db1", "eb->db2"};
  for (int i = 0; i < 4; ++i)
    if (p[i] && !aligned(p[i], 16)) return fail(MOE_ERR_INVALID_ARG, "%s must be 16-byte aligned", name[i]);
  return MOE_OK;
}

int moe_fwd(moe_dims m, const moe_bf16* X, const moe_bf16* W1, const moe_bf16* W2, const moe_expert_bias* eb,
            const moe_routing* r, moe_bf16* H, moe_bf16* O, void* ws, size_t ws_bytes, void* stream_) {
  int rc = check_dims(m);
  if (rc) return rc;
  rc = check_routing(m, r, 1, "r");
  if (rc) return rc;
  rc = check_built(r, "r");
  if (rc) return rc;
  CHECK_PTR(X, 16);
  CHECK_PTR(W1, 16);
  CHECK_PTR(W2, 16);
  CHECK_PTR(H, 16);
  CHECK_PTR(O, 16);
  rc = check_expert_bias(eb);
  if (rc) return rc;
  const float* b1 = eb ? eb->b1 : nullptr;
  const float* b2 = eb ? eb->b2 : nullptr;
  const size_t need = fwd_layout(m, r->capacity, nullptr, nullptr);
  if (ws_bytes < need) return fail(MOE_ERR_WORKSPACE, "forward workspace %zu < required %zu", ws_bytes, need);
  CHECK_PTR(ws, kAlign);
  FwdWs w;
  fwd_layout(m, r->capacity, (char*)ws, &w);
  hipStream_t stream = (hipStream_t)stream_;
  const int64_t mt = smoe::expected_mtiles(m, *r);
  const smoe::UpArgs up{X, W1, r->offsets, r->row_token, H, w.A, m.d, m.n, m.E, r->capacity, mt, w.mtiles, b1};
  const smoe::DownArgs down{w.A, W2, r->offsets, w.Y, m.d, m.n, m.E, r->capacity, mt, w.mtiles, b2};
  const Projections proj(m, *r);
  HIP_TRY(proj.lists(r->offsets, m.E, w.mtiles, stream), "m-tile list");
  LAUNCH(MOE_KC_UP, proj.run_up(up, stream), "up-proj");
  LAUNCH(MOE_KC_DOWN, proj.run_down(down, MOE_AGG_GATHER_SUM, stream), "down-proj");
  LAUNCH(MOE_KC_AGG_O, smoe::launch_agg_o(w.Y, *r, O, m.T, m.d, stream), "aggregation");
  return MOE_OK;
}

size_t moe_fwd_static_max_bytes(void) { return kStaticWsBytes; }

int moe_fwd_static(moe_dims m, const moe_bf16* X, const moe_bf16* W1, const moe_bf16* W2, const moe_expert_bias* eb,
                   const moe_routing* r, moe_bf16* H, moe_bf16* O, void* stream) {
  int rc = check_dims(m);
  if (rc) return rc;
  rc = check_routing(m, r, 1, "r");
  if (rc) return rc;
  const size_t need = fwd_layout(m, r->capacity, nullptr, nullptr);
  if (need > kStaticWsBytes)
    return fail(MOE_ERR_WORKSPACE,
                "the forward workspace for capacity %d (%zu bytes) exceeds the static workspace of %zu bytes; "
                "use moe_fwd with a caller workspace",
                r->capacity, need, kStaticWsBytes);
  void* ws = nullptr;
  rc = static_ws(&ws);
  if (rc) return rc;
  return moe_fwd(m, X, W1, W2, eb, r, H, O, ws, kStaticWsBytes, stream);
}

int moe_fwd_aggregation_ablation(moe_dims m, const moe_bf16* X, const moe_bf16* W1, const moe_bf16* W2,
                                 const moe_routing* r, moe_bf16* H, moe_bf16* O, int strategy, void* ws,
                                 size_t ws_bytes, void* stream_) {
  int rc = check_dims(m);
  if (rc) return rc;
  rc = check_routing(m, r, 1, "r");
  if (rc) return rc;
  rc = check_built(r, "r");
  if (rc) return rc;
  CHECK_PTR(X, 16);
  CHECK_PTR(W1, 16);
  CHECK_PTR(W2, 16);
  CHECK_PTR(H, 16);
  CHECK_PTR(O, 16);
  if (strategy < MOE_AGG_GATHER_SUM || strategy > MOE_AGG_ATOMIC_F32)
    return fail(MOE_ERR_INVALID_ARG, "unknown aggregation strategy %d", strategy);
  int32_t* dst = nullptr;
  float* o32 = nullptr;
  const size_t need = abl_layout(m, r->capacity, nullptr, nullptr, &dst, &o32);
  if (ws_bytes < need) return fail(MOE_ERR_WORKSPACE, "ablation workspace %zu < required %zu", ws_bytes, need);
  CHECK_PTR(ws, kAlign);
  FwdWs w;
  abl_layout(m, r->capacity, (char*)ws, &w, &dst, &o32);
  hipStream_t stream = (hipStream_t)stream_;
  const int64_t mt = smoe::expected_mtiles(m, *r);
  const Projections proj(m, *r);
  HIP_TRY(proj.lists(r->offsets, m.E, w.mtiles, stream), "m-tile list");
  LAUNCH(MOE_KC_UP,
         proj.run_up({X, W1, r->offsets, r->row_token, H, w.A, m.d, m.n, m.E, r->capacity, mt, w.mtiles, nullptr}, stream),
         "up-proj");
  smoe::DownArgs da{w.A, W2, r->offsets, w.Y, m.d, m.n, m.E, r->capacity, mt, w.mtiles, nullptr};
  if (strategy == MOE_AGG_GATHER_SUM) {
    LAUNCH(MOE_KC_DOWN, proj.run_down(da, strategy, stream), "down-proj");
    LAUNCH(MOE_KC_AGG_O, smoe::launch_agg_o(w.Y, *r, O, m.T, m.d, stream), "aggregation");
  } else if (strategy == MOE_AGG_SCATTER_SUM) {
    da.dst = dst;
    LAUNCH(MOE_KC_DOWN,
           [&]() {
             hipError_t e = smoe::launch_tok_slots(*r, m.T, r->capacity, dst, stream);
             return e == hipSuccess ? proj.run_down(da, strategy, stream) : e;
           }(),
           "down-proj (scatter)");
    LAUNCH(MOE_KC_AGG_O, smoe::launch_agg_o_contig(w.Y, *r, O, m.T, m.d, stream), "contiguous sum");
  } else {
    da.O32 = o32;
    da.row_token = r->row_token;
    da.row_w = r->row_w;
    const size_t td = (size_t)m.T * m.d;
    LAUNCH(MOE_KC_DOWN,
           [&]() {
             hipError_t e = smoe::launch_fill_f32(o32, td, stream);
             return e == hipSuccess ? proj.run_down(da, strategy, stream) : e;
           }(),
           "down-proj (fp32 atomics)");
    LAUNCH(MOE_KC_AGG_O, smoe::launch_f32_to_bf16(o32, O, td, stream), "fp32 -> bf16");
  }
  return MOE_OK;
}

// moe_bwd and moe_bwd_ckpt: with ck, its H in the place of H, and its X where X is null
static int backward(moe_dims m, const moe_bf16* dO, const moe_bf16* X, const moe_bf16* H, const moe_ckpt* ck,
                    const moe_bf16* W1, const moe_bf16* W2, const moe_expert_bias* eb, const moe_bf16* Wr,
                    const moe_routing* r, moe_bf16* dX, moe_bf16* dW1, moe_bf16* dW2, float* dWr, float* dbias, float* dS,
                    void* ws, size_t ws_bytes, void* stream_) {
  int rc = check_dims(m);
  if (rc) return rc;
  rc = check_routing(m, r, 1, "r");
  if (rc) return rc;
  rc = check_built(r, "r");
  if (rc) return rc;
  CHECK_PTR(dO, 16);
  if (ck) {
    rc = check_ckpt(m, r, ck, true);
    if (rc) return rc;
    if (!X && !ck->X) return fail(MOE_ERR_INVALID_ARG, "X must not be null: the checkpoint does not keep it (MOE_CKPT_X)");
    if (!aligned(X, 16)) return fail(MOE_ERR_INVALID_ARG, "X must be 16-byte aligned");
  } else {
    CHECK_PTR(X, 16);
    CHECK_PTR(H, 16);
  }
  CHECK_PTR(W1, 16);
  CHECK_PTR(W2, 16);
  CHECK_PTR(dX, 16);
  CHECK_PTR(dW1, 16);
  CHECK_PTR(dW2, 16);
  if (Wr && !aligned(Wr, 16)) return fail(MOE_ERR_INVALID_ARG, "Wr must be 16-byte aligned");
  if (!Wr && (dWr || dbias)) return fail(MOE_ERR_INVALID_ARG, "dWr/dbias need Wr");
  if (dWr && !aligned(dWr, 16)) return fail(MOE_ERR_INVALID_ARG, "dWr must be 16-byte aligned");
  if (dbias && !aligned(dbias, 4)) return fail(MOE_ERR_INVALID_ARG, "dbias must be 4-byte aligned");
  if (dS && !aligned(dS, 4)) return fail(MOE_ERR_INVALID_ARG, "dS must be 4-byte aligned");
  rc = check_expert_bias(eb);
  if (rc) return rc;
  const float* b2 = eb ? eb->b2 : nullptr;
  uint16_t* x16 = nullptr;
  const size_t need = ck ? bwd_ckpt_layout(m, r->capacity, nullptr, nullptr, nullptr) : bwd_layout(m, r->capacity, nullptr, nullptr);
  if (ws_bytes < need) return fail(MOE_ERR_WORKSPACE, "backward workspace %zu < required %zu", ws_bytes, need);
  CHECK_PTR(ws, kAlign);
  BwdWs w;
  if (ck)
    bwd_ckpt_layout(m, r->capacity, (char*)ws, &w, &x16);
  else
    bwd_layout(m, r->capacity, (char*)ws, &w);
  hipStream_t stream = (hipStream_t)stream_;
  smoe::KeptX kept{nullptr, nullptr, nullptr, 0};
  if (!X) {
    kept = smoe::KeptX{ck->X, ck->Xs, x16, m.T * (m.d / smoe::kQBlock)};
    X = x16;
  }
  float* dS_out = dS ? dS : w.dS;
  const int64_t rows = (int64_t)m.T * m.K, mt = smoe::expected_mtiles(m, *r);
  const int nnt = smoe::dh_n_tiles(m.n, mt);
  HIP_TRY(smoe::launch_bwd_lists(r->offsets, m.T, rows, m.E, m.d, m.n, w.mtiles, w.klist2, w.klist1, Wr, Wr ? w.WrT : nullptr,
                                 kept, stream),
          "tile lists, W_r transpose and the kept X");
  if (b2) {
    // <dO_t, b2_e> for every (t, e): dO times b2^T split into bf16 high and low parts
    HIP_TRY(smoe::launch_bias_split(b2, m.E, m.d, w.b2s, stream), "expert-bias split");
    HIP_TRY(smoe::launch_router_gemm({dO, w.b2s, nullptr, w.bq, m.T, m.d, 2 * m.E}, stream), "expert-bias dS term");
  }
  LAUNCH(MOE_KC_DH,
         smoe::launch_dh({dO, W2, H, r->offsets, r->row_token, r->row_w, w.dH, w.Ap, dS_out, w.dS_part, m.d, m.n, m.E,
                          r->capacity, mt, w.mtiles, b2 ? w.bq : nullptr, ck ? ck->H : nullptr, ck ? ck->Hs : nullptr},
                         stream),
         "dH");
  // dS in parts (one per N tile of dH): a few are summed where they are read,
  // unless the caller wants dS itself
  const bool ds_in_parts = nnt > 1 && nnt <= 4 && !dS;
  if (nnt > 1 && !ds_in_parts)
    HIP_TRY(smoe::launch_reduce_rowparts(w.dS_part, dS_out, r->capacity, nnt, stream), "dS reduce");
  LAUNCH(MOE_KC_DW2, smoe::launch_dw2({w.Ap, dO, r->offsets, r->row_token, dW2, m.T, rows, m.d, m.n, m.E, w.klist2, w.dw2_part}, stream), "dW2");
  LAUNCH(MOE_KC_DXT, smoe::launch_dxt({w.dH, W1, r->offsets, w.dXt, m.d, m.n, m.E, r->capacity, mt, w.mtiles}, stream),
         "dX~");
  LAUNCH(MOE_KC_DW1, smoe::launch_dw1({X, w.dH, r->offsets, r->row_token, dW1, m.T, rows, m.d, m.n, m.E, w.klist1, w.dw1_part}, stream), "dW1");
  LAUNCH(MOE_KC_AGG_DX,
         smoe::launch_agg_dx(w.dXt, ds_in_parts ? w.dS_part : dS_out, ds_in_parts ? nnt : 1, Wr ? w.WrT : nullptr, *r, dX, Wr ? w.dL : nullptr, m.T, m.d, m.E, stream),
         "dX aggregation");
  const int splits = smoe::dwr_splits(m.T, m.d, m.E, dbias != nullptr);
  if (dWr || dbias)
    LAUNCH(MOE_KC_DWR,
           smoe::launch_dwr({X, w.dL, dWr ? w.dWr_part : nullptr, dbias ? w.dbias_part : nullptr, m.T, m.d, m.E, splits},
                            stream),
           "dW_r and dbias");
  HIP_TRY(smoe::launch_bwd_final_reduce({w.klist2, w.dw2_part, dW2, w.klist1, w.dw1_part, dW1, w.dWr_part, dWr,
                                         w.dbias_part, dbias, m.T, m.d, m.n, m.E, splits},
                                        stream),
          "final reductions (split experts' weight gradients, dW_r, dbias)");
  if (eb && (eb->db1 || eb->db2))
    HIP_TRY(smoe::launch_expert_colsum({w.dH, dO, r->offsets, r->row_token, r->row_w, w.mtiles, w.colsum_part, eb->db1,
                                        eb->db2, m.d, m.n, m.E, r->capacity},
                                       stream),
            "expert-bias gradients db1, db2");
  return MOE_OK;
}

int moe_bwd(moe_dims m, const moe_bf16* dO, const moe_bf16* X, const moe_bf16* H, const moe_bf16* W1, const moe_bf16* W2,
            const moe_expert_bias* eb, const moe_bf16* Wr, const moe_routing* r, moe_bf16* dX, moe_bf16* dW1,
            moe_bf16* dW2, float* dWr, float* dbias, float* dS, void* ws, size_t ws_bytes, void* stream) {
  return backward(m, dO, X, H, nullptr, W1, W2, eb, Wr, r, dX, dW1, dW2, dWr, dbias, dS, ws, ws_bytes, stream);
}

int32_t moe_scale_stride(int32_t cols) { return cols < 1 ? 0 : smoe::q_stride((cols - 1) / smoe::kQBlock + 1); }

static int check_rows(int64_t rows, int32_t cols) {
  if (rows < 0) return fail(MOE_ERR_INVALID_ARG, "rows must be >= 0 (got %lld)", (long long)rows);
  if (cols < 8 || cols % 8) return fail(MOE_ERR_UNSUPPORTED, "cols must be a positive multiple of 8 (got %d)", cols);
  if (rows > INT32_MAX || rows * ((cols - 1) / smoe::kQBlock + 1) > INT32_MAX)
    return fail(MOE_ERR_UNSUPPORTED, "%lld rows of %d columns have 2^31 blocks or more", (long long)rows, cols);
  return MOE_OK;
}

int moe_quantize_rows(int64_t rows, int32_t cols, const moe_bf16* X, moe_fp8* q, uint8_t* scale, void* stream_) {
  int rc = check_rows(rows, cols);
  if (rc || rows == 0) return rc;
  CHECK_PTR(X, 16);
  CHECK_PTR(q, 8);
  CHECK_PTR(scale, 4);
  hipStream_t stream = (hipStream_t)stream_;
  LAUNCH(MOE_KC_QUANTIZE, smoe::launch_quantize_rows(X, rows, cols, q, scale, stream), "quantize rows");
  return MOE_OK;
}

int moe_dequantize_rows(int64_t rows, int32_t cols, const moe_fp8* q, const uint8_t* scale, moe_bf16* X, void* stream_) {
  int rc = check_rows(rows, cols);
  if (rc || rows == 0) return rc;
  CHECK_PTR(q, 8);
  CHECK_PTR(scale, 4);
  CHECK_PTR(X, 16);
  hipStream_t stream = (hipStream_t)stream_;
  LAUNCH(MOE_KC_QUANTIZE, smoe::launch_dequantize_rows(q, scale, rows, cols, X, stream), "dequantize rows");
  return MOE_OK;
}

size_t moe_qexperts_bytes(moe_dims m) { return check_dims(m) == MOE_OK ? qexperts_layout(m, nullptr, nullptr) : 0; }

int moe_qexperts_init(moe_dims m, void* buf, size_t bytes, moe_qexperts* q) {
  int rc = check_dims(m);
  if (rc) return rc;
  if (!q) return fail(MOE_ERR_INVALID_ARG, "q must not be null");
  CHECK_PTR(buf, kAlign);
  const size_t need = qexperts_layout(m, nullptr, nullptr);
  if (bytes < need) return fail(MOE_ERR_INVALID_ARG, "buffer of %zu bytes < required %zu", bytes, need);
  *q = moe_qexperts{m.d, m.n, m.E, MOE_HELD_EMPTY, nullptr, nullptr, nullptr, nullptr};
  qexperts_layout(m, (char*)buf, q);
  return MOE_OK;
}

int moe_quantize_experts(moe_dims m, const moe_bf16* W1, const moe_bf16* W2, moe_qexperts* q, void* stream_) {
  int rc = check_dims(m);
  if (rc) return rc;
  rc = check_qexperts(m, q, false);
  if (rc) return rc;
  CHECK_PTR(W1, 16);
  CHECK_PTR(W2, 16);
  hipStream_t stream = (hipStream_t)stream_;
  q->state = MOE_HELD_EMPTY;  // until the launch is enqueued
  LAUNCH(MOE_KC_QUANTIZE,
         smoe::launch_quantize_experts({W1, W2, q->W1, q->W1s, q->W2, q->W2s, nullptr, nullptr, m.d, m.n, m.E}, stream),
         "quantize experts");
  q->state = MOE_HELD_WRITTEN;
  return MOE_OK;
}

int moe_dequantize_experts(moe_dims m, const moe_qexperts* q, moe_bf16* W1, moe_bf16* W2, void* stream_) {
  int rc = check_dims(m);
  if (rc) return rc;
  rc = check_qexperts(m, q, true);
  if (rc) return rc;
  CHECK_PTR(W1, 16);
  CHECK_PTR(W2, 16);
  hipStream_t stream = (hipStream_t)stream_;
  LAUNCH(MOE_KC_QUANTIZE,
         smoe::launch_dequantize_experts({nullptr, nullptr, q->W1, q->W1s, q->W2, q->W2s, W1, W2, m.d, m.n, m.E}, stream),
         "dequantize experts");
  return MOE_OK;
}

static int check_ckpt_size(const moe_dims& m, int32_t capacity, int flags) {
  int rc = check_dims(m);
  if (rc) return rc;
  if (capacity < 1) return fail(MOE_ERR_CAPACITY, "capacity must be >= 1 (got %d)", capacity);
  if (flags & ~MOE_CKPT_X) return fail(MOE_ERR_INVALID_ARG, "unknown flags 0x%x", flags);
  return MOE_OK;
}

size_t moe_ckpt_bytes(moe_dims m, int32_t capacity, int flags) {
  return check_ckpt_size(m, capacity, flags) == MOE_OK ? ckpt_layout(m, capacity, flags, nullptr, nullptr) : 0;
}

int moe_ckpt_init(moe_dims m, int32_t capacity, int flags, void* buf, size_t bytes, moe_ckpt* c) {
  int rc = check_ckpt_size(m, capacity, flags);
  if (rc) return rc;
  if (!c) return fail(MOE_ERR_INVALID_ARG, "c must not be null");
  CHECK_PTR(buf, kAlign);
  const size_t need = ckpt_layout(m, capacity, flags, nullptr, nullptr);
  if (bytes < need) return fail(MOE_ERR_INVALID_ARG, "checkpoint buffer of %zu bytes < required %zu", bytes, need);
  *c = moe_ckpt{m.T, m.d, m.n, capacity, MOE_HELD_EMPTY, 0, nullptr, nullptr, nullptr, nullptr};
  ckpt_layout(m, capacity, flags, (char*)buf, c);
  return MOE_OK;
}

int moe_fwd_quant(moe_dims m, const moe_bf16* X, const moe_qexperts* q, const moe_expert_bias* eb, const moe_routing* r,
                  moe_ckpt* c, moe_bf16* O, void* ws, size_t ws_bytes, void* stream_) {
  int rc = check_dims(m);
  if (rc) return rc;
  rc = check_routing(m, r, 1, "r");
  if (rc) return rc;
  rc = check_built(r, "r");
  if (rc) return rc;
  rc = check_qexperts(m, q, true);
  if (rc) return rc;
  if (c) {
    rc = check_ckpt(m, r, c, false);
    if (rc) return rc;
  }
  CHECK_PTR(X, 16);
  CHECK_PTR(O, 16);
  rc = check_expert_bias(eb);
  if (rc) return rc;
  const size_t need = quant_layout(m, r->capacity, nullptr, nullptr);
  if (ws_bytes < need) return fail(MOE_ERR_WORKSPACE, "8-bit forward workspace %zu < required %zu", ws_bytes, need);
  CHECK_PTR(ws, kAlign);
  QuantWs w;
  quant_layout(m, r->capacity, (char*)ws, &w);
  hipStream_t stream = (hipStream_t)stream_;
  if (c) c->state = MOE_HELD_EMPTY;  // until all of it is enqueued
  uint8_t* X8 = c && c->X ? c->X : w.X8;
  uint8_t* Xs = c && c->X ? c->Xs : w.Xs;
  const smoe::QuantArgs a{X, X8, Xs, q->W1, q->W1s, q->W2, q->W2s, r->offsets, r->row_token, w.mtiles256, w.mtiles128,
                          eb ? eb->b1 : nullptr, eb ? eb->b2 : nullptr, w.A32, w.A8, w.As, c ? c->H : nullptr,
                          c ? c->Hs : nullptr, w.Y, w.Y32, m.d, m.n, m.E, r->capacity, smoe::quant_tiles(m, *r),
                          r->row_expert, r->row_w, r->tok_offsets, r->tok_rows, O};
  // (what is kept is written by the tiled projections)
  const smoe::StreamShape few = c ? smoe::StreamShape{0, 0} : smoe::stream8_shape(m, r->capacity, smoe::rounding_tile(*r));
  if (few.mb && smoe::stream8_by_token(m, *r)) {
    LAUNCH(MOE_KC_UP_QUANT, smoe::launch_stream8_row_up(a, m.T, m.K, stream), "8-bit up-proj");
    LAUNCH(MOE_KC_DOWN_QUANT, smoe::launch_stream8_token_down(a, m.T, stream), "8-bit down-proj and aggregation");
    return MOE_OK;
  }
  if (few.mb) {
    LAUNCH(MOE_KC_UP_QUANT, smoe::launch_stream8_up(a, few, stream), "8-bit up-proj");
    LAUNCH(MOE_KC_DOWN_QUANT, smoe::launch_stream8_down(a, few, stream), "8-bit down-proj");
    LAUNCH(MOE_KC_AGG_O, smoe::launch_agg_o_f32(w.Y32, *r, O, m.T, m.d, stream), "aggregation");
  } else {
    LAUNCH(MOE_KC_QUANTIZE, smoe::launch_quant_prepare(a, m.T, stream), "quantize X and m-tile lists");
    LAUNCH(MOE_KC_UP_QUANT, smoe::launch_quant_up(a, stream), "8-bit up-proj");
    LAUNCH(MOE_KC_DOWN_QUANT, smoe::launch_quant_down(a, stream), "8-bit down-proj");
    LAUNCH(MOE_KC_AGG_O, smoe::launch_agg_o(w.Y, *r, O, m.T, m.d, stream), "aggregation");
  }
  if (c) c->state = MOE_HELD_WRITTEN;
  return MOE_OK;
}

int moe_fwd_ckpt(moe_dims m, const moe_bf16* X, const moe_bf16* W1, const moe_bf16* W2, const moe_expert_bias* eb,
                 const moe_routing* r, moe_ckpt* c, moe_bf16* O, void* ws, size_t ws_bytes, void* stream_) {
  int rc = check_dims(m);
  if (rc) return rc;
  rc = check_routing(m, r, 1, "r");
  if (rc) return rc;
  rc = check_built(r, "r");
  if (rc) return rc;
  rc = check_ckpt(m, r, c, false);
  if (rc) return rc;
  CHECK_PTR(X, 16);
  CHECK_PTR(W1, 16);
  CHECK_PTR(W2, 16);
  CHECK_PTR(O, 16);
  rc = check_expert_bias(eb);
  if (rc) return rc;
  const size_t need = fwd_layout(m, r->capacity, nullptr, nullptr);
  if (ws_bytes < need) return fail(MOE_ERR_WORKSPACE, "forward workspace %zu < required %zu", ws_bytes, need);
  CHECK_PTR(ws, kAlign);
  FwdWs w;
  fwd_layout(m, r->capacity, (char*)ws, &w);
  hipStream_t stream = (hipStream_t)stream_;
  c->state = MOE_HELD_EMPTY;  // until all of it is enqueued
  const int64_t mt = smoe::expected_mtiles(m, *r);
  if (c->X)
    LAUNCH(MOE_KC_QUANTIZE, smoe::launch_ckpt_prepare(r->offsets, m.E, w.mtiles, X, m.T, m.d, c->X, c->Xs, stream),
           "quantize X and m-tile list");
  else
    HIP_TRY(smoe::launch_mtiles(r->offsets, m.E, w.mtiles, stream), "m-tile list");
  LAUNCH(MOE_KC_UP,
         smoe::launch_up_ckpt({X, W1, r->offsets, r->row_token, nullptr, w.A, m.d, m.n, m.E, r->capacity, mt, w.mtiles,
                               eb ? eb->b1 : nullptr, c->H, c->Hs},
                              stream),
         "up-proj");
  LAUNCH(MOE_KC_DOWN,
         Projections(m, *r).run_down({w.A, W2, r->offsets, w.Y, m.d, m.n, m.E, r->capacity, mt, w.mtiles, eb ? eb->b2 : nullptr},
                                     MOE_AGG_GATHER_SUM, stream),
         "down-proj");
  LAUNCH(MOE_KC_AGG_O, smoe::launch_agg_o(w.Y, *r, O, m.T, m.d, stream), "aggregation");
  c->state = MOE_HELD_WRITTEN;
  return MOE_OK;
}

int moe_bwd_ckpt(moe_dims m, const moe_bf16* dO, const moe_bf16* X, const moe_ckpt* c, const moe_bf16* W1,
                 const moe_bf16* W2, const moe_expert_bias* eb, const moe_bf16* Wr, const moe_routing* r, moe_bf16* dX,
                 moe_bf16* dW1, moe_bf16* dW2, float* dWr, float* dbias, float* dS, void* ws, size_t ws_bytes,
                 void* stream) {
  if (!c) return fail(MOE_ERR_INVALID_ARG, "the checkpoint must not be null");
  return backward(m, dO, X, nullptr, c, W1, W2, eb, Wr, r, dX, dW1, dW2, dWr, dbias, dS, ws, ws_bytes, stream);
}

// whether [p, p + n) and [q, q + m) share a byte
static bool overlap(const void* p, size_t n, const void* q, size_t m) {
  const uintptr_t a = (uintptr_t)p, b = (uintptr_t)q;
  return p && q && a < b + m && b < a + n;
}

// moe_decode and moe_decode_quant: what they check alike, and the launches
static int decode(const moe_dims& m, const moe_bf16* X, const moe_bf16* Wr, const float* bias, const moe_bf16* W1,
                  const moe_bf16* W2, const moe_qexperts* q, const moe_expert_bias* eb, const moe_bf16* R, moe_bf16* O,
                  int32_t* topk_idx, float* topk_w, void* ws, size_t ws_bytes, hipStream_t stream) {
  CHECK_PTR(X, 16);
  CHECK_PTR(Wr, 16);
  if (!q) {
    CHECK_PTR(W1, 16);
    CHECK_PTR(W2, 16);
  }
  CHECK_PTR(O, 16);
  if (!aligned(R, 16)) return fail(MOE_ERR_INVALID_ARG, "R must be 16-byte aligned");
  if (!aligned(bias, 4)) return fail(MOE_ERR_INVALID_ARG, "bias must be 4-byte aligned");
  if (!aligned(topk_idx, 4)) return fail(MOE_ERR_INVALID_ARG, "topk_idx must be 4-byte aligned");
  if (!aligned(topk_w, 4)) return fail(MOE_ERR_INVALID_ARG, "topk_w must be 4-byte aligned");
  const size_t rows = (size_t)m.T * m.d * 2;
  if (overlap(O, rows, X, rows)) return fail(MOE_ERR_INVALID_ARG, "O must not overlap X, which is read until the end");
  if (R != O && overlap(O, rows, R, rows)) return fail(MOE_ERR_INVALID_ARG, "R must be O itself or not overlap it");
  int rc = check_expert_bias(eb);
  if (rc) return rc;
  const size_t need = decode_layout(m, q, nullptr, nullptr);
  if (ws_bytes < need) return fail(MOE_ERR_WORKSPACE, "workspace %zu < required %zu", ws_bytes, need);
  CHECK_PTR(ws, kAlign);
  DecodeWs w;
  decode_layout(m, q, (char*)ws, &w);
  smoe::DecodeArgs a{X, Wr, bias, W1, W2, eb ? eb->b1 : nullptr, eb ? eb->b2 : nullptr, R, O, topk_idx, topk_w, w.part,
                     w.sync, w.picked, q ? nullptr : (uint16_t*)w.A, w.Y, w.H32, m.T, m.d, m.n, m.E, m.K};
  if (q) {
    a.W1q = q->W1;
    a.W1s = q->W1s;
    a.W2q = q->W2;
    a.W2s = q->W2s;
    a.A32 = (float*)w.A;
  }
  LAUNCH(MOE_KC_DECODE, smoe::launch_decode(a, stream), "layer of few tokens");
  return MOE_OK;
}

int moe_decode(moe_dims m, const moe_bf16* X, const moe_bf16* Wr, const float* bias, const moe_bf16* W1, const moe_bf16* W2,
               const moe_expert_bias* eb, const moe_bf16* R, moe_bf16* O, int32_t* topk_idx, float* topk_w, void* ws,
               size_t ws_bytes, void* stream) {
  int rc = check_decode(m);
  if (rc) return rc;
  return decode(m, X, Wr, bias, W1, W2, nullptr, eb, R, O, topk_idx, topk_w, ws, ws_bytes, (hipStream_t)stream);
}

int moe_decode_quant(moe_dims m, const moe_bf16* X, const moe_bf16* Wr, const float* bias, const moe_qexperts* q,
                     const moe_expert_bias* eb, const moe_bf16* R, moe_bf16* O, int32_t* topk_idx, float* topk_w, void* ws,
                     size_t ws_bytes, void* stream) {
  int rc = check_decode(m);
  if (rc) return rc;
  rc = check_qexperts(m, q, true);
  if (rc) return rc;
  return decode(m, X, Wr, bias, nullptr, nullptr, q, eb, R, O, topk_idx, topk_w, ws, ws_bytes, (hipStream_t)stream);
}

// ---------------------------------------------------------------- dense products
static int check_linear(moe_linear& l) {
  if (l.T < 1) return fail(MOE_ERR_INVALID_ARG, "T must be >= 1 (got %d)", l.T);
  if (l.k < 8 || l.k % 8) return fail(MOE_ERR_UNSUPPORTED, "k must be a positive multiple of 8 (got %d)", l.k);
  if (l.n < 8 || l.n % 8) return fail(MOE_ERR_UNSUPPORTED, "n must be a positive multiple of 8 (got %d)", l.n);
  if (l.act < MOE_ACT_NONE || l.act > MOE_ACT_SWIGLU) return fail(MOE_ERR_INVALID_ARG, "unknown activation %d", l.act);
  if (l.k >= 1 << 24 || l.n >= 1 << 24) return fail(MOE_ERR_UNSUPPORTED, "k = %d, n = %d: must be below 2^24", l.k, l.n);
  // (counts of tiles, row chunks and threads of a launch are 32-bit)
  if (l.T > 1 << 28) return fail(MOE_ERR_UNSUPPORTED, "T must be at most 2^28 (got %d)", l.T);
  const int64_t most = (int64_t)1 << 37, N = l.act == MOE_ACT_SWIGLU ? 2 * (int64_t)l.n : l.n;
  if (l.T * N > most || (int64_t)l.T * l.k > most || l.k * N > most)
    return fail(MOE_ERR_UNSUPPORTED, "T = %d, k = %d, n = %d: no matrix may have more than 2^37 elements", l.T, l.k, l.n);
  int32_t* ld[] = {&l.ldx, &l.ldr, &l.ldy};
  const char* name[] = {"ldx", "ldr", "ldy"};
  const int len[] = {l.k, l.n, l.n};
  for (int i = 0; i < 3; ++i) {
    if (*ld[i] == 0) *ld[i] = len[i];
    if (*ld[i] < len[i] || *ld[i] % 8 || *ld[i] >= 1 << 30)
      return fail(MOE_ERR_INVALID_ARG, "%s must be a multiple of 8, at least %d and below 2^30 (got %d)", name[i], len[i], *ld[i]);
  }
  return MOE_OK;
}
// bytes of T rows of `cols` bf16 that are `ld` apart
static size_t rows_bytes(int64_t T, int64_t cols, int64_t ld) { return 2 * (size_t)((T - 1) * ld + cols); }
struct Region {
  const char* name;
  const void* p;
  size_t bytes;
};
static int check_overlap(const Region& out, std::initializer_list<Region> others) {
  for (const Region& r : others)
    if (overlap(out.p, out.bytes, r.p, r.bytes)) return fail(MOE_ERR_INVALID_ARG, "%s must not overlap %s", out.name, r.name);
  return MOE_OK;
}
static int64_t linear_columns(const moe_linear& l) { return l.act == MOE_ACT_SWIGLU ? 2 * (int64_t)l.n : l.n; }

namespace {
struct LinearBwdWs {
  uint16_t* dP;
  float* db;
  float* dx;
  float* dw;
};
size_t linear_bwd_layout(const moe_linear& l, char* base, LinearBwdWs* w) {
  const int64_t N = linear_columns(l);
  size_t off = 0;
  off = carve(base, off, l.act == MOE_ACT_NONE ? 0 : (size_t)l.T * N * 2, w ? (void**)&w->dP : nullptr);
  off = carve(base, off, smoe::linear_db_part_bytes(l.T, N), w ? (void**)&w->db : nullptr);
  off = carve(base, off, smoe::linear_dx_part_bytes(l.T, l.k, N), w ? (void**)&w->dx : nullptr);
  off = carve(base, off, smoe::linear_dw_part_bytes(l.T, l.k, N), w ? (void**)&w->dw : nullptr);
  return off;
}
}  // namespace

size_t moe_linear_workspace_bytes(moe_linear l, int which) {
  if (check_linear(l) != MOE_OK) return 0;
  if (which == MOE_WS_LINEAR_FWD)
    return kAlign + align_up(smoe::linear_fwd_part_bytes(l.T, l.k, l.n, l.act, l.ldx));
  if (which == MOE_WS_LINEAR_BWD) return kAlign + linear_bwd_layout(l, nullptr, nullptr);
  return 0;
}

int moe_linear_fwd(moe_linear l, const moe_bf16* X, const moe_bf16* W, const float* b, const moe_bf16* R, moe_bf16* H,
                   moe_bf16* Y, void* ws, size_t ws_bytes, void* stream_) {
  int rc = check_linear(l);
  if (rc) return rc;
  CHECK_PTR(X, 16);
  CHECK_PTR(W, 16);
  CHECK_PTR(Y, 16);
  if (!aligned(b, 16)) return fail(MOE_ERR_INVALID_ARG, "b must be 16-byte aligned");
  if (!aligned(R, 16)) return fail(MOE_ERR_INVALID_ARG, "R must be 16-byte aligned");
  if (!aligned(H, 16)) return fail(MOE_ERR_INVALID_ARG, "H must be 16-byte aligned");
  const int64_t N = linear_columns(l);
  const Region x{"X", X, rows_bytes(l.T, l.k, l.ldx)}, wr{"W", W, 2 * (size_t)l.k * N}, bb{"b", b, 4 * (size_t)N};
  const Region h{"H", H, 2 * (size_t)l.T * N}, y{"Y", Y, rows_bytes(l.T, l.n, l.ldy)};
  const bool in_place = R == Y && l.ldr == l.ldy;
  const Region r{"R (unless it is Y, with ldr = ldy)", in_place ? nullptr : R, rows_bytes(l.T, l.n, l.ldr)};
  rc = check_overlap(y, {x, wr, bb, h, r});
  if (rc) return rc;
  rc = check_overlap(h, {x, wr, bb, r});
  if (rc) return rc;
  const size_t need = moe_linear_workspace_bytes(l, MOE_WS_LINEAR_FWD);
  if (ws_bytes < need) return fail(MOE_ERR_WORKSPACE, "workspace %zu < required %zu", ws_bytes, need);
  CHECK_PTR(ws, kAlign);
  hipStream_t stream = (hipStream_t)stream_;
  LAUNCH(MOE_KC_LINEAR,
         smoe::launch_linear_fwd({X, W, b, R, H, Y, (float*)ws, l.T, l.k, l.n, l.act, l.ldx, l.ldr, l.ldy}, stream),
         "dense product");
  return MOE_OK;
}

int moe_linear_bwd(moe_linear l, const moe_bf16* dY, const moe_bf16* X, const moe_bf16* W, const moe_bf16* H,
                   const moe_bf16* G, moe_bf16* dX, moe_bf16* dW, float* db, void* ws, size_t ws_bytes, void* stream_) {
  int rc = check_linear(l);
  if (rc) return rc;
  CHECK_PTR(dY, 16);
  if (dW) CHECK_PTR(X, 16);
  if (dX) CHECK_PTR(W, 16);
  if (l.act != MOE_ACT_NONE) CHECK_PTR(H, 16);
  if (!aligned(G, 16)) return fail(MOE_ERR_INVALID_ARG, "G must be 16-byte aligned");
  if (!aligned(dX, 16)) return fail(MOE_ERR_INVALID_ARG, "dX must be 16-byte aligned");
  if (!aligned(dW, 16)) return fail(MOE_ERR_INVALID_ARG, "dW must be 16-byte aligned");
  if (!aligned(db, 16)) return fail(MOE_ERR_INVALID_ARG, "db must be 16-byte aligned");
  if (!dX && !dW && !db) return fail(MOE_ERR_INVALID_ARG, "dX, dW and db must not all be null");
  const int64_t N = linear_columns(l);
  const Region dy{"dY", dY, rows_bytes(l.T, l.n, l.ldy)}, x{"X", X, rows_bytes(l.T, l.k, l.ldx)}, wr{"W", W, 2 * (size_t)l.k * N};
  const Region h{"H", H, 2 * (size_t)l.T * N}, g{"G (unless it is dX)", G == dX ? nullptr : G, rows_bytes(l.T, l.k, l.ldx)};
  const Region dx{"dX", dX, rows_bytes(l.T, l.k, l.ldx)}, dw{"dW", dW, 2 * (size_t)l.k * N}, b{"db", db, 4 * (size_t)N};
  rc = check_overlap(dx, {dy, x, wr, h, g, dw, b});
  if (rc) return rc;
  rc = check_overlap(dw, {dy, x, wr, h, g, b});
  if (rc) return rc;
  rc = check_overlap(b, {dy, x, wr, h, g});
  if (rc) return rc;
  const size_t need = moe_linear_workspace_bytes(l, MOE_WS_LINEAR_BWD);
  if (ws_bytes < need) return fail(MOE_ERR_WORKSPACE, "workspace %zu < required %zu", ws_bytes, need);
  CHECK_PTR(ws, kAlign);
  LinearBwdWs w;
  linear_bwd_layout(l, (char*)ws, &w);
  hipStream_t stream = (hipStream_t)stream_;
  LAUNCH(MOE_KC_LINEAR_BWD,
         smoe::launch_linear_bwd({dY, X, W, H, G, dX, dW, db, l.act == MOE_ACT_NONE ? nullptr : w.dP, w.db, w.dx, w.dw, l.T, l.k,
                                  l.n, l.act, l.ldx, l.ldy},
                                 stream),
         "dense product's gradients");
  return MOE_OK;
}

int moe_prof_select(int kc) {
  if (kc < -1 || kc >= MOE_KC_COUNT) return fail(MOE_ERR_INVALID_ARG, "unknown kernel class %d", kc);
  std::lock_guard<std::mutex> lk(g_prof_mu);
  g_prof_class = kc;
  return MOE_OK;
}

int moe_prof_read(double* ms, int32_t* launches) {
  std::lock_guard<std::mutex> lk(g_prof_mu);
  double total = 0.0;
  int32_t count = 0;
  for (auto& ev : g_prof_events) {
    hipError_t e = hipEventSynchronize(ev.second);
    if (e != hipSuccess) return hip_fail(e, "prof event");
    float t = 0.f;
    e = hipEventElapsedTime(&t, ev.first, ev.second);
    if (e != hipSuccess) return hip_fail(e, "prof elapsed");
    total += t;
    ++count;
    g_prof_pool.push_back(ev);
  }
  g_prof_events.clear();
  if (ms) *ms = total;
  if (launches) *launches = count;
  return MOE_OK;
}

const char* moe_kernel_class_name(int kc) {
  static const char* names[MOE_KC_COUNT] = {"router_gemm", "topk", "routing_meta", "token_round", "up_proj",
                                            "down_proj", "aggregate_O", "dH", "dW2", "dXtilde",
                                            "dW1", "aggregate_dX", "dWr", "router_topk", "quantize",
                                            "up_proj_quant", "down_proj_quant", "decode", "linear",
                                            "linear_bwd"};
  return (kc >= 0 && kc < MOE_KC_COUNT) ? names[kc] : "unknown";
}

}  // extern "C"

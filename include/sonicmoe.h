/*
 * sonicmoe.h -- C ABI of an MI355X (gfx950) implementation of the SonicMoE
 * layer: "SonicMoE: Accelerating MoE with IO and Tile-aware Optimizations"
 * (arXiv 2512.14080).
 *
 * The layer follows the paper's problem statement (Appendix A, notation table):
 *   X[T,d]            token embeddings
 *   W_r[d,E]          router weights (token-choice top-K, Section 2.3)
 *   W1[E,d,2n]        expert up-projections; columns [0,n) are the SwiGLU gate,
 *                     columns [n,2n) the up branch
 *   W2[E,n,d]         expert down-projections
 *   K                 experts per token
 *
 * Conventions for every entry point:
 *   - bf16 tensors are raw IEEE bfloat16 bit patterns (uint16_t).
 *   - Every pointer is a DEVICE pointer unless stated otherwise, caller-owned,
 *     row-major and contiguous.  The library never allocates device memory,
 *     never synchronises the stream and keeps no pointer after it returns.
 *   - `stream` is a hipStream_t (NULL = the default stream); all work is
 *     enqueued asynchronously on it.
 *   - Arguments are validated on the host before anything is enqueued; on a
 *     validation error nothing is enqueued and a negative MOE_ERR_* code is
 *     returned.  moe_last_error() returns a thread-local description of the
 *     last failure.  A HIP launch failure returns MOE_ERR_HIP.
 *   - Outputs are overwritten, never accumulated into.
 */
#ifndef SONICMOE_H
#define SONICMOE_H

#include <stddef.h>
#include <stdint.h>

#ifdef __cplusplus
extern "C" {
#endif

typedef uint16_t moe_bf16;

typedef struct {
  int32_t T; /* tokens in the microbatch, >= 1 */
  int32_t d; /* model dimension, multiple of 128 */
  int32_t n; /* expert intermediate dimension, multiple of 64 */
  int32_t E; /* experts, multiple of 8, <= 4096 */
  int32_t K; /* experts per token, 1 <= K <= min(E, 16) */
} moe_dims;

/* Error codes. */
enum {
  MOE_OK = 0,
  MOE_ERR_INVALID_ARG = -1, /* null pointer, bad size, misaligned pointer   */
  MOE_ERR_UNSUPPORTED = -2, /* a shape outside the supported range          */
  MOE_ERR_CAPACITY = -3,    /* routing capacity below the worst-case rows   */
  MOE_ERR_WORKSPACE = -4,   /* workspace smaller than moe_workspace_bytes() */
  MOE_ERR_HIP = -5          /* a HIP runtime call or kernel launch failed   */
};

/*
 * Routing metadata of one routing matrix pi in {0,1}^{T x E} (Appendix A) and
 * its softmax scores.  "Rows" are routed (token, expert) pairs; P = sum_e f_e
 * of them exist after routing (P = T*K for token choice).  All arrays live in
 * one caller-allocated device buffer laid out by moe_routing_init().
 *
 * Integer results are a deterministic function of the fp32 scores:
 *   - experts are selected by (score descending, expert index ascending);
 *   - expert-major rows are ordered by (expert ascending, token ascending);
 *   - each token's rows are listed by expert ascending.
 */
typedef struct {
  int32_t capacity;      /* rows the row_* / tok_rows arrays can hold          */
  int32_t words;         /* W = ceil(T/64), 64-bit words per expert in mask    */
  int32_t state;         /* host-side build state, MOE_ROUTING_STATE_*: set by
                            moe_routing_init / moe_route / moe_round_tokens
                            (what has been enqueued), checked by the consumers */
  int32_t reserved;      /* internal, host-side: m_tile of the rounding that built
                            it, else zero; it only guides the choice of kernels */
  float *logits;         /* [T,E] router logits (nullable: MOE_ROUTING_LOGITS)  */
  float *scores;         /* [T,E] S_full = softmax over all E experts          */
  float *scores_t;       /* [E,T] transposed S_full (nullable: MOE_ROUTING_SCORES_T;
                            required by moe_round_tokens on the TC routing)    */
  int32_t *topk_idx;     /* [T,K] TC selection, (score desc, expert asc)       */
  float *topk_w;         /* [T,K] renormalised weights of topk_idx             */
  uint64_t *mask;        /* [E,W] membership bitmap: bit t%64 of word t/64     */
  int32_t *mask_prefix;  /* [E,W] set bits of expert e before each word        */
  int32_t *counts;       /* [E]   f_e, rows per expert                         */
  int32_t *offsets;      /* [E+1] exclusive scan of counts; offsets[E] = P     */
  int32_t *row_token;    /* [capacity] token of each expert-major row (gather) */
  int32_t *row_expert;   /* [capacity] expert of each row                      */
  float *row_w;          /* [capacity] weight s_{t,e} of each row              */
  int32_t *tok_offsets;  /* [T+1] CSR offsets of the token-major view          */
  int32_t *tok_rows;     /* [capacity] rows of each token, expert ascending    */
  int32_t *tok_count;    /* [T]   experts of each token                        */
  float *tok_denom;      /* [T]   sum of the token's selected scores           */
  int32_t *round_dir;    /* [E]   -1 dropped / 0 kept / +1 padded (rounding)   */
  int32_t *scratch;      /* internal: scans, the rounding select's lists, the
                            router's partial logits of few tokens             */
  int32_t *status;       /* [1]   device word: 0 once the metadata kernels have
                            run on a consistent selection; otherwise the OR of
                            MOE_STATUS_* bits, and the rows are not valid
                            (every index written is still in bounds)        */
} moe_routing;

/* moe_routing.state */
enum {
  MOE_ROUTING_STATE_EMPTY = 0,  /* laid out by moe_routing_init; nothing written  */
  MOE_ROUTING_STATE_COUNTS = 1, /* mask, mask_prefix, counts (MOE_ROUTE_COUNTS_ONLY) */
  MOE_ROUTING_STATE_BUILT = 2   /* complete metadata: moe_fwd / moe_bwd accept it */
};

/* bits of the device status word */
enum {
  MOE_STATUS_DUPLICATE_EXPERT = 1 /* a token's topk_idx lists an expert twice   */
};

enum {
  MOE_ROUTING_LOGITS = 1,   /* carve the logits array                 */
  MOE_ROUTING_SCORES_T = 2  /* carve the transposed-scores array      */
};

/* Bytes of the routing buffer for `capacity` rows; 0 if the dims are invalid. */
size_t moe_routing_bytes(moe_dims dims, int32_t capacity, int flags);

/* Lays out the routing arrays inside `buf` (device, 256-byte aligned, at least
 * moe_routing_bytes() bytes) and fills `*r` (host struct, state
 * MOE_ROUTING_STATE_EMPTY).  Enqueues nothing. */
int moe_routing_init(moe_dims dims, int32_t capacity, int flags, void *buf, size_t bytes,
                     moe_routing *r);

/* Smallest capacity that token rounding to multiples of m_tile may need:
 * min(T*E, T*K + E*(m_tile-1)); -1 for invalid dims or an m_tile outside
 * the powers of two in [8, 256]. */
int32_t moe_round_capacity(moe_dims dims, int32_t m_tile);

/* moe_route flags */
enum {
  MOE_ROUTE_SCORES_IN = 1,     /* skip the router GEMM and softmax; r->scores is
                                  an input holding S_full                      */
  MOE_ROUTE_WRITE_LOGITS = 2,  /* keep the logits in r->logits                 */
  MOE_ROUTE_WRITE_SCORES_T = 4, /* also write r->scores_t                      */
  MOE_ROUTE_COUNTS_ONLY = 8,    /* metadata stops at mask, mask_prefix and
                                   counts: enough for moe_round_tokens, which
                                   builds the rounded routing's own metadata;
                                   offsets and the row lists are not written,
                                   and r->state becomes MOE_ROUTING_STATE_COUNTS,
                                   which moe_fwd and moe_bwd refuse          */
  MOE_ROUTE_SEPARATE_TOPK = 16  /* run the router GEMM and softmax/top-K as two
                                   launches even where they fuse (with more
                                   than 4096 tokens the logits then pass
                                   through r->logits or r->scores)           */
};

/*
 * Token-choice top-K routing (Section 2.3; top-K selection of Appendix D).
 *   logits = X W_r (+ bias)  fp32 accumulation of bf16 inputs
 *   S_full = softmax over E  (row maximum subtracted)
 *   sel(t) = first K experts by (S_full desc, expert asc)
 *   s_{t,e} = S_full[t,e] / sum_{e' in sel(t)} S_full[t,e']   (denominator
 *             summed over selected experts in ascending index order)
 * then the metadata of the routing matrix: mask, counts, offsets, expert-major
 * rows (row_token, row_expert, row_w), token-major CSR (tok_offsets, tok_rows).
 *   X     [T,d] bf16;  Wr [d,E] bf16 (unused with MOE_ROUTE_SCORES_IN)
 *   bias  [E] fp32, nullable
 * r->capacity must be >= T*K.  On success r->state is MOE_ROUTING_STATE_BUILT
 * (MOE_ROUTING_STATE_COUNTS with MOE_ROUTE_COUNTS_ONLY) and the device word
 * r->status is cleared by the metadata kernels.
 * With T > 4096, E <= 256 and K <= 8 the softmax and top-K run in the
 * router GEMM's epilogue (one launch; the logits are written only with
 * MOE_ROUTE_WRITE_LOGITS).  Its scores may differ from the two-launch path's
 * in the last bits (the order of the softmax sum); selection, mask and weights
 * are those the two-launch path derives from the scores it writes.
 * With T <= 4096 and E <= 1024 (d E < 2^31) other kernels run, built for few
 * tokens: the router GEMM's partial sums pass through r->scratch or r->scores.
 * MOE_ROUTE_SEPARATE_TOPK only changes the timing classes there.  Calls with
 * MOE_ROUTE_COUNTS_ONLY take them for small T K only.
 * Scores are compared through the order-preserving image of their fp32 bit
 * pattern, which is the float order for numbers (+0 = -0) and extends it to
 * NaN (sign clear: above +Inf; sign set: below -Inf), so non-finite scores
 * still select K distinct experts per token (their weights are then not
 * finite).  Token rounding orders scores the same way.
 */
int moe_route(moe_dims dims, const moe_bf16 *X, const moe_bf16 *Wr, const float *bias, int flags,
              moe_routing *r, void *stream);

/* rounding subroutines (Section 5.2 and the appendix ablation on rounding) */
enum {
  MOE_ROUND_NEAREST = 0,   /* NR-f: pad iff ceil - f < f - floor (default)        */
  MOE_ROUND_UP = 1,        /* always pad                                          */
  MOE_ROUND_DOWN = 2,      /* always drop (TC token dropping)                     */
  MOE_ROUND_BALANCE = 3,   /* Balance-f: running residual over experts in order   */
  MOE_ROUND_STOCHASTIC = 4 /* SR-f: pad iff u_e * m_tile < f - floor               */
};

/*
 * Token rounding (Section 5.2): rounds every expert's TC frequency f_e to a
 * multiple of m_tile.  Per expert, tokens are ordered by (TC first, score
 * descending, token ascending) and the first f^TR_e are kept, so a rounded-down
 * expert drops its lowest-scored TC tokens and a rounded-up expert adds the
 * highest-scored non-TC tokens; |f^TR_e - f_e| < m_tile.  An expert whose
 * ceiling exceeds T is rounded down.  Weights are renormalised over each
 * token's new expert set.
 *   tc     routing written by moe_route (state at least
 *          MOE_ROUTING_STATE_COUNTS; needs tc->scores_t written, i.e.
 *          MOE_ROUTE_WRITE_SCORES_T)
 *   tr     output routing; tr->capacity >= moe_round_capacity(dims, m_tile);
 *          tr->scores may alias tc->scores (it is read, not written); on
 *          success tr->state is MOE_ROUTING_STATE_BUILT
 *   m_tile power of two in [8, 256] (otherwise MOE_ERR_INVALID_ARG)
 *   u      [E] fp32 uniforms in [0,1), device, required by MOE_ROUND_STOCHASTIC
 */
int moe_round_tokens(moe_dims dims, int32_t m_tile, int mode, const float *u, const moe_routing *tc,
                     moe_routing *tr, void *stream);

/*
 * Optional per-expert biases of the two projections (the expert-bias footnote
 * of the "Gradient computation" appendix).  With them the expert computes
 *   h = x W1_e + b1_e,  y = SwiGLU(h) W2_e + b2_e,
 * and the score gradient dS_{t,e} = <dO_t, y> becomes <dA', A> + <dO_t, b2_e>.
 * Every pointer is a device pointer, fp32, 16-byte aligned, and nullable:
 *   b1   [E,2n] up-projection bias (gate columns first, as W1)
 *   b2   [E,d]  down-projection bias
 *   db1  [E,2n] out of moe_bwd: column sums of dH over the expert's rows
 *   db2  [E,d]  out of moe_bwd: column sums of s * dO_t over the expert's rows
 * Experts without rows get zero bias gradients.  moe_fwd reads b1 and b2;
 * moe_bwd reads b2 (for dS) and writes db1 and db2 where they are given.
 */
typedef struct {
  const float *b1;
  const float *b2;
  float *db1;
  float *db2;
} moe_expert_bias;

/* Workspace bytes for moe_fwd (which = 1), moe_bwd (which = 2),
 * moe_fwd_aggregation_ablation (which = 3), moe_fwd_quant (which = 4),
 * moe_fwd_ckpt (which = 5), moe_bwd_ckpt (which = 6), moe_decode (which = 7) and
 * moe_decode_quant (which = 8; these two whatever the capacity). */
enum {
  MOE_WS_FWD = 1, MOE_WS_BWD = 2, MOE_WS_FWD_AGG_ABLATION = 3,
  MOE_WS_FWD_QUANT = 4, MOE_WS_FWD_CKPT = 5, MOE_WS_BWD_CKPT = 6,
  MOE_WS_DECODE = 7, MOE_WS_DECODE_QUANT = 8
};
size_t moe_workspace_bytes(moe_dims dims, int32_t capacity, int which);

/*
 * Forward (Section 3, forward algorithm: up-proj A kernel, down-proj Y kernel,
 * expert aggregation O kernel):
 *   H = gather(X) W1_e (+ b1_e)   -> H [capacity,2n] bf16 (cached for backward;
 *                                    the first P rows are written)
 *   A = SiLU(H_gate) * H_up       (workspace)
 *   Y = A W2_e (+ b2_e)           (workspace)
 *   O_t = sum_{rows of t} s * Y   -> O [T,d] bf16 (zero for a token without experts)
 *   eb  expert biases, nullable (b1 and b2 are read; see moe_expert_bias)
 *   r   routing in state MOE_ROUTING_STATE_BUILT (otherwise MOE_ERR_INVALID_ARG)
 *   ws  device workspace of moe_workspace_bytes(dims, r->capacity, MOE_WS_FWD)
 */
int moe_fwd(moe_dims dims, const moe_bf16 *X, const moe_bf16 *W1, const moe_bf16 *W2,
            const moe_expert_bias *eb, const moe_routing *r, moe_bf16 *H, moe_bf16 *O, void *ws,
            size_t ws_bytes, void *stream);

/*
 * Backward (down-projection backward algorithm of Section 3; up-projection
 * backward algorithm of Appendix E; dS identity of the "Gradient computation"
 * appendix), recomputing A from the cached H:
 *   dA' = gather(dO) W2_e^T, dS = <dA', A>, dA = s dA', dH = dSwiGLU(dA, H),
 *   A' = s A, dW2_e = A'^T gather(dO), dX~ = dH W1_e^T, dW1_e = gather(X)^T dH,
 *   dX_t = sum_{rows of t} dX~ + dL_t W_r^T,
 * where the router gradient on each token's selected set is
 *   dl_j = s_j (dS_j - sum_k s_k dS_k)  (softmax over the selected logits),
 *   dW_r = X^T dL, dbias = column sums of dL.
 *   eb   expert biases, nullable: b2 adds <dO_t, b2_e> to dS; db1 and db2 are
 *        written where given (see moe_expert_bias)
 *   r    routing in state MOE_ROUTING_STATE_BUILT (otherwise MOE_ERR_INVALID_ARG)
 *   dO   [T,d] bf16           H [capacity,2n] bf16 from moe_fwd
 *   Wr   [d,E] bf16, nullable: then no router gradient is formed and dX holds
 *        only the expert part
 *   dX   [T,d] bf16 out;  dW1 [E,d,2n] bf16 out;  dW2 [E,n,d] bf16 out
 *        (experts without rows get zero weight gradients)
 *   dWr  [d,E] fp32 out, nullable;  dbias [E] fp32 out, nullable
 *   dS   [capacity] fp32 out, nullable (dS of each expert-major row)
 *   ws   device workspace of moe_workspace_bytes(dims, r->capacity, MOE_WS_BWD)
 */
int moe_bwd(moe_dims dims, const moe_bf16 *dO, const moe_bf16 *X, const moe_bf16 *H,
            const moe_bf16 *W1, const moe_bf16 *W2, const moe_expert_bias *eb, const moe_bf16 *Wr,
            const moe_routing *r,
            moe_bf16 *dX, moe_bf16 *dW1, moe_bf16 *dW2, float *dWr, float *dbias, float *dS, void *ws,
            size_t ws_bytes, void *stream);

/*
 * moe_fwd for callers that cannot allocate device memory (code under HIP
 * graph capture, tight serving loops, harnesses that forbid allocation): the
 * same forward, with its workspace (A, Y and the m-tile list) in a static
 * device array of moe_fwd_static_max_bytes() = 64 MiB that the library holds
 * on every GPU it runs on until the process ends.  No allocation happens in
 * the call.  A routing whose forward workspace
 * (moe_workspace_bytes(dims, r->capacity, MOE_WS_FWD)) exceeds the array is
 * refused with MOE_ERR_WORKSPACE before anything is enqueued.  Every call on
 * one GPU uses that GPU's one array: calls that overlap on a GPU (on
 * different streams, or from different threads without ordering) race.  The
 * array belongs to the current device (hipGetDevice), which must be the
 * stream's.  Other arguments as moe_fwd.
 */
size_t moe_fwd_static_max_bytes(void);
int moe_fwd_static(moe_dims dims, const moe_bf16 *X, const moe_bf16 *W1, const moe_bf16 *W2,
                   const moe_expert_bias *eb, const moe_routing *r, moe_bf16 *H, moe_bf16 *O, void *stream);

/*
 * Expert-aggregation ablation (Appendix F.3 and the expert-aggregation
 * figure of the "Referenced tables" appendix): the forward of moe_fwd with
 * the down-projection and the aggregation done by one of three strategies.
 * Not on the layer's path; it exists to measure the choice.
 *   MOE_AGG_GATHER_SUM   Y stored expert-major, each token gathers and sums
 *                        its rows (what moe_fwd does; deterministic)
 *   MOE_AGG_SCATTER_SUM  the down-projection epilogue scatters each Y row to
 *                        its token-major slot, then a contiguous weighted sum
 *   MOE_AGG_ATOMIC_F32   the epilogue adds s * bf16(Y) into an fp32 O with
 *                        atomics (order-dependent rounding), then O -> bf16
 * No expert biases.  ws: moe_workspace_bytes(dims, r->capacity,
 * MOE_WS_FWD_AGG_ABLATION) bytes; other arguments as moe_fwd.
 */
enum { MOE_AGG_GATHER_SUM = 0, MOE_AGG_SCATTER_SUM = 1, MOE_AGG_ATOMIC_F32 = 2 };
int moe_fwd_aggregation_ablation(moe_dims dims, const moe_bf16 *X, const moe_bf16 *W1, const moe_bf16 *W2,
                                 const moe_routing *r, moe_bf16 *H, moe_bf16 *O, int strategy, void *ws,
                                 size_t ws_bytes, void *stream);

/*
 * 8-bit block format.  A block of up to 128 values is held as e4m3 codes (OCP
 * 8-bit floating point: no infinities, largest value 448) and one scale byte b,
 * which stands for 2^(b - 127):
 *   amax  = the largest finite |x| of the block
 *   e     = the least integer >= -126 with amax <= 448 * 2^e;  b = e + 127
 *   code  = e4m3(x * 2^-e), rounded to nearest even; infinities and NaN become
 *           the NaN code (and stay visible: they do not move the others' scale)
 *   value = code * 2^e; at most 2^-4 |x| off where |value| >= 2^(e - 6)
 * Blocks are 128 consecutive columns of a row (the last one of a row may be
 * shorter) and, for expert weights, 128 x 128 (W1: within the gate and within
 * the up half; H likewise).
 */
typedef uint8_t moe_fp8;

/* Bytes from one row's scales to the next: a row of `cols` columns has
 * ceil(cols / 128) scale bytes, padded to a multiple of 4.  0 for cols < 1. */
int32_t moe_scale_stride(int32_t cols);

/*
 * Rows of activations into the 8-bit block format and back (values of a block
 * whose scale is the smallest may be rounded to bf16's own smallest, 2^-133).
 *   rows   >= 0 (0: nothing is enqueued); cols a multiple of 8, >= 8;
 *          rows * ceil(cols / 128) below 2^31
 *   X      [rows,cols] bf16, 16-byte aligned
 *   q      [rows,cols] codes, 8-byte aligned
 *   scale  [rows][moe_scale_stride(cols)] bytes, 4-byte aligned; the bytes past a
 *          row's last block are written as 127
 * Inputs and outputs must not overlap.
 */
int moe_quantize_rows(int64_t rows, int32_t cols, const moe_bf16 *X, moe_fp8 *q, uint8_t *scale, void *stream);
int moe_dequantize_rows(int64_t rows, int32_t cols, const moe_fp8 *q, const uint8_t *scale, moe_bf16 *X,
                        void *stream);

/* moe_qexperts.state and moe_ckpt.state */
enum {
  MOE_HELD_EMPTY = 0,  /* laid out; nothing written                            */
  MOE_HELD_WRITTEN = 1 /* a call that writes it has been enqueued              */
};

/*
 * The expert weights in the 8-bit block format, in the layout that the products
 * of moe_fwd_quant read (k contiguous, n padded with zeros to a multiple of
 * 128): written by moe_quantize_experts, read back by moe_dequantize_experts.
 * One caller-allocated device buffer, laid out by moe_qexperts_init.
 */
typedef struct {
  int32_t d, n, E; /* of the layer                                             */
  int32_t state;   /* host-side, MOE_HELD_*                                    */
  moe_fp8 *W1;
  uint8_t *W1s;
  moe_fp8 *W2;
  uint8_t *W2s;
} moe_qexperts;

/* (T and K of the dims only have to be valid) */
size_t moe_qexperts_bytes(moe_dims dims);
int moe_qexperts_init(moe_dims dims, void *buf, size_t bytes, moe_qexperts *q);
/* W1 [E,d,2n], W2 [E,n,d] bf16; q->state becomes MOE_HELD_WRITTEN */
int moe_quantize_experts(moe_dims dims, const moe_bf16 *W1, const moe_bf16 *W2, moe_qexperts *q, void *stream);
/* the values that q stands for, as bf16 (exact, but for values below 2^-133) */
int moe_dequantize_experts(moe_dims dims, const moe_qexperts *q, moe_bf16 *W1, moe_bf16 *W2, void *stream);

/*
 * The activations a forward keeps for the backward, in the 8-bit block format:
 * H (blocks of 128 columns within the gate and the up half: a row's scales are
 * its ceil(n/128) gate blocks, then its up blocks) and, with MOE_CKPT_X, X.  2 P n (+ T d)
 * bytes instead of 4 P n (+ 2 T d), held from the forward to the backward.  The
 * workspaces hold the other form of X all the same, whether or not a call uses it:
 * MOE_WS_BWD_CKPT is MOE_WS_BWD and 2 T d bytes, MOE_WS_FWD_QUANT has a q(X) of T d.
 * One caller-allocated device buffer, laid out by moe_ckpt_init, written by
 * moe_fwd_ckpt or moe_fwd_quant, read by moe_bwd_ckpt.
 */
typedef struct {
  int32_t T, d, n, capacity;
  int32_t state;   /* host-side, MOE_HELD_*                                    */
  int32_t reserved;
  moe_fp8 *H;      /* [capacity,2n]                                            */
  uint8_t *Hs;     /* [capacity][moe_scale_stride(256 * ceil(n/128))]          */
  moe_fp8 *X;      /* [T,d], null without MOE_CKPT_X                           */
  uint8_t *Xs;     /* [T][moe_scale_stride(d)]                                 */
} moe_ckpt;

enum { MOE_CKPT_X = 1 /* X is kept too, so that the backward needs no bf16 X */ };
/* capacity: of the routing that the calls use */
size_t moe_ckpt_bytes(moe_dims dims, int32_t capacity, int flags);
int moe_ckpt_init(moe_dims dims, int32_t capacity, int flags, void *buf, size_t bytes, moe_ckpt *c);

/*
 * Forward with 8-bit expert products: with q() the block format,
 *   H = gather(q(X)) q(W1_e) (+ b1_e);  A = SiLU(H_gate) * H_up
 *   Y = q(A) q(W2_e) (+ b2_e);          O_t = sum_{rows of t} s * Y
 * The block-scaled 8-bit matrix instruction sums a product to 1.3e-5 of its value (fp32 sums:
 * 1e-7); A is quantised from fp32 (blocks of 128 columns of a row); Y is rounded to bf16
 * before its weighted sum, as in moe_fwd.  For few rows and without c, Y stays in fp32 (T <=
 * 16, or a mean of up to 10 rows per expert, 16 where d >= 4096 and n <= 4096), and for fewer
 * the up-projection's codes are multiplied with fp32 sums (T <= 16, or a mean of up to 2).
 * O's error to this definition in 64 bits is 2.7e-3 of it, 2.1e-3 and 1.7e-3 in that order;
 * one rounding to bf16 alone is 1.7e-3.  With c the up-projection's sums are fp32 too, so that
 * the codes of H that a backward reads are the definition's but for a few in 10^6 (O: 2.4e-3).
 *   w    weights in state MOE_HELD_WRITTEN (otherwise MOE_ERR_INVALID_ARG), of the
 *        same d, n and E
 *   c    nullable: then nothing is kept for a backward.  Otherwise q(H) (and
 *        q(X)) are written and c->state becomes MOE_HELD_WRITTEN, for
 *        moe_bwd_ckpt (which see: an approximation of this forward's gradient)
 *   ws   moe_workspace_bytes(dims, r->capacity, MOE_WS_FWD_QUANT) bytes
 * Other arguments as moe_fwd.
 */
int moe_fwd_quant(moe_dims dims, const moe_bf16 *X, const moe_qexperts *w, const moe_expert_bias *eb,
                  const moe_routing *r, moe_ckpt *c, moe_bf16 *O, void *ws, size_t ws_bytes, void *stream);

/*
 * moe_fwd that keeps its activations in 8 bits: the same O (up to the order of
 * sums, where moe_fwd streams the weights past few rows); in the place of H, c
 * receives q(H) (from the fp32 H) and, with MOE_CKPT_X, q(X).
 *   ws   moe_workspace_bytes(dims, r->capacity, MOE_WS_FWD_CKPT) bytes
 */
int moe_fwd_ckpt(moe_dims dims, const moe_bf16 *X, const moe_bf16 *W1, const moe_bf16 *W2, const moe_expert_bias *eb,
                 const moe_routing *r, moe_ckpt *c, moe_bf16 *O, void *ws, size_t ws_bytes, void *stream);

/*
 * moe_bwd from an 8-bit checkpoint: the gradients of moe_bwd with the kept
 * values in the place of H and, where X is null, of X.  So W1, W2 and a given X
 * enter as they are, and A is SwiGLU of the kept H, without a rounding of its own.
 * After moe_fwd_ckpt that is the layer's backward but for the rounding of what is
 * kept.  After moe_fwd_quant it is the 16-bit layer's backward at that forward's
 * H, not the gradient of its 8-bit products: with every rounding passed straight
 * through, that has q(W1), q(W2), q(X) and q(A) in their place.  The two are 4 to
 * 5% of the gradients' norm apart, 7% for dWr (a code is up to 2^-4 of its value
 * off); with the weights of moe_dequantize_experts and the kept X 3 to 6%, the rest
 * being A's and H's roundings.
 *   c    checkpoint in state MOE_HELD_WRITTEN (otherwise MOE_ERR_INVALID_ARG), of
 *        the same T, d, n and capacity
 *   X    [T,d] bf16, or null to use the kept one (then c needs MOE_CKPT_X)
 *   ws   moe_workspace_bytes(dims, r->capacity, MOE_WS_BWD_CKPT) bytes
 */
int moe_bwd_ckpt(moe_dims dims, const moe_bf16 *dO, const moe_bf16 *X, const moe_ckpt *c, const moe_bf16 *W1,
                 const moe_bf16 *W2, const moe_expert_bias *eb, const moe_bf16 *Wr, const moe_routing *r, moe_bf16 *dX,
                 moe_bf16 *dW1, moe_bf16 *dW2, float *dWr, float *dbias, float *dS, void *ws, size_t ws_bytes,
                 void *stream);

/*
 * The whole layer for a few tokens in two launches: token-choice routing as moe_route's,
 * then the experts and the sum of moe_fwd, without a routing or an H.
 *   O = R + sum over t's K experts of s * (SwiGLU(X W1_e + b1_e) W2_e + b2_e)
 * A is rounded to bf16 between the products; H, Y and the sum are fp32, O is rounded once.
 *   dims  T at most MOE_DECODE_MAX_T, E at most 1024, an expert's W1 below 2^31 bytes
 *   bias  [E] fp32, of the router, nullable;  eb  b1 and b2 are read, nullable
 *   R     [T,d] bf16, what the layer's output is added to, nullable; may be O itself.
 *         O must not overlap X.
 *   topk_idx, topk_w   [T,K] out, nullable: the selection by (score descending, expert
 *         ascending) and its weights, as moe_route writes them
 *   ws    moe_workspace_bytes(dims, capacity, MOE_WS_DECODE) bytes.  Calls that share
 *         one must be ordered, like those of moe_fwd: of two at once the results are
 *         undefined (NaN where a wait for counts that the other took gave up), and either
 *         may take seconds; both end, and touch nothing but their operands.
 * moe_route and moe_fwd compute the same but for R.  Measured beside them, moe_decode takes up
 * to a quarter less time at n <= 3584 (at some sizes, mostly of 2 to 4 tokens, up to 8% more);
 * at n = 14336 one token, or 32 and more, take 9% more.
 */
enum { MOE_DECODE_MAX_T = 64 };
int moe_decode(moe_dims dims, const moe_bf16 *X, const moe_bf16 *Wr, const float *bias, const moe_bf16 *W1,
               const moe_bf16 *W2, const moe_expert_bias *eb, const moe_bf16 *R, moe_bf16 *O, int32_t *topk_idx,
               float *topk_w, void *ws, size_t ws_bytes, void *stream);

/*
 * The same with 8-bit expert products, as moe_fwd_quant's: H = q(X) q(W1_e) (+ b1_e), Y =
 * q(A) q(W2_e) (+ b2_e), A quantised from fp32.  The up-projection's codes are multiplied
 * with fp32 sums, so that A's codes are an fp32 form's but where a sum's order moves one.
 * moe_route and moe_fwd_quant compute the same but for R and those sums.  Beside them, one token
 * of n <= 2048 takes up to 3 us less; from two tokens on they are mostly the faster pair, by up
 * to 6 us where few experts are hit, up to 14% at 16 to 32 tokens of d = 4096, and more where n
 * is long: 64 tokens of d = 4096 take 104 us, not 127, at n = 3584, and 306, not 441, at n = 14336.
 *   q   weights in state MOE_HELD_WRITTEN, of the same d, n and E
 *   ws  moe_workspace_bytes(dims, capacity, MOE_WS_DECODE_QUANT) bytes
 */
int moe_decode_quant(moe_dims dims, const moe_bf16 *X, const moe_bf16 *Wr, const float *bias, const moe_qexperts *q,
                     const moe_expert_bias *eb, const moe_bf16 *R, moe_bf16 *O, int32_t *topk_idx, float *topk_w,
                     void *ws, size_t ws_bytes, void *stream);

/*
 * The dense matrix product with bias, activation and residual: what stands beside the
 * routed experts (a shared expert's projections, a dense layer), so that O = R +
 * shared(X) + experts(X) is three calls, the last adding to the one before.
 *   H = X W + b;   Y = act(H) + R
 * MOE_ACT_SWIGLU: W [k,2n], gate columns [0,n) and up columns [n,2n), as W1's, b and H
 * as wide; act(H) = SiLU(H_gate) * H_up.  MOE_ACT_GELU is the form with erf.
 */
enum { MOE_ACT_NONE = 0, MOE_ACT_RELU = 1, MOE_ACT_SILU = 2, MOE_ACT_GELU = 3, MOE_ACT_SWIGLU = 4 };

typedef struct {
  int32_t T;   /* rows, 1 to 2^28; no matrix has more than 2^37 elements      */
  int32_t k;   /* columns of X, a positive multiple of 8 below 2^24           */
  int32_t n;   /* columns of Y, a positive multiple of 8 below 2^24           */
  int32_t act; /* MOE_ACT_*                                                   */
  /* elements from a row to the next of X (and dX), of R, and of Y (and dY): multiples
   * of 8, at least the row's length, below 2^30; 0: the row's length */
  int32_t ldx, ldr, ldy;
} moe_linear;

enum { MOE_WS_LINEAR_FWD = 1, MOE_WS_LINEAR_BWD = 2 };
/* Workspace bytes of moe_linear_fwd or moe_linear_bwd, at least 256; 0 for an invalid l. */
size_t moe_linear_workspace_bytes(moe_linear l, int which);

/*
 *   X [T,k] bf16;  W [k,n] bf16 ([k,2n]: swiglu), contiguous
 *   b [n] fp32 ([2n]), nullable;  R [T,n] bf16, nullable; may be Y itself (with ldr = ldy)
 *   H [T,n] ([T,2n]) bf16 out, contiguous, nullable: the pre-activation for the backward
 *   Y [T,n] bf16 out: rounded once.  What lies between its rows is left as it was.
 * X, W, R, H, Y are 16-byte aligned, b too; outputs overlap no input but R = Y.
 */
int moe_linear_fwd(moe_linear l, const moe_bf16 *X, const moe_bf16 *W, const float *b, const moe_bf16 *R, moe_bf16 *H,
                   moe_bf16 *Y, void *ws, size_t ws_bytes, void *stream);

/*
 * The gradients at the kept H (dR is dY itself):
 *   dP = dY * act'(H);  dX = dP W^T + G;  dW = X^T dP;  db = column sums of dP
 * MOE_ACT_RELU: dP is dY where H > 0 and 0 elsewhere, whatever dY is there.
 *   dY [T,n] bf16, with ldy between rows;  H as written by moe_linear_fwd, null and not
 *      read with MOE_ACT_NONE
 *   G  [T,k] bf16, nullable: what reaches X by its other ways, with ldx between rows;
 *      may be dX itself
 *   dX [T,k], dW as W, bf16, db as b, fp32: out, each nullable (X only for dW, W only for dX)
 * dP is rounded to bf16 for the two products; db sums it before that, in a fixed order.
 */
int moe_linear_bwd(moe_linear l, const moe_bf16 *dY, const moe_bf16 *X, const moe_bf16 *W, const moe_bf16 *H,
                   const moe_bf16 *G, moe_bf16 *dX, moe_bf16 *dW, float *db, void *ws, size_t ws_bytes, void *stream);

/* Static description of an error code. */
const char *moe_strerror(int code);
/* Thread-local description of the last error returned on this thread. */
const char *moe_last_error(void);

/*
 * Kernel timing (measurement support).  moe_prof_select(k) brackets every
 * later launch of kernel class k with HIP events on the launch stream
 * (k = -1 disables); moe_prof_read() synchronises those events and returns the
 * summed milliseconds and the number of launches since the last reset.
 */
enum {
  MOE_KC_ROUTER_GEMM = 0, MOE_KC_TOPK, MOE_KC_META, MOE_KC_ROUND,
  MOE_KC_UP, MOE_KC_DOWN, MOE_KC_AGG_O,
  MOE_KC_DH, MOE_KC_DW2, MOE_KC_DXT, MOE_KC_DW1, MOE_KC_AGG_DX, MOE_KC_DWR,
  MOE_KC_ROUTER_TOPK, /* the router GEMM with fused softmax/top-K; for few tokens
                         (see moe_route) two launches, counted as one */
  MOE_KC_QUANTIZE, /* rows and weights into or out of the 8-bit block format (moe_fwd_quant: and its m-tile lists) */
  MOE_KC_UP_QUANT, MOE_KC_DOWN_QUANT, /* (two launches over a long n, counted as one; for few
                                          tokens with the aggregation in it) */
  MOE_KC_DECODE, /* moe_decode, moe_decode_quant: the two launches, counted as one */
  MOE_KC_LINEAR, MOE_KC_LINEAR_BWD, /* moe_linear_fwd, moe_linear_bwd: all launches of a call */
  MOE_KC_COUNT
};
int moe_prof_select(int kernel_class);
int moe_prof_read(double *ms, int32_t *launches);
const char *moe_kernel_class_name(int kernel_class);

#ifdef __cplusplus
}
#endif
#endif /* SONICMOE_H */

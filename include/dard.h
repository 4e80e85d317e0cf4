/*
 * dard.h - C ABI of the GB300 (sm_103a) DARD step library, libdard.so.
 *
 * DARD (Dependency-Aware Revocable Decoding, arXiv 2608.26574) adds two pieces of compute
 * to every denoising step of a diffusion LLM:
 *
 *   dard_step_attention        bidirectional softmax attention over the augmented sequence
 *                              x~_t = (x_t; s_t) under the state-specific mask of Sec. 3
 *                              (Eq. 2, Eq. 3 and query blocks 1-6 of Sec. 3.2), one layer;
 *   dard_score_and_transition  vocabulary-wide confidence and argmax (Eq. 1), verification
 *                              outcomes and guidance weights (Eq. 5, Eq. 6), logit mixing
 *                              (Eq. 7) and the three-state transition (Eq. 8), in the order
 *                              of Algorithm 1.
 *
 * Beside them: the MLP half of a layer with experts (dard_residual_norm .. dard_experts) and
 * decoding behind a shared prefix (dard_prefix_attention, _weights, _evict).
 *
 * Conventions shared by every entry point
 *   - Pointers named "device" are CUDA device memory owned by the caller; pointers named
 *     "host" are ordinary host memory owned by the caller and read during the call only.
 *   - Every call is asynchronous on the given stream; nothing is synchronised.
 *   - The library never allocates memory. Scratch space is passed in by the caller, or
 *     (dard_score_and_transition_noalloc) is a fixed array inside the library.
 *   - Argument and shape errors are detected on the host and returned before any launch;
 *     nothing is launched when a call returns an error. A failed launch returns
 *     DARD_ERR_CUDA (the CUDA error string is available from dard_last_error()).
 *   - Problems found only on the device (a state byte above 2, a shadow row that points
 *     outside its block, a row whose softmax normaliser is not finite) never trap: they set
 *     bits of the optional device status word (DARD_STATUS_*) and the affected outputs follow
 *     the documented fallback.
 *
 * Sequence layout (per sequence i of a ragged batch, everything stored back to back):
 *   rows      N_i original rows (prompt + full generation length, positions 0..N_i-1),
 *             then S_i shadow rows. Row N_i + k is the shadow copy s^j, j = shadow_src[k].
 *   block     positions [b0_i, b0_i + B_i) are the block being decoded. Positions before
 *             it are decoded context (state U); positions after it are still masked
 *             (state M) and have no shadow row.
 *   states    one byte per block position: 0 = M (masked), 1 = C (candidate),
 *             2 = U (unmasked), the three states of Sec. 3.2.
 */
#ifndef DARD_H_
#define DARD_H_

#include <stddef.h>
#include <stdint.h>

#ifdef __cplusplus
extern "C" {
#endif

typedef enum {
  DARD_OK = 0,
  DARD_ERR_NULL = 1,         /* a required pointer is NULL                              */
  DARD_ERR_SHAPE = 2,        /* inconsistent sizes / offsets                            */
  DARD_ERR_VALUE = 3,        /* a parameter out of its range (tau, lambda, p0, scale)   */
  DARD_ERR_UNSUPPORTED = 4,  /* valid but not implemented (e.g. head_dim not 64 or 128) */
  DARD_ERR_CUDA = 5,         /* a CUDA runtime call failed                              */
  DARD_ERR_ALIGN = 6,        /* a pointer or stride breaks the alignment rule           */
  DARD_ERR_WORKSPACE = 7     /* workspace missing or smaller than required              */
} dard_status;

typedef enum { DARD_F32 = 0, DARD_BF16 = 1 } dard_dtype;

/* Orderings of candidate tokens in the mask (Eq. 3 compares one key per block position).
 * The attention-mask ablation of Sec. 5 compares DARD's confidence ordering with a
 * bidirectional mask and with left-to-right, entropy and margin orderings; each is a choice
 * of key, which the scoring call can write for the next step (dard_score_args.order_key):
 *   CONFIDENCE  c_t (the paper's DARD)          BIDIR   0 (equal keys: every C pair attends
 *   L2R         minus the block position          both ways, Eq. 3 ties being mutual)
 *   ENTROPY     minus the entropy (nats)        MARGIN  p(x^) minus the second probability */
typedef enum {
  DARD_ORDER_CONFIDENCE = 0,
  DARD_ORDER_BIDIR = 1,
  DARD_ORDER_L2R = 2,
  DARD_ORDER_ENTROPY = 3,
  DARD_ORDER_MARGIN = 4
} dard_order_mode;

/* Bits of the optional device status word (OR-ed in, never cleared by the library). */
#define DARD_STATUS_BAD_STATE 0x1u     /* a state byte > 2 (treated as M)                    */
#define DARD_STATUS_BAD_SHADOW 0x2u    /* shadow_src outside its block or repeated (row
                                          treated as a masked-out key and left unwritten)    */
#define DARD_STATUS_INVALID_ROW 0x4u   /* softmax normaliser not finite or zero (NaN, +inf or
                                          all -inf logits): conf 0, token -1, state M        */
#define DARD_STATUS_TIMEOUT 0x8u       /* a bounded in-kernel wait gave up (the launch's
                                          outputs are incomplete)                             */

#define DARD_MAX_SEQS 256       /* sequences per call                                     */
#define DARD_MAX_BLOCK 128      /* block length B_i                                       */

/* ------------------------------------------------------------------------------------- *
 * Masked attention (Sec. 3.1 Eq. 2; Sec. 3.2 query blocks 1-6 and Eq. 3).
 *
 * For every sequence, head h and row r:
 *     O[r,h,:] = sum_j softmax_j(scale * <Q[r,h,:], K[key(r,j),g,:]>) V[key(r,j),g,:]
 * where j runs over the N_i original positions, key(r,j) is the row of x^j or of s^j as
 * the mask selects (exactly one per position, Eq. 2), and g = h / (hq / hkv) (grouped-query
 * heads share a key/value head). The mask is built inside the kernel from the state vector
 * and prev_conf; no L x L tensor exists anywhere. Selection rule (q = query copy):
 *   key j state U : x^j, except a shadow query s^i takes s^i for j = i;
 *   key j state M : x^j for original queries of M positions, s^j for every other query;
 *   key j state C : original query of an M position       -> x^j
 *                   query of a C position i (x or s)      -> x^j if c_i <= c_j, else s^j
 *                                                            (a shadow query takes s^i at j=i)
 *                   query of a U position, or s^i of an M -> s^j
 *   and x^j whenever j has no shadow row (positions outside the block, or a block position
 *   the caller gave no shadow row). Out-of-block queries are original queries of U (before
 *   the block) or M (after it) positions.
 * Arithmetic: bf16 operands on the tcgen05 tensor cores with fp32 accumulation and an fp32
 * online softmax (dtype BF16); fp32 CUDA cores throughout (dtype F32).
 * ------------------------------------------------------------------------------------- */
typedef struct {
  const void* q;             /* device [total_rows, hq,  head_dim] row-major              */
  const void* k;             /* device [total_rows, hkv, head_dim]                        */
  const void* v;             /* device [total_rows, hkv, head_dim]                        */
  void* o;                   /* device [total_rows, hq,  head_dim], same dtype as q       */
  int32_t dtype;             /* dard_dtype of q, k, v and o                                */
  int32_t hq, hkv;           /* query heads, key/value heads; hq % hkv == 0                */
  int32_t head_dim;          /* 64 or 128                                                  */
  int32_t num_seqs;          /* 1 .. DARD_MAX_SEQS                                         */
  const int32_t* n_orig;     /* host [num_seqs] N_i >= 1                                   */
  const int32_t* block_start;/* host [num_seqs] b0_i, 0 <= b0_i, b0_i + B_i <= N_i         */
  const int32_t* block_len;  /* host [num_seqs] B_i in 0 .. DARD_MAX_BLOCK                 */
  const int32_t* shadow_len; /* host [num_seqs] S_i in 0 .. B_i                            */
  const uint8_t* state;      /* device [sum B_i] states of block positions, seq by seq     */
  const float* prev_conf;    /* device [sum B_i] c_{t-1} of block positions (Eq. 3 order)  */
  const int32_t* shadow_src; /* device [sum S_i] original position of each shadow row,
                                in [b0_i, b0_i + B_i), distinct within a sequence          */
  float scale;               /* softmax scale; 0 means 1/sqrt(head_dim)                    */
  uint32_t* status;          /* optional device word, DARD_STATUS_* bits OR-ed in          */
  const int32_t* query_start;/* optional host [num_seqs] q_i in 0 .. N_i + S_i: only rows
                                q_i .. N_i + S_i - 1 of sequence i are queries (prefix
                                caching: the prompt's outputs are not recomputed, its
                                K/V rows still serve as keys); rows before q_i of o are
                                left untouched. NULL means 0 for every sequence.           */
  /* Rotary position embedding inside the call (Sec. 3.1: x^i and s^i share the positional
   * embedding of position i). rope_theta = 0: q and k already carry their positions (no
   * rotation here, k_rope unused). rope_theta >= 1: q and k arrive before RoPE and the call
   * rotates them, original row r of a sequence at position r and shadow row N_i + k at
   * position shadow_src[k]; see "RoPE" below. */
  float rope_theta;          /* 0, or the RoPE base theta >= 1                             */
  int32_t rope_style;        /* dard_rope_style: which elements form a rotated pair        */
  void* k_rope;              /* device [total_rows, hkv, head_dim], dtype: receives k after
                                RoPE, the keys the attention reads (a key cache may take
                                it); may be k itself (rotated in place). Required when
                                rope_theta > 0, 16-byte aligned.                           */
} dard_attn_args;

/* RoPE (rotary position embedding, Su et al., RoFormer, 2021) as dard_step_attention applies
 * it when rope_theta > 0. For head dimension D and frequency index i in 0 .. D/2 - 1 the
 * pair (a, b) of a row at position p is replaced by
 *     (a cos(p f_i) - b sin(p f_i),  a sin(p f_i) + b cos(p f_i)),   f_i = theta^(-2i/D),
 * in every head of q and of k. DARD_ROPE_INTERLEAVED pairs elements (2i, 2i + 1);
 * DARD_ROPE_HALF pairs (i, i + D/2). The call first rotates k into k_rope (one pass over the
 * key rows, launched on the stream ahead of the attention kernel, which waits for it with
 * programmatic dependent launch), then the attention kernel rotates each query tile as it
 * loads it; the rotated q is not written out. Arithmetic: the angle p f_i is carried in two
 * floats (f_i split into a float and its remainder), reduced modulo 2 pi with a two-constant
 * additive (Cody-Waite) split of 2 pi, and its cosine and sine taken by the hardware
 * approximations on the reduced angle (absolute error near 1e-6 in all); rotated values are
 * rounded to dtype. Every N_i must be at most 2^20 (DARD_ERR_SHAPE). A shadow row whose
 * shadow_src is invalid (DARD_STATUS_BAD_SHADOW) is rotated by an unspecified angle; it is a
 * masked-out key and an unwritten query row anyway. */
typedef enum { DARD_ROPE_INTERLEAVED = 0, DARD_ROPE_HALF = 1 } dard_rope_style;
#define DARD_ROPE_MAX_POSITIONS (1 << 20)

/* Rows are total_rows = sum_i (N_i + S_i). q, k, v, o must be 16-byte aligned; with dtype
 * BF16 a tensor-core kernel runs (head_dim 64 or 128), with F32 the CUDA-core kernel.
 * Of the two tensor-core kernels (one or two 128-row query tiles per CTA) the library
 * picks the one a cost model of the batch (query tiles, key tiles, SM count) predicts to be
 * faster; the environment variable DARD_ATTN_TC=1 or 2 forces one of them (results agree
 * within rounding).
 * Errors: DARD_ERR_NULL (also: k_rope NULL with rope_theta > 0), _SHAPE, _VALUE (scale < 0
 * or not finite; rope_theta neither 0 nor a finite value >= 1; rope_style not a
 * dard_rope_style), _UNSUPPORTED, _ALIGN, _CUDA. */
dard_status dard_step_attention(const dard_attn_args* args, void* stream /* cudaStream_t */);

/* The attention kernel dard_step_attention would launch for these arguments, without
 * launching anything: *kernel = 1 or 2 (the tensor-core kernel with one or two 128-row
 * query tiles per CTA, as the cost model or DARD_ATTN_TC picks), 4 (the kernel on CTA
 * pairs, head_dim 128, chosen only by DARD_ATTN_TC=4), 3 (the fp32 CUDA-core kernel), or 0
 * (no query rows, no launch). The arguments go through the same host
 * validation as dard_step_attention and fail with the same codes; device pointers are
 * checked but never read. The cost model uses the current device's SM count (148 when no
 * device is visible, so that the choice can be planned on a host without one). An
 * interface addition: the paper has no counterpart. */
dard_status dard_attention_kernel(const dard_attn_args* args, int32_t* kernel);

/* The launch plan of dard_step_attention for these arguments, computed on the host without
 * launching anything (an interface addition: the paper has no counterpart). The arguments
 * go through the same host validation as dard_step_attention and fail with the same codes.
 *   kernel              as dard_attention_kernel (0: no query rows, nothing launched)
 *   ctas                CTAs of the launch (the CTA-pair kernel: two per cluster, as many
 *                       clusters as fit on the current device, or SMs / 2 without one)
 *   tile_pairs          (query tile, key tile) pairs a tensor-core kernel computes: 128 query
 *                       rows of one head against 128 key rows, over every head and sequence
 *   tile_pairs_skipped  pairs it leaves out because no query of the rows a CTA (or CTA pair)
 *                       handles attends any key of the tile: tiles holding only shadow keys,
 *                       for rows that are all original queries of positions after the block
 *                       (Sec. 3.2, query block 1 attends x copies only). The fp32 kernel,
 *                       which masks key by key, reports 0 for both.                         */
typedef struct {
  int32_t kernel;
  int64_t ctas;
  int64_t tile_pairs;
  int64_t tile_pairs_skipped;
} dard_attn_plan;
dard_status dard_attention_plan(const dard_attn_args* args, dard_attn_plan* plan);

/* ------------------------------------------------------------------------------------- *
 * Confidence scoring and state transition (Eq. 1, Eq. 5-8, Algorithm 1).
 *
 * Rows are the block positions of all sequences, seq by seq (sum B_i rows). For row i of a
 * sequence with incoming state s_i:
 *   s_i in {C, U}: (c_i, x^_i) = (max softmax, argmax) of logits_s row i          (Eq. 1)
 *   then every C row that moves to U joins P, every C row that moves to M joins D (Eq. 8);
 *   s_i = M: P_i = sum_{j in P} lambda^|i-j|, D_i likewise over D                  (Eq. 5)
 *            w_i = (P_i + p0) / (P_i + D_i + p0)                                  (Eq. 6)
 *            mix = ls + w_i (lx - ls), each operation rounded to fp32              (Eq. 7)
 *            (c_i, x^_i) = (max softmax, argmax) of mix
 *   new state: c <= tau_c -> M, c <= tau_u -> C, else U                            (Eq. 8)
 * Argmax ties go to the lowest index. Softmax sums and w accumulate in fp32 (the terms
 * lambda^k as 2^(k log2 lambda)); w then enters Eq. 7 as an fp32 value.
 * Invalid rows (normaliser not finite or 0): conf 0, token -1, state M, status bit.
 * ------------------------------------------------------------------------------------- */
typedef struct {
  const void* logits_x;      /* device [rows, row_stride] logits of the original copies   */
  const void* logits_s;      /* device [rows, row_stride] logits of the shadow copies     */
  int32_t dtype;             /* dard_dtype of both logit tensors                           */
  int32_t vocab;             /* V >= 1                                                     */
  int64_t row_stride;        /* elements between consecutive rows, >= vocab               */
  int32_t num_seqs;          /* 1 .. DARD_MAX_SEQS                                         */
  const int32_t* block_len;  /* host [num_seqs] B_i in 0 .. DARD_MAX_BLOCK                 */
  const uint8_t* state_in;   /* device [rows] incoming states                              */
  float tau_c, tau_u;        /* 0 <= tau_c <= tau_u <= 1                                   */
  float lambda;              /* 0 < lambda < 1 (paper: 0.5^(1/8))                          */
  float p0;                  /* p0 > 0 (paper: 0.1)                                        */
  float* conf;               /* device [rows] out: c_t                                     */
  int32_t* token;            /* device [rows] out: x^_t (or -1 for an invalid row)         */
  uint8_t* state_out;        /* device [rows] out: state after Eq. 8                       */
  float* w_out;              /* optional device [rows] out: w for M rows, NaN otherwise    */
  int32_t* counts;           /* optional device [num_seqs * 3] out: M, C, U counts         */
  uint32_t* status;          /* optional device word, DARD_STATUS_* bits OR-ed in          */
  void* workspace;           /* device scratch of dard_score_workspace_size() bytes: three
                                counters per sequence, then two bytes per block row (each
                                C row's promotion / demotion outcome, each row's new
                                state). Fill it with zeros before its first use; every
                                call leaves the counters at zero again, except a call that
                                sets DARD_STATUS_TIMEOUT, after which it must be zeroed
                                again. Calls that overlap on the GPU need separate
                                workspaces.                                                */
  size_t workspace_bytes;
  /* Optional, the end of a step (each may be NULL):                                       */
  const int32_t* cur_token;  /* device [rows] the token currently at each block position   */
  float* p_cur;              /* device [rows] out: the probability the scored distribution
                                (shadow logits for C/U rows, mixed logits for M rows) gives
                                to cur_token; 0 for a token outside [0, vocab) or an invalid
                                row. Needs cur_token.                                      */
  int32_t* tokens;           /* device [rows] out: the next step's tokens, as the last line
                                of Algorithm 1's step fills them: x^ where the new state is
                                C or U, mask_token where it is M                           */
  int32_t mask_token;        /* the mask token id written by `tokens`                      */
  float* entropy;            /* device [rows] out: entropy (nats) of the scored
                                distribution; 0 for an invalid row                         */
  float* margin;             /* device [rows] out: p(x^) minus the second-largest
                                probability (a repeated maximum gives 0); 0 if invalid     */
  float* order_key;          /* device [rows] out: the next step's ordering key, to pass as
                                dard_attn_args.prev_conf, per order_mode                   */
  int32_t order_mode;        /* dard_order_mode of order_key                               */
} dard_score_args;

/* In place: state_out may be the state_in buffer (the next step's states replace this
 * step's), and conf can serve directly as the next step's prev_conf of dard_step_attention;
 * tokens may be the buffer cur_token points to. */

/* Bytes of workspace a call with these sizes needs (0 on invalid sizes). */
size_t dard_score_workspace_size(int32_t rows, int32_t vocab, int32_t num_seqs);

/* Logits pointers must be 16-byte aligned and row_stride * element size a multiple of 16.
 * Two launches (C and U rows, then M rows: Algorithm 1's order), the second a programmatic
 * dependent of the first. DARD_SCORE_PATH=fused selects one launch instead, whose M rows
 * wait (bounded) for their block's C rows of the same launch, when every row's group of
 * CTAs fits on the device at once. Errors: DARD_ERR_NULL, _SHAPE, _VALUE, _ALIGN,
 * _WORKSPACE, _CUDA. */
dard_status dard_score_and_transition(const dard_score_args* args, void* stream);

/* ------------------------------------------------------------------------------------- *
 * dard_score_and_transition_noalloc: the same scoring and transition, with the scratch
 * inside the library. The paper has no counterpart: this is an interface addition.
 *
 * Who needs it: a caller that only holds the buffers another component handed to it (a
 * plug-in inside an inference server, a C host program driving a model it did not load)
 * and has no device allocator, or one whose device memory is planned in advance so that no
 * call may ask for more. Such a caller cannot provide `workspace`; this entry point needs
 * none and neither allocates nor frees device memory.
 *
 * Arguments, outputs and errors are those of dard_score_and_transition, except that
 * `workspace` and `workspace_bytes` are ignored. The scratch is a fixed array in the
 * library's device memory sized for DARD_SCORE_NOALLOC_MAX_ROWS block rows and DARD_MAX_SEQS
 * sequences (the workspace layout of dard_score_and_transition). A call with more block
 * rows (sum of block_len) than that returns DARD_ERR_WORKSPACE before any launch; use
 * dard_score_and_transition with a workspace for it. Each call clears the array's counters
 * on its stream (cudaMemsetAsync, which allocates nothing) before the kernels run, so no
 * call depends on what an earlier one left.
 *
 * The first call on each device (the device current at the call) looks up the array's
 * address there (cudaGetSymbolAddress) and caches it with the current context; a later call
 * in another context of the device (after a device reset, say) looks it up again. Make the
 * first call in a context before any stream capture there. A failed lookup returns
 * DARD_ERR_CUDA.
 *
 * There is one array per device, shared by every call on it: calls whose kernels can
 * overlap on one device (different streams, different host threads) race on it and may
 * return wrong results. Order them (one stream, or events between streams).
 * ------------------------------------------------------------------------------------- */
#define DARD_SCORE_NOALLOC_MAX_ROWS 8192
dard_status dard_score_and_transition_noalloc(const dard_score_args* args, void* stream);

/* ------------------------------------------------------------------------------------- *
 * The MLP half of a layer with experts, in microscaled 8-bit floating point (MXFP8). The
 * paper has no counterpart: these are interface additions, for models whose MLP is a mixture
 * of experts (a dense MLP is the case of one expert). In a layer's order:
 *
 *   dard_residual_norm   residual addition, root-mean-square norm, optional MXFP8 output
 *   dard_mx_quantize     the MXFP8 rounding alone (weights, other activations)
 *   dard_route           router scores -> experts and weights of each token, and the plan
 *   dard_experts         the experts' products and the weighted sum over a token's experts
 *
 * MXFP8: e4m3 codes, one byte each, with one scale byte for each 32 consecutive elements of
 * a row. The scale byte b stands for 2^(b - 127) (e8m0). Rounding: b is the smallest for which
 * max|v| 2^(127 - b) <= 448 (the largest e4m3 value) over the 32 values, at least 0; a code
 * is v 2^(127 - b) rounded to the nearest e4m3 value, ties to even. A block that holds a NaN
 * or an infinity gets the scale byte 255 and NaN codes, so that what is computed from it is
 * NaN. Row lengths are multiples of 32.
 *
 * Scale layouts of a [rows, cols] matrix:
 *   DARD_MX_SCALE_ROWS   row-major bytes [rows, pitch], pitch a multiple of 16, at least
 *                        cols / 32; the bytes after cols / 32 are not written or used.
 *   DARD_MX_SCALE_TILES  tiles of 128 rows x 4 scales, 512 bytes each, in the layout that the
 *                        tensor core's scale copies take: tile (r / 128, c / 4) of
 *                        [ceil(rows / 128), ceil(cols / 128)] tiles, and in it row r, scale c
 *                        at byte (r % 32) * 16 + (r % 128) / 32 * 4 + c % 4. Bytes without an
 *                        element are 0. A batch of matrices stores each matrix's tiles in turn.
 * ------------------------------------------------------------------------------------- */
typedef enum { DARD_MX_SCALE_ROWS = 0, DARD_MX_SCALE_TILES = 1 } dard_mx_scale_layout;

/* Residual addition and root-mean-square norm of `rows` rows of `dim` elements:
 *     r = round(x + delta)                  (round: to dtype; r = x without delta)
 *     n = r / sqrt(mean(r^2) + eps) * weight
 *     residual = r,  y = round(n),  (y8, y8_scale) = MXFP8(n)
 * Sums and n are fp32; n enters the MXFP8 rounding unrounded. A row with a NaN is NaN
 * throughout; a row with an infinity is NaN there and 0 elsewhere. Strides are in elements.
 * Rows whose pointers, strides and dim are multiples of 16 bytes (y8: 8 bytes) take 16-byte
 * accesses, others element accesses. */
typedef struct {
  const void* x;             /* device [rows, dim], row stride x_stride                    */
  const void* delta;         /* optional device [rows, dim]                                */
  const void* weight;        /* optional device [dim], dtype; NULL means 1                 */
  void* residual;            /* optional device [rows, dim] out: r; may be x or delta      */
  void* y;                   /* optional device [rows, dim] out; may be x or delta         */
  uint8_t* y8;               /* optional device [rows, dim] out: e4m3 codes                */
  uint8_t* y8_scale;         /* device [rows, y8_scale_stride] out, required with y8       */
  int32_t dtype;             /* dard_dtype of x, delta, weight, residual and y             */
  int32_t dim;               /* 1 .. DARD_NORM_MAX_DIM; a multiple of 32 with y8           */
  int64_t rows;              /* 0 .. 2^31 - 1                                              */
  int64_t x_stride, delta_stride, residual_stride, y_stride, y8_stride, y8_scale_stride;
  float eps;                 /* >= 0, finite                                               */
} dard_norm_args;
#define DARD_NORM_MAX_DIM 32768

/* residual and y must be different buffers. One launch. Errors: DARD_ERR_NULL (x, every output
 * NULL, or y8 without y8_scale), _SHAPE (rows < 0, dim, a stride below dim), _VALUE (dtype,
 * eps), _ALIGN (x, delta, weight, residual or y not a multiple of the element size;
 * y8_scale_stride no multiple of 16, y8_scale not 16-byte aligned), _CUDA. */
dard_status dard_residual_norm(const dard_norm_args* args, void* stream);

/* The MXFP8 rounding of a batch of matrices. One launch (two where the tile layout has bytes
 * without an element). */
typedef struct {
  const void* x;             /* device [batch, rows, cols]                                 */
  uint8_t* codes;            /* device [batch, rows, cols] out, contiguous                 */
  uint8_t* scales;           /* device out: layout ROWS [batch * rows, scale_stride],
                                layout TILES [batch, ceil(rows/128), ceil(cols/128), 512]  */
  int32_t dtype;             /* dard_dtype of x                                            */
  int32_t layout;            /* dard_mx_scale_layout                                       */
  int32_t batch, cols;       /* batch >= 0; cols a positive multiple of 32; 2^40 elements  */
  int64_t rows;              /* of each matrix, >= 0                                       */
  int64_t x_row_stride, x_batch_stride;  /* elements                                       */
  int64_t scale_stride;      /* layout ROWS only: a multiple of 16, >= cols / 32           */
} dard_mx_args;

/* Errors: DARD_ERR_NULL, _SHAPE, _VALUE (dtype, layout), _ALIGN (x no multiple of the element
 * size; codes or scales not 16-byte aligned; scale_stride no multiple of 16), _CUDA. */
dard_status dard_mx_quantize(const dard_mx_args* args, void* stream);

/* Routing of tokens to experts. Per token, from its E logits l:
 *     score     SOFTMAX: softmax(l);  SIGMOID: 1 / (1 + exp(-l))
 *     choice    score + bias (bias: balances the experts' load; it enters the choice only)
 *     groups    E experts in `groups` runs of E / groups; with top_groups < groups a group's
 *               rank is the sum of its two largest choices (its only one if it has one
 *               expert), and only the top_groups best groups stay
 *     ids       the top_k largest choices left, in falling order
 *     weights   their scores; with renormalise divided by their sum (0 if the sum is 0);
 *               times `scale`
 * Ties go to the lowest group or expert. A logit of -inf switches its expert off for the token:
 * it is never chosen (and counts as -inf in its group's rank). Slots for which no expert is
 * left get id -1 and weight 0. A token with a NaN or +inf logit is invalid: every id -1,
 * every weight 0, and DARD_STATUS_INVALID_ROW in the status word. Arithmetic is fp32.
 *
 * The plan (optional): the (token, slot) pairs token * top_k + slot sorted by expert, pairs of
 * one expert in rising order. offsets[e] .. offsets[e + 1] are expert e's entries of `rows`;
 * entries from offsets[experts] on (slots without an expert) are -1. It stays on the device:
 * dard_experts reads it there, with no host round trip. */
typedef enum { DARD_ROUTE_SOFTMAX = 0, DARD_ROUTE_SIGMOID = 1 } dard_route_scoring;
#define DARD_MAX_EXPERTS 512
#define DARD_MAX_TOP_K 32
#define DARD_MAX_GROUPS 32
typedef struct {
  const void* logits;        /* device [tokens, experts], row stride logits_stride         */
  int64_t logits_stride;     /* elements, >= experts                                       */
  const float* bias;         /* optional device [experts], finite                          */
  int32_t dtype;             /* dard_dtype of logits                                       */
  int32_t scoring;           /* dard_route_scoring                                         */
  int32_t tokens;            /* >= 0; tokens * top_k at most 2^31 - 1                      */
  int32_t experts;           /* 1 .. DARD_MAX_EXPERTS                                      */
  int32_t top_k;             /* 1 .. min(experts, DARD_MAX_TOP_K)                          */
  int32_t groups;            /* 1 .. DARD_MAX_GROUPS, divides experts                      */
  int32_t top_groups;        /* 1 .. groups                                                */
  int32_t renormalise;       /* 0 or 1                                                     */
  float scale;               /* finite                                                     */
  int32_t* ids;              /* device [tokens, top_k] out                                 */
  float* weights;            /* device [tokens, top_k] out                                 */
  int32_t* offsets;          /* optional device [experts + 1] out                          */
  int32_t* rows;             /* device [tokens * top_k] out, required with offsets         */
  uint32_t* status;          /* optional device word, DARD_STATUS_* bits OR-ed in          */
  void* workspace;           /* device scratch of dard_route_workspace_size() bytes, 16-byte
                                aligned (with offsets); needs no preparation. Calls that
                                overlap on the GPU need separate workspaces.               */
  size_t workspace_bytes;
} dard_route_args;

/* Bytes of workspace for a call with these sizes or fewer tokens (0 where none is needed, or on
 * invalid sizes). */
size_t dard_route_workspace_size(int32_t tokens, int32_t experts, int32_t top_k);

/* One launch for few tokens or without the plan, else two. Errors: DARD_ERR_NULL, _SHAPE,
 * _VALUE, _ALIGN (logits no multiple of the element size), _WORKSPACE, _CUDA. */
dard_status dard_route(const dard_route_args* args, void* stream);

/* The experts' products. For token t and slot s with expert e = ids[t, s] >= 0:
 *     h = silu(w1[e] x_t) * (w3[e] x_t)       silu(g) = g / (1 + exp(-g))
 *     o = w2[e] MXFP8(h)                      (dtype BF16: w2[e] round(h))
 *     y_t = sum_s weights[t, s] o             (slots with id -1 add nothing)
 * x and the weights are MXFP8 (dtype DARD_MXFP8: e4m3 codes, x_scale by rows, weight scales
 * in tiles) or bf16 (dtype DARD_BF16, the scales unused). Products and sums are fp32 on the
 * tcgen05 tensor cores; the block scales are applied by the matrix instruction. The products of
 * one token's experts are added in slot order, so that equal calls give equal bits.
 * ids, weights, offsets and rows are what dard_route writes, or a caller's own of that form (in
 * which a token may name an expert in several slots). */
#define DARD_MXFP8 2         /* a dtype of dard_experts_args only                          */
typedef struct {
  const void* x;             /* device [tokens, dim], row stride x_stride                  */
  const uint8_t* x_scale;    /* device [tokens, x_scale_stride]                            */
  const void* w1;            /* device [experts, hidden, dim]: the gate                    */
  const void* w3;            /* device [experts, hidden, dim]: the value the gate scales   */
  const void* w2;            /* device [experts, dim, hidden]                              */
  const uint8_t* w1_scale;   /* device, layout TILES of [experts] matrices                 */
  const uint8_t* w3_scale;
  const uint8_t* w2_scale;
  const int32_t* ids;        /* device [tokens, top_k]                                     */
  const float* weights;      /* device [tokens, top_k]                                     */
  const int32_t* offsets;    /* device [experts + 1]                                       */
  const int32_t* rows;       /* device [tokens * top_k]                                    */
  void* y;                   /* device [tokens, dim] out, row stride y_stride              */
  int64_t x_stride, x_scale_stride, y_stride;   /* elements                                */
  int32_t dtype;             /* DARD_MXFP8 or DARD_BF16                                    */
  int32_t y_dtype;           /* dard_dtype of y                                            */
  int32_t tokens;            /* >= 0; tokens * top_k at most 2^24                          */
  int32_t experts;           /* 1 .. DARD_MAX_EXPERTS                                      */
  int32_t top_k;             /* 1 .. min(experts, DARD_MAX_TOP_K)                          */
  int32_t dim, hidden;       /* multiples of 32, at most DARD_EXPERTS_MAX_DIM              */
  void* workspace;           /* device scratch of dard_experts_workspace_size() bytes, 256-byte
                                aligned; needs no preparation. Calls that overlap on the GPU
                                need separate workspaces.                                  */
  size_t workspace_bytes;
  uint32_t* status;          /* optional device word: DARD_STATUS_TIMEOUT                  */
} dard_experts_args;
#define DARD_EXPERTS_MAX_DIM 65536

/* Bytes of workspace for these sizes or fewer tokens and either dtype (0 on invalid sizes): x in
 * the plan's order, the product in between, and the products of each (token, slot) pair before
 * their sum. */
size_t dard_experts_workspace_size(int32_t tokens, int32_t experts, int32_t top_k, int32_t dim,
                                   int32_t hidden);

/* Two to four launches, chained by programmatic dependent launch. x, the weights and their scales
 * must be 16-byte aligned, with x_stride and x_scale_stride multiples of 16 bytes; y and
 * y_stride multiples of 16 bytes. Entries of rows outside [0, tokens * top_k) are skipped.
 * Errors: DARD_ERR_NULL, _SHAPE, _VALUE (dtype), _ALIGN, _WORKSPACE, _CUDA. */
dard_status dard_experts(const dard_experts_args* args, void* stream);

/* ------------------------------------------------------------------------------------- *
 * Decoding behind a shared prefix. The paper has no counterpart: these are interface additions,
 * for batches whose sequences all follow one prefix (a system prompt, an image, a document)
 * whose keys and values are kept in a cache, once for all:
 *
 *   dard_prefix_attention  a step's attention over the prefix and each sequence's own rows
 *   dard_prefix_weights    the attention weight that each key of the prefix has received
 *   dard_prefix_evict      the keys to keep by that weight, moved together
 *
 * The cache of a layer: prefix_k and prefix_v, prefix_len rows of hkv heads of head_dim elements;
 * row r of head g starts at element r * prefix_row_stride + g * prefix_head_stride (so that
 * [rows, hkv, head_dim], [hkv, rows, head_dim] and slices of wider buffers all serve). Keys carry
 * their positions (RoPE applied); after an eviction the heads hold different positions.
 * Pointers are 16-byte aligned, strides multiples of 16 bytes and positive.
 * ------------------------------------------------------------------------------------- */

/* For every query row r of sequence i and head h, with c the scale and g = h / (hq / hkv):
 *     z_j  = c <q[r,h], prefix_k[j,g]>   for every row j of the prefix
 *     z'_j = c <q[r,h], k[key(r,j),g]>   for every position j of the sequence's own rows, the
 *                                        copy key(r,j) chosen as in dard_step_attention
 *     lse[r,h] = log(sum_j exp(z_j) + sum_j exp(z'_j))
 *     o[r,h]   = sum_j exp(z_j - lse) prefix_v[j,g] + sum_j exp(z'_j - lse) v[key(r,j),g]
 * The query rows of all sequences, times the heads that share a key/value head, are one run of
 * queries against the prefix, so that the prefix is read once for many sequences of few rows;
 * where there are few queries the keys are split over the SMs and the parts joined.
 * A key that a row does not see (the other copy of a position, another sequence's rows) does not
 * enter its output, whatever it holds; a NaN or an infinity in a key or value that a row sees does.
 * Rows that are no query rows (before query_start, and shadow rows with an invalid shadow_src) are
 * left as they were in o and in lse.
 * Arithmetic: as dard_step_attention (probabilities rounded to bf16 for the product with the
 * values when dtype is BF16, and divided by the sum of the rounded ones; the normaliser in lse is
 * that of the unrounded ones). */
typedef struct {
  dard_attn_args own;        /* the sequences' own rows, as dard_step_attention takes them;
                                rope_theta must be 0 (q and k carry their positions)       */
  const void* prefix_k;      /* device, dtype of own; not read when prefix_len is 0        */
  const void* prefix_v;
  int64_t prefix_row_stride, prefix_head_stride;  /* elements, of both                     */
  int32_t prefix_len;        /* 0 .. DARD_PREFIX_MAX_LEN                                   */
  float* lse;                /* optional device [total_rows, hq] out                       */
  void* workspace;           /* optional device scratch of
                                dard_prefix_attention_workspace_size() bytes, 16-byte aligned;
                                needs no preparation. Without it the keys are not split.
                                Calls that overlap on the GPU need separate workspaces.    */
  size_t workspace_bytes;
} dard_prefix_attn_args;
#define DARD_PREFIX_MAX_LEN (1 << 30)

/* Bytes of workspace for these sizes or smaller ones, any dtype and batch (0 on invalid sizes). */
size_t dard_prefix_attention_workspace_size(int32_t total_rows, int32_t hq, int32_t hkv,
                                            int32_t head_dim, int32_t prefix_len);

/* One launch, or two where the keys are split. Errors: DARD_ERR_NULL, _SHAPE, _VALUE (as
 * dard_step_attention; rope_theta not 0), _UNSUPPORTED, _ALIGN, _WORKSPACE (smaller than
 * needed), _CUDA. */
dard_status dard_prefix_attention(const dard_prefix_attn_args* args, void* stream);

/* The attention weight that the keys of the prefix have received, per key/value head g and key j:
 *     weights[g,j] = decay * weights_in[g,j] + sum_{r, h of group g} exp(c <q[r,h], prefix_k[j,g]>
 *                                                                       - lse[r,h])
 * over every row r of q (lse as dard_prefix_attention writes it). A row whose lse is +inf adds
 * nothing, whatever its q holds: fill lse with +inf once, and rows that are no queries stay out.
 * Without weights_in the first term is 0. Sums are fp32 in a fixed order: equal calls give equal
 * bits. */
typedef struct {
  const void* q;             /* device [rows, hq, head_dim], contiguous                    */
  const float* lse;          /* device [rows, hq], contiguous                              */
  const void* prefix_k;      /* device, dtype of q                                         */
  const float* weights_in;   /* optional device [hkv, prefix_len]; weights itself, or apart
                                from it                                                    */
  float* weights;            /* device [hkv, prefix_len] out                               */
  int64_t prefix_row_stride, prefix_head_stride;           /* elements                     */
  int64_t weights_in_stride, weights_stride;  /* elements between heads, >= prefix_len     */
  int32_t dtype;             /* dard_dtype of q and prefix_k                               */
  int32_t rows;              /* >= 0                                                       */
  int32_t hq, hkv, head_dim; /* as dard_step_attention                                     */
  int32_t prefix_len;        /* 0 .. DARD_PREFIX_MAX_LEN                                   */
  float scale;               /* softmax scale; 0 means 1/sqrt(head_dim)                    */
  float decay;               /* finite                                                     */
  uint32_t* status;          /* optional device word: DARD_STATUS_TIMEOUT                  */
  void* workspace;           /* optional device scratch of
                                dard_prefix_weights_workspace_size() bytes, 16-byte aligned;
                                needs no preparation. Without it the rows are not split. Calls
                                that overlap on the GPU need separate workspaces.          */
  size_t workspace_bytes;
} dard_prefix_weights_args;

/* Bytes of workspace for these sizes or smaller ones, any dtype (0 on invalid sizes). */
size_t dard_prefix_weights_workspace_size(int32_t rows, int32_t hq, int32_t hkv, int32_t head_dim,
                                          int32_t prefix_len);

/* One launch, or two where the rows are split. Errors: DARD_ERR_NULL, _SHAPE, _VALUE,
 * _UNSUPPORTED, _ALIGN, _WORKSPACE, _CUDA. */
dard_status dard_prefix_weights(const dard_prefix_weights_args* args, void* stream);

/* Per key/value head g, `keep` of the prefix's keys: the first keep_first, the last keep_last, and
 * of those in between the keep - keep_first - keep_last with the largest weights (of equal weights
 * the lowest index; -0 equals 0; a NaN counts as smaller than every number). kept[g] lists them in
 * rising order, and
 *     k_out[i,g] = k[kept[g,i],g],   v_out[i,g] = v[kept[g,i],g],   weights_out[g,i] =
 *     weights[g,kept[g,i]]
 * The outputs must not overlap the inputs or one another, nor rows of an output by its strides
 * (k_out and v_out may lie row by row beside each other in one buffer). */
typedef struct {
  const float* weights;      /* device [hkv, prefix_len]                                   */
  const void* prefix_k;      /* device, both optional together                             */
  const void* prefix_v;
  int32_t* kept;             /* device [hkv, keep] out, contiguous                         */
  void* k_out;               /* device out, required with prefix_k                         */
  void* v_out;
  float* weights_out;        /* optional device [hkv, keep] out, contiguous                */
  int64_t weights_stride;    /* elements between heads, >= prefix_len                      */
  int64_t prefix_row_stride, prefix_head_stride;  /* elements, of prefix_k and prefix_v    */
  int64_t out_row_stride, out_head_stride;        /* elements, of k_out and v_out          */
  int32_t dtype;             /* dard_dtype of the keys and values                          */
  int32_t hkv, head_dim;     /* head_dim 64 or 128                                         */
  int32_t prefix_len;        /* 0 .. DARD_PREFIX_MAX_LEN                                   */
  int32_t keep;              /* keep_first + keep_last .. prefix_len                       */
  int32_t keep_first, keep_last;  /* >= 0                                                  */
} dard_prefix_evict_args;

/* Two launches, the second a programmatic dependent of the first. Errors: DARD_ERR_NULL, _SHAPE,
 * _VALUE (dtype; an output that overlaps an input, another output or itself), _UNSUPPORTED, _ALIGN,
 * _CUDA. */
dard_status dard_prefix_evict(const dard_prefix_evict_args* args, void* stream);

/* Human-readable name of a status code; never NULL. */
const char* dard_status_string(dard_status s);

/* The message of the last DARD_ERR_CUDA / validation failure on this thread; never NULL. */
const char* dard_last_error(void);

/* Library version as major * 10000 + minor * 100 + patch. */
int32_t dard_version(void);

#ifdef __cplusplus
}
#endif
#endif /* DARD_H_ */

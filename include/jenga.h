/*
 * jenga.h - C ABI of the MI355X (gfx950) attention-carving library.
 *
 * The library computes, for one attention layer of a video diffusion transformer, the
 * block-sparse self-attention of "Training-Free Efficient Video Generation via Dynamic Token
 * Carving" (Sec. 3.1 "Block-Wise Attention Carving", appendix Alg. 2-4):
 *
 *   jenga_curve_permute     z_blk = G(z_thw)                      Eq. 2
 *   jenga_select_blocks     B = B_top u B_cond u B_adja           Eq. 3, Alg. 3, appendix Eq. 5
 *   jenga_block_sparse_attn O = attention over the blocks of B    Alg. 4, Alg. 2, Eq. 1
 *   jenga_unpermute         z_thw = G^-1(z_blk)                   Eq. 2
 *   jenga_stage_switch      resolution switch between stages      Eq. 4
 *
 * and what a transformer block has in front of that attention and behind it: layer norm and its gradient
 * (jenga_layer_norm), matrix products in 8-bit floating point (jenga_quantize, jenga_matmul), rotary positions
 * over time, height and width (jenga_rotary, jenga_forward_rotary).
 *
 * Conventions
 *   - All tensor arguments are DEVICE pointers unless a comment says "host".  The caller owns
 *     every tensor and every workspace; the library owns only what is inside a jenga_plan.
 *   - bf16 tensors are raw 16-bit bfloat16 bit patterns.
 *   - "thw side" layout:   [batch][N_v + N_c][heads][head_dim]   vision tokens in (t,h,w)
 *     row-major order (w fastest) followed by the N_c text tokens.
 *   - "curve side" layout: [batch][heads][N_pad][head_dim]       sequence positions are
 *     [vision in curve order | pad to M_v*m | text | pad to M_c*m]; N_pad = M*m, M = M_v + M_c.
 *   - `stream` is a hipStream_t passed as void* (NULL = the null stream).  The four hot calls
 *     only enqueue work: no allocation, no host synchronisation, no host<->device copies.
 *   - Every function returns JENGA_OK (0) or a negative jenga_status; nothing is thrown across
 *     the ABI and nothing is launched when validation fails.
 *   - One GPU: a plan belongs to the device that was current when it was created; a call that uses
 *     the plan's device tables with another device current returns JENGA_EINVAL.
 */
#ifndef JENGA_H_
#define JENGA_H_

#include <stddef.h>
#include <stdint.h>

#ifdef __cplusplus
extern "C" {
#endif

typedef enum {
  JENGA_OK = 0,
  JENGA_EINVAL = -1,       /* null pointer, non-positive size, ratio out of range            */
  JENGA_EUNSUPPORTED = -2, /* head_dim / block / sequence length outside what is built       */
  JENGA_EWORKSPACE = -3,   /* workspace smaller than jenga_plan_info reports                 */
  JENGA_EHIP = -4,         /* a HIP runtime call or a kernel launch failed                   */
  JENGA_ENOMEM = -5        /* host or device allocation failed while creating a plan         */
} jenga_status;

enum {
  JENGA_FLAG_ADJACENCY = 1u, /* union with B_adja (Sec. 3.1 item 3)                          */
  JENGA_FLAG_CONDITION = 2u, /* union with B_cond: all text key blocks (Sec. 3.1 item 2)      */
  JENGA_FLAG_CURVE = 4u,     /* 1: generalized Hilbert order; 0: linear thw order (ablation)  */
  JENGA_FLAG_PACED_WALK = 8u /* attention with blocks of 128 tokens visits the selected key blocks in an
                                order paced by a chip-wide clock instead of list order, so that the
                                workgroups of an XCD share tiles in the L2 (Alg. 4 sums over a set: the
                                order is free).  Faster; the last bits of the output may differ between
                                runs; a block listed twice is visited once.  Ignored for other block sizes */
};

/* Problem statement of one layer (Sec. 3.1; Alg. 2 and Alg. 3 inputs). */
typedef struct {
  int32_t T, H, W;     /* latent grid, each >= 1; N_v = T*H*W vision tokens.  A layer without vision
                          tokens (the text-only branch of Alg. 2) is plain dense attention and is not
                          taken: JENGA_EINVAL                                                  */
  int32_t n_text;      /* N_c >= 0 condition tokens, stored behind the vision tokens           */
  int32_t batch;       /* >= 1                                                                 */
  int32_t heads;       /* >= 1                                                                 */
  int32_t head_dim;    /* d_k: 64 or 128                                                       */
  int32_t block;       /* m: 32, 64 or 128 tokens per block                                    */
  double topk_ratio;   /* k in (0, 1]: keep at least K_top = max(1, floor(k*M_v + 1e-6)) blocks */
  double cum_prob;     /* p in [0, 1): extend until the kept probability mass exceeds p         */
  float text_bias;     /* beta of the text-attention amplifier (Sec. 3.2), added to the scaled
                          logits of vision-query x text-key pairs; 0 switches it off; must be
                          finite (NaN or +-inf: JENGA_EINVAL)                                  */
  uint32_t flags;      /* JENGA_FLAG_*                                                         */
} jenga_config;

/* Sizes derived from a config (all counts in tokens or blocks, workspaces in bytes). */
typedef struct {
  int32_t N_v, M_v, M_c, M, N_pad, pad_v, pad_c, K_top;
  uint64_t select_workspace_bytes; /* for jenga_select_blocks                                  */
  uint64_t attn_workspace_bytes;   /* for jenga_block_sparse_attn; enough for the packed entries */
} jenga_plan_info_t;

typedef struct jenga_plan jenga_plan; /* opaque, library-owned */

/*
 * Host precompute for one grid (Alg. 1 step "compute block reordering G, G^-1 and adjacency
 * masks"; Sec. 3.1: B_cond and B_adja depend only on the resolution and on G).  Builds the curve
 * permutation, the padded layout and the adjacency bit mask on the host, copies them to the
 * current device (synchronous) and returns the plan in *out.  cfg and out are host pointers.
 */
int jenga_plan_create(const jenga_config* cfg, jenga_plan** out);

/* Frees the device tables and the plan.  NULL is accepted. */
int jenga_plan_destroy(jenga_plan* plan);

/* Fills *info (host pointer). */
int jenga_plan_info(const jenga_plan* plan, jenga_plan_info_t* info);

/*
 * Copies the plan's tables to HOST arrays for inspection; any pointer may be NULL.
 *   perm[N_v]      thw index of the token at curve position i        (Eq. 2)
 *   inv_perm[N_v]  curve position of thw index n
 *   adja[M_v*M_v]  1 where blocks i and j hold tokens within Chebyshev distance 1 (Sec. 3.1)
 */
int jenga_plan_export(const jenga_plan* plan, int32_t* perm, int32_t* inv_perm, uint8_t* adja);

/*
 * Host-only form of create + info + export: computes the same tables without touching a device
 * (no plan is kept).  cfg and info are host pointers; perm, inv_perm, adja as in
 * jenga_plan_export, any of them may be NULL.  Same validation and status codes as create.
 */
int jenga_plan_tables(const jenga_config* cfg, jenga_plan_info_t* info, int32_t* perm, int32_t* inv_perm,
                      uint8_t* adja);

/*
 * Eq. 2, z_blk = G(z_thw), fused with the change of layout:
 *   dst_curve[b][h][i][:] = src_thw[b][src(i)][h][:]    for every valid position i, 0 for pads.
 * src_thw: bf16 thw side, read only.  dst_curve: bf16 curve side, fully overwritten.
 */
int jenga_curve_permute(const jenga_plan* plan, const void* src_thw, void* dst_curve, void* stream);

/*
 * jenga_curve_permute of Q, K and V in one launch: the same results as three calls in this order, also
 * where a result lies over a tensor that has moved by then (K's over Q): that is done in three launches.
 */
int jenga_curve_permute_qkv(const jenga_plan* plan, const void* q_thw, const void* k_thw, const void* v_thw,
                            void* q_curve, void* k_curve, void* v_curve, void* stream);

/*
 * Eq. 2 applied to a per-token table that has to follow the tokens into curve order, such as the
 * rotary position-embedding frequencies (appendix, implementation details, "Frequency re-ordering":
 * f_blk = G(f); Alg. 1, the step that remaps the positional frequencies once per stage):
 *   dst_rows[i][:] = src_rows[src(i)][:]   for every valid position i, 0 for pads.
 * src_rows: [N_v + N_c][row_bytes] bytes in thw order (text rows last), read only.
 * dst_rows: [N_pad][row_bytes], fully overwritten.  Both 16-byte aligned.
 * row_bytes: a power of two in [16, 4096] (e.g. 128 float32 = 512), else JENGA_EUNSUPPORTED.
 * The batch and heads of the plan play no part.
 */
int jenga_curve_permute_rows(const jenga_plan* plan, const void* src_rows, void* dst_rows, int32_t row_bytes,
                             void* stream);

/*
 * Alg. 3 with Alg. 2's rule for text queries.  For every (batch, head, query block i):
 *   i < M_v : mean-pool Q and K per block over their valid tokens (Eq. 3), R = softmax over all M
 *             key blocks of Q^.K^/sqrt(d_k); order by (R descending, index ascending);
 *             N_k = min(M, max(#{n : C_n <= p} + 1, K_top)) with C the running sum; keep the
 *             first N_k; union with the text key blocks and the adjacent blocks per the flags.
 *   i >= M_v: every block.
 * The arithmetic is float64 so that the integer decisions do not depend on summation order
 * beyond 1e-15 relative.
 *   q_curve, k_curve : bf16 curve side, read only (pad rows are ignored, not assumed zero)
 *   sel_count        : int32 [batch][heads][M]       number of selected key blocks
 *   sel_index        : int32 [batch][heads][M][M]    their indices, ascending; entries at and
 *                      beyond sel_count are left untouched
 *   mask_or_null     : uint8 [batch][heads][M][M]    dense 0/1 copy of B, or NULL
 *   workspace        : at least select_workspace_bytes, 256-byte aligned, contents undefined after
 */
int jenga_select_blocks(const jenga_plan* plan, const void* q_curve, const void* k_curve,
                        int32_t* sel_count, int32_t* sel_index, uint8_t* mask_or_null,
                        void* workspace, size_t workspace_bytes, void* stream);

/*
 * jenga_select_blocks for callers that cannot allocate or pass a workspace: code under HIP graph capture,
 * tight serving loops, harnesses that forbid hipMalloc.  Same computation, same outputs, same kernels; the
 * workspace is a static device array of JENGA_SELECT_STATIC_MAX_BYTES inside the library (one per GPU, resident
 * from module load until the process ends).  The call allocates nothing and frees nothing.
 *   - JENGA_EWORKSPACE when the plan's select_workspace_bytes exceeds JENGA_SELECT_STATIC_MAX_BYTES
 *     (nothing is launched); JENGA_EINVAL for null pointers or when the current device is not the plan's.
 *   - All calls on one GPU share that GPU's array: calls that may overlap in time on one GPU (different
 *     streams, different threads) race on it and must be serialised by the caller.  The array keeps the
 *     last call's contents; the kernels overwrite everything they read, so no clearing is needed.
 */
#define JENGA_SELECT_STATIC_MAX_BYTES (64u << 20)
int jenga_select_blocks_static(const jenga_plan* plan, const void* q_curve, const void* k_curve,
                               int32_t* sel_count, int32_t* sel_index, uint8_t* mask_or_null, void* stream);

/*
 * Alg. 4 (and Alg. 2's dense rows for text queries, which simply carry a full index list).
 * For query block i of (batch, head): softmax attention of its valid rows over the valid keys of
 * the blocks sel_index[..][i][0 .. sel_count), logits q.k/sqrt(d_k) (+ text_bias for a vision
 * query block and a text key block), bf16 MFMA products with float32 accumulation and float32
 * online softmax.  Pad query rows produce zeros.
 *   q, k, v    : bf16 curve side, read only
 *   sel_count, sel_index : as written by jenga_select_blocks.  Counts are clamped to [0, M] and
 *                indices to [0, M) on the device, so a malformed list cannot cause an access
 *                out of range; a count of 0 gives zero rows.  The order of a list does not matter
 *                beyond rounding (any permutation of the same blocks is accepted)
 *   out_curve  : bf16 curve side, fully overwritten
 *   lse_or_null: float32 [batch][heads][N_pad] or NULL.  For every valid query row the natural
 *                logarithm of the sum of exp(logit) over the keys it visited (logits scaled and
 *                biased as above): Alg. 4's running maximum and running sum combined, the value a
 *                caller needs to merge this result with attention over other keys.  Pad query rows
 *                and rows of an empty list get -inf.  Fully overwritten when given
 *   workspace  : at least attn_workspace_bytes, 256-byte aligned (where needed K and V re-tiled for the
 *                matrix cores, 256 bytes of launch parameters, and the results of the parts that long
 *                lists are cut into on grids that leave the chip idle, and some lists at the end of grids that
 *                do not, 129 MiB of them at most), contents undefined after
 * Equivalent to jenga_pack_kv followed by jenga_block_sparse_attn_packed on the same workspace (the latter
 * never cuts lists, since calls on one packed workspace may overlap: where this call does, the two differ
 * in the last bits; so may a call whose outputs lie over both K and V, or with both off the 16-byte grid).
 */
int jenga_block_sparse_attn(const jenga_plan* plan, const void* q, const void* k, const void* v,
                            const int32_t* sel_count, const int32_t* sel_index, void* out_curve,
                            float* lse_or_null, void* workspace, size_t workspace_bytes, void* stream);

/*
 * First half of jenga_block_sparse_attn: re-tiles K and V of every block (Alg. 4's "load key-value
 * block") into the matrix-core fragment order inside `workspace`; pad rows of V are zeroed.
 * A caller that attends several times to the same K and V (a sweep of k or p) packs once: what is packed
 * depends on T, H, W, n_text, batch, heads, head_dim and block alone.
 *   workspace  : 256-byte aligned, at least 2 * B + 256 bytes with B = batch * heads * N_pad * head_dim * 2 rounded
 *                up to a multiple of 256 (attn_workspace_bytes is never less); JENGA_EWORKSPACE below that
 */
int jenga_pack_kv(const jenga_plan* plan, const void* k, const void* v, void* workspace,
                  size_t workspace_bytes, void* stream);

/*
 * Second half of jenga_block_sparse_attn: the block-sparse attention kernel itself, reading K and V
 * from a workspace filled by jenga_pack_kv for this plan or for one that differs in topk_ratio, cum_prob,
 * text_bias or flags only (jenga_block_sparse_attn leaves nothing in its workspace that could be read
 * here); it may be as small as that call takes it.  The packed tiles are only read; the 256 bytes behind
 * them (launch parameters) may be written.
 * Other arguments as above.
 */
int jenga_block_sparse_attn_packed(const jenga_plan* plan, const void* q, void* packed_kv_workspace,
                                   size_t workspace_bytes, const int32_t* sel_count,
                                   const int32_t* sel_index, void* out_curve, float* lse_or_null,
                                   void* stream);

/*
 * Eq. 2, z_thw = G^-1(z_blk): dst_thw[b][src(i)][h][:] = src_curve[b][h][i][:] for every valid
 * position i; pad rows are dropped.  dst_thw is fully overwritten.
 */
int jenga_unpermute(const jenga_plan* plan, const void* src_curve, void* dst_thw, void* stream);

/*
 * A whole layer on thw-side tensors: jenga_curve_permute_qkv, jenga_select_blocks, jenga_block_sparse_attn and jenga_unpermute
 * in one call and fewer launches, with the same results in the same places (all of those calls' arguments are outputs here too; the
 * same bits, but for the last ones of the attention under the paced walk, which differ from run to run).
 * Refuses what they refuse, before anything is launched.  An output that lies over an input is taken as those calls one after the
 * other take it.
 */
int jenga_forward(const jenga_plan* plan, const void* q_thw, const void* k_thw, const void* v_thw, void* q_curve,
                  void* k_curve, void* v_curve, int32_t* sel_count, int32_t* sel_index, uint8_t* mask_or_null,
                  void* select_workspace, size_t select_workspace_bytes, void* out_curve, float* lse_or_null,
                  void* attn_workspace, size_t attn_workspace_bytes, void* out_thw, void* stream);

/*
 * Progressive-resolution stage switch (Sec. 3.2, Eq. 4), one fused elementwise pass:
 *   x_out = (1 - sigma_t) * U(x_t - sigma_t * eps_t) + sigma_t * eps_tilde
 * U is 3D area interpolation from (T_in, H_in, W_in) to (T_out, H_out, W_out): along each axis with I
 * input and O output cells, output cell o is the unweighted mean of input cells
 * floor(o*I/O) .. ceil((o+1)*I/O) - 1 (for integer factors: replication); any sizes >= 1 are accepted,
 * also smaller outputs.
 *   x_t, eps_t : float32 [channels][T_in][H_in][W_in]   latent and the model's prediction at step t (batch
 *                folded into channels), read only
 *   eps_tilde  : float32 [channels][T_out][H_out][W_out] standard-normal draw supplied by the caller
 *   x_out      : float32 [channels][T_out][H_out][W_out], fully overwritten; must not alias the inputs
 *   sigma_t    : scheduler noise level in [0, 1]
 * No plan is needed.  float32 arithmetic, window sums in (t, h, w) order.  Only enqueues work on `stream`.
 * JENGA_EINVAL for null pointers, sizes < 1 or sigma_t outside [0, 1] (NaN included); JENGA_EUNSUPPORTED
 * when an extent exceeds 2^14 or the output has more than 2^32 rows or 2^34 cells.
 */
int jenga_stage_switch(const float* x_t, const float* eps_t, const float* eps_tilde, float* x_out,
                       int32_t channels, int32_t T_in, int32_t H_in, int32_t W_in, int32_t T_out,
                       int32_t H_out, int32_t W_out, float sigma_t, void* stream);

/* ---- around the attention -------------------------------------------------------------------
 *
 * These calls need no plan and keep nothing; they only enqueue work on `stream`, on the device that is
 * current, whose memory all device pointers have to be.  Configs are host pointers, read before the call
 * returns.  Strides are in elements; values of a row, a head or a group lie next to each other.  A pointer
 * to elements is a multiple of their size unless a comment asks for more; rows off the 16-byte grid are
 * taken.  An output may lie over nothing else that the call reads or writes, except where a comment says so:
 * JENGA_EINVAL.  Calls with no rows return JENGA_OK and touch nothing.
 */

/* Types of elements.  JENGA_E4M3: OCP 8-bit floating point, 4 exponent and 3 mantissa bits, no infinities. */
typedef enum { JENGA_BF16 = 0, JENGA_F16 = 1, JENGA_F32 = 2, JENGA_E4M3 = 3 } jenga_type;

/*
 * 8-bit tensors.  A matrix of r rows and c columns is held as
 *   values  e4m3 [r][C], C = c rounded up to a multiple of 128; the columns that fill up are 0.  16-byte aligned
 *   scales  uint8 [r][S] (a block is 1 row x 128 columns) or [ceil(r / 128)][S] (128 x 128), S = ceil(c / 512) * 4;
 *           byte e + 127, 0 to 254, for the scale 2^e of a block; the bytes that fill up a row are 0.  4-byte aligned
 * and stands for values * 2^e.  e is the least whole number >= -127 with |x| <= 448 * 2^e for all finite x of the
 * block (0 where they are all 0): nothing saturates, and the only rounding is the one to e4m3, to nearest even.
 * What is not finite becomes NaN.
 */

/*
 * x -> 8-bit tensor with blocks of block_rows (1 or 128) rows and 128 columns.
 *   x: x_type (JENGA_BF16, JENGA_F16 or JENGA_F32) [rows][cols], x_stride >= cols elements from row to row
 * A matrix product takes its left operand with blocks of 1 row and its right one (weights) with 128; the
 * transpose of a matrix with blocks of 128 x 128 holds the same values.
 * JENGA_EINVAL: null or misaligned pointers, cols < 1, rows < 0, another block_rows; JENGA_EUNSUPPORTED: more
 * than 2^17 columns or 2^30 rows.
 */
int jenga_quantize(const void* x, int64_t x_stride, int32_t x_type, int64_t rows, int32_t cols, int32_t block_rows,
                   void* q, uint8_t* scale, void* stream);

/* out = a b^T + bias.  m >= 0, n >= 1, k a positive multiple of 128 (the columns of both operands as held). */
typedef struct {
  int64_t m, out_stride; /* rows of a and out; elements between rows of out, >= n               */
  int32_t n, k;          /* rows of b; columns of a and b                                       */
  int32_t out_type;      /* JENGA_BF16, JENGA_F16 or JENGA_F32                                  */
  int32_t reserved;      /* 0                                                                   */
} jenga_matmul_config;

/*
 * Product of two 8-bit tensors:
 *   out[i][j] = sum over blocks kb of 2^(ea[i][kb] + eb[j / 128][kb]) * sum over k in kb of a[i][k] b[j][k] + bias[j]
 *   a, a_scale   : [m][k] with blocks of 1 x 128
 *   b, b_scale   : [n][k] with blocks of 128 x 128
 *   bias_or_null : float32 [n]
 * Sums are float32 and rounded once.  For 16-bit results the f8 matrix core multiplies, which adds eight products
 * at a time and cuts them off at 2^-13 of the largest of the eight (for normally distributed values 1.5e-5 of the
 * result's norm), and sums below 2^-126 may be taken as 0; for float32 results the operands are widened to bf16, and nothing is cut
 * off but values * 2^e below 2^-126, which may lose digits or be taken as 0, and of 2^128 (what x above 3.29e38 is rounded to), which
 * are infinite.
 * The gradients are products of the same kind: of a, from out's gradient in rows of blocks and b's transpose; of b,
 * from the transposes of out's gradient (blocks of 1 x 128) and of a (128 x 128).
 * JENGA_EUNSUPPORTED: more than 2^23 tiles of 128 x 128, k above 2^17, n above 2^22.
 */
int jenga_matmul(const jenga_matmul_config* cfg, const void* a, const uint8_t* a_scale, const void* b,
                 const uint8_t* b_scale, const float* bias_or_null, void* out, void* stream);

/*
 * Layer norm over the columns of each row.  Rows come in groups of group_rows consecutive ones (the last may be
 * short) that share a weight and a bias: all rows in one group are the ordinary affine norm, a group for each batch
 * entry with weight_offset 1 the modulation of a diffusion transformer, (1 + scale) and shift.
 */
typedef struct {
  int64_t rows, group_rows; /* >= 0; >= 1                                                       */
  int64_t x_stride;         /* elements between rows of x (and dx), >= cols                     */
  int64_t y_stride;         /* of y, or dy in the gradient, >= cols; JENGA_E4M3: cols rounded up to 128 */
  int64_t param_stride;     /* between groups of weight and bias, >= cols                       */
  int32_t cols;             /* 1 to 2^17                                                        */
  int32_t x_type;           /* JENGA_BF16, JENGA_F16 or JENGA_F32                               */
  int32_t y_type;           /* of y (or dy): x_type, or in the forward pass JENGA_E4M3          */
  int32_t param_type;       /* of weight and bias: x_type or JENGA_F32                          */
  float eps, weight_offset; /* finite, eps >= 0                                                 */
} jenga_norm_config;

/*
 *   mu = mean(x)   r = 1 / sqrt(mean((x - mu)^2) + eps)   y = (x - mu) r (weight_offset + weight) + bias
 *   weight, bias : param_type [groups][cols], or NULL for zeros
 *   y            : [rows][cols]; may be x itself (same address, stride and type).  JENGA_E4M3: an 8-bit tensor with
 *                  blocks of 1 x 128, its scales in y_scale (else NULL)
 *   mean, rstd   : float32 [rows], mu and r for the gradient, or NULL
 * Sums are float32, y is rounded once.
 */
int jenga_layer_norm(const jenga_norm_config* cfg, const void* x, const void* weight_or_null, const void* bias_or_null,
                     void* y, uint8_t* y_scale_or_null, float* mean_or_null, float* rstd_or_null, void* stream);

/*
 * Its gradient, from dy and what the forward pass left in mean and rstd:
 *   h = (x - mean) rstd   g = dy (weight_offset + weight)   dx = rstd (g - mean(g) - h mean(g h))
 *   dweight[group] = sum over its rows of dy h   dbias[group] = sum of dy
 *   dy              : x_type, y_stride elements between rows
 *   dx              : x_type, x_stride elements between rows
 *   dweight, dbias  : float32 [groups][cols] next to each other, fully overwritten, or NULL
 *   workspace       : jenga_layer_norm_grad_workspace bytes, 256-byte aligned, contents undefined after; NULL if
 *                     both of them are.  Calls that may run at the same time (on two streams, in graphs that are
 *                     replayed on two streams) need one each
 * Sums are float32 and in an order that depends on the sizes alone: the same call gives the same bits.
 * JENGA_EUNSUPPORTED: more than 2^20 groups.
 */
int jenga_layer_norm_grad(const jenga_norm_config* cfg, const void* x, const void* dy, const void* weight_or_null,
                          const float* mean, const float* rstd, void* dx, float* dweight_or_null, float* dbias_or_null,
                          void* workspace, size_t workspace_bytes, void* stream);

/* Bytes of its workspace (host only): (1024 + groups) * cols * 8. */
int jenga_layer_norm_grad_workspace(const jenga_norm_config* cfg, uint64_t* bytes);

/*
 * Rotary positions over the axes of a T x H x W grid.  The first dim[0] channels of a head turn with the token's
 * t, the next dim[1] with its h, the next dim[2] with its w, the rest stay as they are.  Pair i of an axis with d
 * channels turns by (origin + step * cell) * theta^(-2i / d):  (x, y) -> (x cos - y sin, x sin + y cos).
 * JENGA_EUNSUPPORTED, in all calls with such a config: more than 2^24 cells, an odd head_dim or one above 1024, more than
 * 2^31 - 1024 pairs of all axes and cells, (T dim[0] + H dim[1] + W dim[2]) / 2.
 */
enum {
  JENGA_ROTARY_HALVES = 1u, /* pair i of an axis is its channels i and i + d/2; else 2i and 2i + 1   */
  JENGA_ROTARY_INVERSE = 2u /* turns back: the inverse, and the gradient                          */
};
typedef struct {
  int32_t T, H, W;           /* cells, each >= 1, at most 2^24 together                          */
  int32_t head_dim;          /* even, 2 to 1024                                                  */
  int32_t dim[3];            /* channels of each axis: even, >= 0, together 2 to head_dim         */
  int32_t type;              /* JENGA_BF16, JENGA_F16 or JENGA_F32                               */
  double theta;              /* > 0                                                              */
  double origin[3], step[3]; /* position of cell n of an axis: origin + step * n                 */
  uint32_t flags;            /* JENGA_ROTARY_*                                                   */
  uint32_t reserved;         /* 0                                                                */
} jenga_rotary_config;

/*
 * cos and sin of every pair and cell, axis by axis: float32 [T][dim[0]/2][2], [H][dim[1]/2][2], [W][dim[2]/2][2] one
 * behind the other, T dim[0] + H dim[1] + W dim[2] floats in HOST memory, from float64 angles.  The caller copies them
 * to the device once per grid.  Host only.  JENGA_EINVAL, with the table undefined: an angle that is not finite.
 */
int jenga_rotary_table(const jenga_rotary_config* cfg, float* table);

/* A tensor [batch][tokens][heads][head_dim] where its strides say; dst may be src itself (same address and strides). */
typedef struct {
  const void* src;
  void* dst;
  int64_t src_batch, src_token, src_head; /* elements, >= 0                                      */
  int64_t dst_batch, dst_token, dst_head; /* no two elements of dst in one place                 */
  int32_t heads, reserved;                /* >= 1; 0                                             */
} jenga_rotary_tensor;

/*
 * Turns one or two tensors (Q and K) in one launch.  Angles and products are float32, results rounded once.
 *   table   : of this grid, dims, theta, origin and step, on the device, 8-byte aligned
 *   tensors : host array of `count` (1 or 2)
 * The cell of a token:
 *   plan and cells NULL : token n < T*H*W is cell n in (t,h,w) row-major order; tokens behind (text) are copied
 *   plan                : curve side; position i has the cell of its token, text and pads are copied.  The plan has the
 *                         same T, H and W, and tokens = N_pad
 *   cells               : int32 [batch][tokens][3], the cell on each axis: sequences of several grids, padded batches.
 *                         Channels of an axis where it is negative are copied; cells past the end are taken as the last
 * JENGA_EUNSUPPORTED: more than 2^32 - 256 pairs in one head of all tokens.
 */
int jenga_rotary(const jenga_rotary_config* cfg, const jenga_plan* plan_or_null, const int32_t* cells_or_null,
                 const float* table, const jenga_rotary_tensor* tensors, int32_t count, int64_t batch, int64_t tokens,
                 void* stream);

/*
 * jenga_forward of Q and K turned by their rotary positions: jenga_rotary of both and jenga_forward, with the same results, in the
 * launches of jenga_forward alone (the turn is part of the re-ordering pass).
 *   rotary, table : as in jenga_rotary, of the plan's grid and head_dim and type JENGA_BF16
 *   q, k, v_thw   : bf16 thw side, read only, consecutive tokens (of all batch entries) token_stride >= heads * head_dim
 *                   elements apart: 3 * heads * head_dim for the columns of one projection, q, k and v_thw in the same rows
 * Other arguments as in jenga_forward.  No output may lie over another tensor.
 * JENGA_EUNSUPPORTED: more than 21845 batch entries, token_stride above 2^24.
 */
int jenga_forward_rotary(const jenga_plan* plan, const jenga_rotary_config* rotary, const float* table, const void* q_thw,
                         const void* k_thw, const void* v_thw, int64_t token_stride, void* q_curve, void* k_curve,
                         void* v_curve, int32_t* sel_count, int32_t* sel_index, uint8_t* mask_or_null,
                         void* select_workspace, size_t select_workspace_bytes, void* out_curve, float* lse_or_null,
                         void* attn_workspace, size_t attn_workspace_bytes, void* out_thw, void* stream);

/* Static, NUL-terminated description of a status code. */
const char* jenga_strerror(int status);

#ifdef __cplusplus
}
#endif
#endif /* JENGA_H_ */

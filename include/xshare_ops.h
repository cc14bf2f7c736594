/*
 * xshare_ops.h — operators of libxshare.so around the layer of xshare.h:
 * expert gating from router logits, and float8 experts.
 *
 * xshare.h routes on scores that the caller holds and runs bf16 experts.  The
 * layers it is shaped after score with a sigmoid or a softmax, balance their
 * load with a bias that only takes part in the choice, restrict a token to a
 * few expert groups, and store their experts as 8-bit floating point with one
 * scale per 128 x 128 block.  These are their operators:
 *
 *   xshare_gate            logits -> ids, weights (and scores, counts, offsets, permutation)
 *   xshare_quant_fp8_rows, xshare_quant_fp8_blocks   values and scales of tokens and weights
 *   xshare_matmul_fp8      product of such operands, dense or grouped by expert
 *   xshare_experts_fp8     routed SwiGLU experts on such weights
 *
 * xshare_gate's scores may be handed to xshare_route, the ids and weights of
 * either to xshare_experts_fp8, and xshare_route's sel_mask to xshare_gate.
 *
 * The conventions, error codes and limits of xshare.h hold: device pointers of
 * the current device, contiguous, 16-byte aligned; caller-owned outputs and
 * workspaces (256-byte aligned); asynchronous on `stream`; arguments checked on
 * the host, nothing written after a negative return.  An output overlaps neither
 * an input nor another output.  All calls may be captured
 * into a CUDA graph; calls that share a workspace must not overlap.  A workspace that
 * is large enough for some sizes is so for smaller ones.  Every call gives the same
 * bits for the same arguments; how a float8 product groups its sums over K
 * depends on the number of rows, so a row's last bits may change with its company.
 * A wait inside a product that runs out is reported in stats->status where stats is given; in
 * any case the part of the output that the product could not finish is NaN (and more may be).
 * The library serves: nothing here has a backward pass.
 *
 * 8-bit floating point is e4m3 (finite values up to 448, NaN, no infinity), one
 * byte per value, passed as uint8_t.  A block's scale is
 *   s = max(amax, 2^-100) / 448    (fp32, correctly rounded; amax = largest |x| of the block)
 * and its values are q = e4m3(fp32(x / s)), both roundings to nearest even, so
 * that x is about q s.  A NaN becomes a NaN and does not count in amax; in a
 * block with an infinity s is infinite, the infinities become NaN, other
 * values 0 (whose products are NaN).
 */
#ifndef XSHARE_OPS_H
#define XSHARE_OPS_H

#include "xshare.h"

#ifdef __cplusplus
extern "C" {
#endif

/* Element types of arguments passed as void *. */
enum { XS_F32 = 0, XS_BF16 = 1, XS_F16 = 2 };

enum { XS_SCORE_SOFTMAX = 0, XS_SCORE_SIGMOID = 1 };

typedef struct {
  int32_t scoring;     /* XS_SCORE_* */
  int32_t n_groups;    /* G: contiguous groups of N / G experts; 1 <= G <= 32, N % G == 0 */
  int32_t top_groups;  /* groups a token may use; 1 <= top_groups <= G (G: no restriction) */
  int32_t group_top;   /* a group is worth the sum of its best 1 or 2 choice values */
  int32_t renorm;      /* 1: weights divided by their sum; 0: the scores themselves */
  float scale;         /* factor of every weight; finite */
} xs_gate_params;

/* Bytes of workspace xshare_gate needs for expert_counts, expert_offsets or
 * perm; 0 for arguments the call would reject. */
size_t xshare_gate_workspace_size(int B, int N, int k);

/* Routes every token by its router logits.
 *
 *   logits  [B, N] fp32, bf16 or fp16 (`dtype`), device.
 *   s[e] = softmax over the eligible experts, or 1 / (1 + exp(-logit)), fp32.
 *   c[e] = s[e] + bias[e]: the choice value.  bias [N] fp32, nullable (0).
 *   ids  = the k experts of largest c among the eligible ones of the top_groups
 *          best groups, best first; equal values: the lower index first, among
 *          groups too.  Values are ordered as real numbers: where fp32 cannot
 *          tell two of them apart, the row is evaluated again with about 40 bits; where
 *          those agree too, the larger bias goes first, then the larger logit, so that
 *          equal biases (of zeros, say) leave experts in the order of their logits.
 *          (A choice value or a sum of two beyond fp32's range counts as infinite.)
 *   w    = s[ids], divided by their sum (renorm; 1 / (number routed) if the sum
 *          is 0), times scale.
 *
 * An expert is eligible for a token if expert_mask[e] != 0 (or no mask), and
 * its logit and its choice value are neither NaN nor -infinity.  A logit of
 * +infinity counts as the largest finite fp32 value.  With fewer than k experts to choose
 * from, the remaining slots get id -1 and weight 0.  Rows with token_mask[t] ==
 * 0 (padding) get -1, 0 and scores 0 throughout; nothing of them is read.
 *
 *   expert_mask [N], token_mask [B] uint8, device, nullable.
 *   topk_ids [B, k] int32, topk_w [B, k] fp32, out.
 *   scores_out [B, N] fp32, out, nullable: s, 0 for experts that are not eligible.
 *   expert_counts [N], expert_offsets [N + 1], perm [B * k] int32, out, nullable:
 *          as in xshare_route; only the first offsets[N] entries of perm are written.
 *   workspace: xshare_gate_workspace_size bytes if one of the last three is
 *          asked for, else nullable.
 * Limits: 1 <= B <= 8192, 1 <= N <= 1024, 1 <= k <= min(N, 16). */
int xshare_gate(const void *logits, int dtype, const float *bias, const uint8_t *expert_mask,
                const uint8_t *token_mask, int B, int N, int k, const xs_gate_params *prm,
                int32_t *topk_ids, float *topk_w, float *scores_out, int32_t *expert_counts,
                int32_t *expert_offsets, int32_t *perm, void *workspace, size_t ws_bytes,
                xs_stream_t stream);

/* x [M, K] (fp32, bf16 or fp16) -> q [M, K] e4m3 and scales [M, ceil(K / 128)]
 * fp32, one scale per row and 128 columns (the last block may be shorter).
 * 1 <= M, K <= 2^20. */
int xshare_quant_fp8_rows(const void *x, int dtype, int M, int K, uint8_t *q, float *scales,
                          xs_stream_t stream);

/* n matrices x [n, R, K] -> q [n, R, K] and scales [n, ceil(R / 128), ceil(K / 128)],
 * one scale per 128 x 128 block.  1 <= R, K <= 2^20, 1 <= n <= 1024, at most 2^31 - 512
 * blocks. */
int xshare_quant_fp8_blocks(const void *x, int dtype, int n, int R, int K, uint8_t *q, float *scales,
                            xs_stream_t stream);

/* Bytes of workspace of xshare_matmul_fp8; 0 for arguments that it would reject. */
size_t xshare_matmul_fp8_workspace_size(int M, int N, int K, int E);

/* y[m, n] = sum over blocks j of a_scale[m, j] b_scale[e, n / 128, j]
 *           * (sum over k in block j of a[m, k] b[e, n, k])
 * with the inner sums on the tensor cores (fp32 accumulators), the outer one in
 * fp32, rounded once to y's type.
 *
 *   a [M, K] e4m3, a_scale [M, ceil(K / 128)] fp32   (xshare_quant_fp8_rows)
 *   b [E, N, K] e4m3, b_scale [E, ceil(N / 128), ceil(K / 128)] fp32   (xshare_quant_fp8_blocks)
 *   offsets: NULL (then E == 1 and every row takes matrix 0), or [E + 1] int32,
 *          device: rows offsets[e] .. offsets[e + 1] - 1 take matrix e.  Entries
 *          are clamped to 0 .. M and made non-decreasing; rows before the first
 *          and behind the last entry are not written and have no influence (tiles that
 *          end or begin beside them are loaded whole, so a of all M rows is read).
 *   y [M, N] of type y_dtype (XS_*).
 *   stats: nullable; status is set (XS_DEV_*), and with offsets n_pairs = rows
 *          and n_used = matrices with a row; the other fields are 0.
 * 1 <= M, N, K <= 2^20, K % 16 == 0, 1 <= E <= 1024, E N <= 2^31 - 512. */
int xshare_matmul_fp8(const uint8_t *a, const float *a_scale, const uint8_t *b, const float *b_scale,
                      const int32_t *offsets, int M, int N, int K, int E, void *y, int y_dtype,
                      xs_stats *stats, void *workspace, size_t ws_bytes, xs_stream_t stream);

/* The weights of n float8 experts, device pointers, as xshare_quant_fp8_blocks
 * makes them of bf16 ones: gate, up [n, F, d], gate_s, up_s [n, F / 128, d / 128];
 * down [n, d, F], down_s [n, d / 128, F / 128]. */
typedef struct {
  const uint8_t *gate, *up, *down;
  const float *gate_s, *up_s, *down_s;
  int32_t n;
} xs_fp8_experts;

/* Bytes of workspace of xshare_experts_fp8; 0 for arguments it would reject. */
size_t xshare_experts_fp8_workspace_size(int B, int N, int k, int d, int F);

/* The experts of a routed batch on float8 weights:
 *   q(x_t): x_t in 1 x 128 blocks;   g, u = W_gate[e] q(x_t), W_up[e] q(x_t)  (fp32)
 *   h = silu(g) * u in fp32 (silu within 2^-20 + |g| 2^-24 of its value; 0 where e^-g
 *   passes 2^126), q(h) in 1 x 128 blocks;   o_ts = W_down[e] q(h)  (fp32
 *   sums; above 64 slots per expert kept in fp16 with one power of two per 64 columns)
 *   y_t = sum over slots s, in order, of topk_w[t, s] o_ts, fp32, rounded once to bf16.
 *
 *   x [B, d], y [B, d] bf16; topk_ids [B, k] int32, topk_w [B, k] fp32, as
 *   xshare_gate, xshare_route or the caller makes them.  A slot whose id is
 *   outside 0 .. experts->n - 1 is unused, whatever its weight; a token
 *   without a used slot gets y_t = 0.  An id may occur twice in a row.  A shared
 *   expert is one more matrix that every row lists, with weight 1.
 *   Only the experts that receive a token are read.
 *   stats: nullable; n_pairs, n_used and status are set, the other fields are 0.
 * 1 <= B <= 8192, 1 <= k <= 32, 1 <= experts->n <= 1024, d % 128 == 0, F % 128 == 0,
 * experts->n * max(d, F) <= 2^31 - 512. */
int xshare_experts_fp8(const uint16_t *x, const int32_t *topk_ids, const float *topk_w,
                       const xs_fp8_experts *experts, int B, int k, int d, int F, uint16_t *y,
                       xs_stats *stats, void *workspace, size_t ws_bytes, xs_stream_t stream);

#ifdef __cplusplus
}
#endif

#endif /* XSHARE_OPS_H */

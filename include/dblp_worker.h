/*
 * dblp_worker -- the two ends of a worker's training step on one AMD MI355X (gfx950): what makes the
 * gradient that dblp_packetize cuts into packets and what the tokens go through first.
 *
 *   dblp_embed           tokens (and positions) -> rows of the embedding tables, scaled, dropped out
 *   dblp_embed_grad      its gradient: the table's whole fp32 gradient, by sorted tokens
 *   dblp_dropout         dropout from a counter-based generator, with a residual; its own backward pass
 *   dblp_token_logprobs  log probability of one given token a row of logits
 *   dblp_policy_loss     clipped policy loss with a KL term, and the gradient of the logits
 *
 * The protocol sends a lost packet again byte for byte, so a worker that computes its step again must
 * find the same gradient: every result here is a function of the arguments alone.  There are no
 * floating-point atomics, a gradient row's sum is grouped by the tokens alone, and a dropout mask is
 * computed from (seed, draw, place) wherever it is needed and never stored.
 *
 * Conventions (those of dblp_agg.h, without a context)
 *   - Every call returns DBLP_OK or a negative DBLP_E* code; nothing throws, aborts or prints.
 *     dblp_worker_error() gives the text of this thread's last failure.  Arguments are checked on the
 *     host before the device is touched; on an error nothing has been enqueued, unless it is EHIP.
 *   - d_* are DEVICE pointers owned by the caller, h_* HOST pointers.  The calls enqueue on `stream`
 *     (hipStream_t as void*, NULL = the null stream) of `device`, never allocate, never wait, and may
 *     be recorded into a HIP graph.  The calling thread's current device is the same afterwards.
 *   - A matrix is rows of consecutive elements, rows `stride` ELEMENTS apart; pointers are aligned to one
 *     element.  An input's rows may overlap or be the same row (stride 0); an output's stride is at least
 *     its columns.  An output overlaps no other argument except where "in place" says so.  Rows whose
 *     address and stride are multiples of 16 bytes are fastest.
 *   - Types of matrices: DBLP_F32, DBLP_BF16, DBLP_F16.  Everything is computed in fp32 (what is
 *     made of a token's score, and sums of whole batches, in fp64) and rounded once, to nearest even, when it is stored.
 *   - A token, position or target outside its table (negative, or not below the number of rows) is "none":
 *     its row of the table is taken as zero, it has no gradient, it is not counted in a loss.  This is
 *     how padding and prompts are marked; nothing is read out of bounds.
 *   - Zero tokens or rows are allowed.  Limits: tokens, rows, vocabulary and columns below 2^31, columns of
 *     dblp_embed_grad below 2^22.
 *   - A workspace is DEVICE memory of the size that dblp_*_workspace gives, 256-byte aligned, of any
 *     contents; it is free again when the stream has passed the call.  One of a larger call (more tokens, a
 *     larger vocabulary, more columns) is large enough for a smaller one.
 */
#ifndef DBLP_WORKER_H
#define DBLP_WORKER_H

#include <stdint.h>

#include "dblp_agg.h"

#ifdef __cplusplus
extern "C" {
#endif

#define DBLP_F32 0
#define DBLP_BF16 1
#define DBLP_F16 2

/* A dropout mask over a matrix.  Eight neighbouring columns of a row share one call of Philox4x32 with
 * ten rounds (Salmon, Moraes, Dror, Shaw: Parallel Random Numbers: As Easy as 1, 2, 3; SC 2011): key =
 * seed, counter = {g, d} as four 32-bit words, low ones first, g = row * ceil(columns / 8) + column / 8,
 * d = draw + *d_draw.  Column c takes 16 of the 128 bits, bits 16 (c % 8) and up.  The value is dropped iff
 * they are less than t = rint(65536 p); what is kept is multiplied by 65536 / (65536 - t), so the mean is
 * exact for the probability that is really used.  p below 2^-17 drops nothing, p = 1 everything.
 * d_draw (may be NULL) is read when the kernel runs, so that a recorded graph draws anew at each replay. */
typedef struct {
    uint64_t seed;
    uint64_t draw;
    const uint64_t* d_draw; /* DEVICE, one word, or NULL */
    double p;               /* 0..1 */
} dblp_drop;

/* out[t] = drop(scale * table[tokens[t]] + pos_table[positions[t]]), n_tokens x dim.
 * d_positions NULL: no position term (then d_pos_table must be NULL).  The position table has the token
 * table's type.  h_drop NULL or p = 0: nothing is dropped.  A dropped value is +0 whatever was there. */
int dblp_embed(int device, void* stream, const int64_t* d_tokens, uint64_t n_tokens, uint32_t dim,
               const void* d_table, uint64_t table_stride, uint64_t vocab, int table_type, float scale,
               const int64_t* d_positions, const void* d_pos_table, uint64_t pos_stride, uint64_t n_positions,
               const dblp_drop* h_drop, void* d_out, uint64_t out_stride, int out_type);

/* grad[v] = base[v] + scale * sum of drop(dy[t]) over all t with tokens[t] = v, for every v below vocab; the
 * terms are added in ascending t within groups that n_tokens and the tokens fix.  grad is fp32, what a packet carries.  d_base NULL: zeros; d_base == d_grad (and equal strides):
 * in place, only rows that have a token are touched (a tied table's other gradient, or an earlier micro-batch);
 * another fp32 matrix: every row is written.  The position table's gradient is the same call on the positions.
 * h_drop: the mask of the forward pass. */
int dblp_embed_grad(int device, void* stream, const int64_t* d_tokens, uint64_t n_tokens, uint32_t dim, uint64_t vocab,
                    float scale, const dblp_drop* h_drop, const void* d_dy, uint64_t dy_stride, int dy_type,
                    const float* d_base, uint64_t base_stride, float* d_grad, uint64_t grad_stride,
                    void* d_workspace, uint64_t workspace_bytes);
/* Bytes of its workspace; 0 if an argument is out of range. */
uint64_t dblp_embed_grad_workspace(uint64_t n_tokens, uint64_t vocab, uint32_t dim);

/* y = drop(x) + residual (d_residual NULL: drop(x)); x, residual and y have one type.  The gradient of x is
 * the same call on y's gradient without a residual; the residual's is y's itself.  In place: y may be x or the
 * residual, with the same stride. */
int dblp_dropout(int device, void* stream, uint64_t rows, uint32_t cols, const void* d_x, uint64_t x_stride,
                 const void* d_residual, uint64_t residual_stride, const dblp_drop* h_drop,
                 void* d_y, uint64_t y_stride, int type);

/* logp[t] = logits[t][targets[t]] - lse[t], lse[t] = log sum_j exp(logits[t][j]).  d_lse may be NULL.  A row
 * without a target is not read, its logp and lse are 0.  A row whose logits are all -inf has lse = logp = -inf,
 * one that holds NaN or +inf has NaN. */
int dblp_token_logprobs(int device, void* stream, uint64_t n_tokens, uint32_t vocab, const void* d_logits,
                        uint64_t logits_stride, int type, const int64_t* d_targets, float* d_logp, float* d_lse,
                        void* d_workspace, uint64_t workspace_bytes);

/* Clipped policy loss with a KL term.  For each counted token t, with lp = log probability of targets[t]:
 *   r  = exp(lp - old_logp[t])                          (d_old_logp NULL: the policy is its own old one, r = 1)
 *   pl = -min(r A, clip(r, 1 - clip_low, 1 + clip_high) A),      A = advantages[t]
 *   kl = exp(ref_logp[t] - lp) - (ref_logp[t] - lp) - 1          (d_ref_logp NULL: 0)
 *      (a ratio past fp64 counts as the largest number, so that A = 0 has no part in the loss)
 *   loss = sum of weights[t] (pl + kl_coef kl)          (kl_coef 0: no KL term in loss and gradient, its sum is watched)
 *   d loss / d lp = weights[t] ([clipped term larger or equal] -r A + kl_coef (1 - exp(ref_logp[t] - lp)))
 *   dlogits[t][j] = grad_scale (d loss / d lp) ([j = targets[t]] - softmax(logits[t])[j])
 * A reference of -inf or far below the policy (a token that it masks) has an endless or large kl, and its gradient is that of a
 * slope of kl_coef.  Where lp is -inf (a token of probability zero was taken) kl is exp(inf) - inf, NaN, and the row's gradient infinite or NaN.
 * The weights hold the normalisation (one over the number of tokens, or of a sequence's tokens, ...).  With A = 1 and no old
 * and reference policy the gradient is that of the cross-entropy, whose value is -sum weights logp.
 * Not counted: targets[t] is none, weights[t] = 0, or all of the row's logits are -inf.  Such a token's row of
 * dlogits is +0 and its logp 0 (-inf in the last case), whatever its other inputs hold, NaN included; a row of the first
 * two kinds is not read.
 *   d_stats  5 floats: loss, sum weights pl, sum weights kl, tokens clipped (min took the clipped term), tokens counted
 *   d_dlogits  of the logits' type, in place (== d_logits, same stride) or apart; NULL: no gradient
 *   d_logp   n_tokens floats or NULL */
int dblp_policy_loss(int device, void* stream, uint64_t n_tokens, uint32_t vocab, const void* d_logits,
                     uint64_t logits_stride, int type, const int64_t* d_targets, const float* d_advantages,
                     const float* d_weights, const float* d_old_logp, const float* d_ref_logp, float clip_low,
                     float clip_high, float kl_coef, float grad_scale, void* d_dlogits, uint64_t dlogits_stride,
                     float* d_logp, float* d_stats, void* d_workspace, uint64_t workspace_bytes);
/* Bytes of the workspace of both; 0 if an argument is out of range. */
uint64_t dblp_logits_workspace(uint64_t n_tokens, uint32_t vocab);

const char* dblp_worker_error(void);

#ifdef __cplusplus
}
#endif
#endif /* DBLP_WORKER_H */

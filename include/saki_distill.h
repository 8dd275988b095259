/*
 * saki_distill.h -- supervision without the teacher's whole rows, and without the student's.
 *
 *   1. saki_top_logits: the k largest logits of every row, best first, with their tokens, and
 *      one number for all the others: what a teacher's pass keeps of a row.
 *   2. saki_distill_top: the divergence between a student's row and such a list, and its
 *      gradient with respect to the student's logits.
 *   3. saki_linear_ce: cross entropy of softmax(hidden weight^T) at a token of each row and the
 *      gradients of hidden and weight, without logits for every row and token in memory.
 *
 * Memory, streams, layout of logit rows, alignment and errors are those of saki.h: arrays are
 * the caller's device memory, calls only enqueue on `stream`, may be captured into a graph, and
 * allocate nothing; workspaces have any contents before and after a call, and calls that may run
 * at the same time need separate ones.  Their sizes are those of a call's own shapes: one of fewer rows may need more
 * (rows that are read in parts, logits that are kept), so a workspace for several shapes is as large as the largest of them.  Results do not depend on how rows are split into
 * calls and are the same bits for the same call, apart from saki_linear_ce's grad_weight, which is a sum over the
 * rows of a call, and from the order of 32-bit sums: how many rows a call has decides how its products are split, and
 * how long rows of few are read (rest_logit).  n_rows == 0: sums over the rows (loss_sum, grad_weight) are 0,
 * nothing else is written.
 */
#ifndef SAKI_DISTILL_H
#define SAKI_DISTILL_H

#include "saki.h"

#ifdef __cplusplus
extern "C" {
#endif

#define SAKI_MAX_TOP_K 256   /* longest list of top logits               */
#define SAKI_MAX_HIDDEN 65536 /* most elements of a hidden state          */

/* Operation codes for saki_workspace_bytes (vocab: entries of a row, for both). */
#define SAKI_OP_TOP_LOGITS 7
#define SAKI_OP_DISTILL_TOP 8

/* Row status beside those of saki.h: the row's list, token or weight cannot be used. */
#define SAKI_ROW_BAD_TARGET 4

/* The k largest logits of every row of x = logits[r, 0 .. vocab):
 *   top_logit[r, i]  the i-th largest logit (i < k), equal ones by ascending token
 *   top_token[r, i]  its token
 *   rest_logit[r]    tau log sum exp(x_j / tau) over all tokens that are not listed
 *                    (-infinity where every token is)
 * so that softmax(x / tau) gives the listed tokens and all others together the same shares as
 * softmax over the k + 1 numbers (top_logit, rest_logit) / tau.
 *   top_stride   elements between rows of top_logit and of top_token, >= k
 *   rest_logit, row_status [n_rows] may be NULL
 *   1 <= k <= min(SAKI_MAX_TOP_K, vocab); temperature tau > 0, at least 2^-64 and at most 2^64
 *   ws           ws_bytes >= saki_workspace_bytes(SAKI_OP_TOP_LOGITS, n_rows, vocab), 16-byte
 *                aligned (0 bytes for calls of many rows: NULL is fine then)
 * A row with a NaN or infinite logit gets NaN, -1, NaN and SAKI_ROW_NONFINITE. */
saki_status saki_top_logits(const void *logits, int32_t dtype, int64_t n_rows, int64_t vocab,
                            int64_t row_stride, int32_t k, float temperature, float *top_logit,
                            int32_t *top_token, int64_t top_stride, float *rest_logit,
                            uint8_t *row_status, void *ws, size_t ws_bytes, saki_stream_t stream);

/* A teacher's list for each row, as saki_top_logits writes it. */
typedef struct {
  const int32_t *token;    /* [n_rows, stride] distinct tokens, in any order; -1: no entry    */
  const float *logit;      /* [n_rows, stride] their logits (not read where the token is -1)  */
  const float *rest_logit; /* [n_rows] the others' logit, or NULL: -infinity for every row    */
  int64_t stride;          /* elements between rows, >= k                                     */
  int32_t k;               /* entries of a row, 1 .. SAKI_MAX_TOP_K (may be above vocab)      */
  int32_t reserved;        /* must be 0                                                       */
} saki_top_list;

#define SAKI_KL_FORWARD 0 /* KL(t || p): cover what the teacher holds likely          */
#define SAKI_KL_REVERSE 1 /* KL(p || t): the on-policy direction                      */

/* Divergence from a teacher's list.  Over the buckets b = the listed tokens, each by itself,
 * and one bucket R of all the other tokens:
 *   t = softmax over b of (logit, rest_logit) / tau      (the bucket R has rest_logit)
 *   p = softmax(student / tau), p_R = the sum of p over the tokens not listed
 *   forward  l = sum_b t_b log(t_b / p_b)     (terms of t_b = 0 are 0)
 *   reverse  l = sum_b p_b log(p_b / t_b)     (terms of p_b = 0 are 0)
 * and the gradient  grad[r, j] = grad_scale * d l_r / d student[r, j]
 *   forward  1/tau (p_j - t_j) at listed tokens, 1/tau (p_R - t_R) p_j / p_R at the others
 *   reverse  1/tau p_j (log(p_j / t_j) - l) at listed tokens, 1/tau p_j (log(p_R / t_R) - l) at the others
 * (no factor tau^2: put it into grad_scale where it is wanted).  Without rest_logit t_R = 0:
 * the list's own softmax against the student's whole row.
 *   valid_mask   [n_rows] (0 / non-zero) or NULL; rows with 0, and rows that list nothing and
 *                have rest_logit = -infinity or none, have loss 0 and gradient 0
 *   row_loss     [n_rows] unscaled l_r, or NULL
 *   loss_sum     one double: OVERWRITTEN with sum_r grad_scale * l_r, or NULL
 *   grad         [n_rows, grad_stride], grad_dtype F32 or BF16, or NULL; it may be the student's
 *                own buffer where both have the same dtype and stride
 *   row_status   [n_rows] or NULL
 *   ws           ws_bytes >= saki_workspace_bytes(SAKI_OP_DISTILL_TOP, n_rows, vocab), 8-byte aligned
 * Rows of valid_mask 0 are not looked at (status OK).  Others get NaN in loss and gradient and
 *   SAKI_ROW_NONFINITE   a student logit is NaN or infinite
 *   SAKI_ROW_BAD_TARGET  a token below -1, not below vocab, or listed twice; a logit or
 *                        rest_logit that is NaN or +infinity; a divergence that is infinite
 *                        (forward: a finite rest_logit where every token is listed; reverse: a
 *                        listed logit of -infinity, or a rest_logit of -infinity where not every
 *                        token is listed)
 * Reverse without rest_logit is SAKI_E_NULLPTR. */
saki_status saki_distill_top(const void *student, int32_t dtype, int64_t n_rows, int64_t vocab,
                             int64_t row_stride, const saki_top_list *list, float temperature,
                             int32_t direction, const uint8_t *valid_mask, float grad_scale,
                             float *row_loss, double *loss_sum, void *grad, int32_t grad_dtype,
                             int64_t grad_stride, uint8_t *row_status, void *ws, size_t ws_bytes,
                             saki_stream_t stream);

/* A student's head: logits = hidden weight^T. */
typedef struct {
  const void *hidden;    /* [n_rows, hidden_stride]                                            */
  const void *weight;    /* [vocab, weight_stride]                                             */
  int64_t hidden_stride; /* elements between rows; rows are 16-byte aligned                    */
  int64_t weight_stride;
  int64_t n_rows;
  int64_t vocab;         /* 1 .. SAKI_MAX_VOCAB                                                */
  int64_t hidden_size;   /* D, a multiple of 8, 8 .. SAKI_MAX_HIDDEN                           */
  int32_t dtype;         /* saki_dtype of hidden, weight and both gradients                    */
  int32_t reserved;      /* must be 0                                                          */
} saki_head;

/* l_r = -row_weight[r] log p_r(token[r]), p_r = softmax(hidden_r weight^T):
 *   grad_hidden[r] = grad_scale d l_r / d hidden[r]
 *                  = grad_scale row_weight[r] sum_v (p_r(v) - 1[v = token[r]]) weight[v]
 *   grad_weight[v] = grad_scale sum_r row_weight[r] (p_r(v) - 1[v = token[r]]) hidden[r]
 * (OVERWRITTEN, not added to).  With row_weight = 1 at corrections and the detached advantage A at accepted rows,
 * and token = the supervised token, this is the routed objective of saki_route_args. */
typedef struct {
  const int32_t *token;      /* [n_rows]                                                        */
  const float *row_weight;   /* [n_rows], or NULL: 1 for every row                              */
  const uint8_t *valid_mask; /* [n_rows] (0 / non-zero), or NULL                                */
  float grad_scale;
  uint32_t reserved;         /* must be 0                                                       */
  float *row_loss;           /* [n_rows] unscaled l_r, or NULL                                  */
  float *logp_token;         /* [n_rows] log p_r(token[r]), or NULL                             */
  double *loss_sum;          /* one double: OVERWRITTEN with sum_r grad_scale l_r, or NULL      */
  uint8_t *row_status;       /* [n_rows], or NULL                                               */
  void *grad_hidden;         /* [n_rows, grad_hidden_stride], or NULL                           */
  void *grad_weight;         /* [vocab, grad_weight_stride], or NULL                            */
  int64_t grad_hidden_stride;
  int64_t grad_weight_stride;
} saki_ce_args;

/* Cross entropy from hidden states.  The logits exist a tile at a time in registers; with gradients, those of calls
 * of at most 1 GiB of them (n_rows vocab 4 bytes) are kept in the workspace in between, others are computed a second
 * time, a piece of the vocabulary at a time.
 *   ws   ws_bytes >= saki_linear_ce_workspace_bytes(head, grads), 256-byte aligned
 * Rows of valid_mask 0 are not read: loss, logp_token and grad_hidden are 0 there, and they add
 * nothing to grad_weight, whatever they hold.  A token outside [0, vocab) or a row_weight that
 * is not finite gives the row NaN in its outputs and grad_hidden and SAKI_ROW_BAD_TARGET, and it
 * adds nothing to grad_weight if its hidden state is finite.  A row whose logits' log-sum-exp is not finite gets NaN
 * and SAKI_ROW_NONFINITE, and makes grad_weight NaN.  An element of weight that is not finite may do so to every row,
 * those whose logit there would be -infinity among them.
 * f32 elements of at least 2^128 (1 - 2^-9), about 3.396e38, count as infinite.
 * Rounding: products in 32 bits of bf16 or f32 elements; for the gradients row_weight (p - 1[..])
 * is rounded once to the inputs' type (f32: to 24 bits).  Where p_r(token[r]) is near 1, log p and p - 1 come from
 * the other tokens' sum: their errors are relative to themselves, beside what the logits' rounding makes.  n_rows < 2^31 / 256, and rows of hidden and weight
 * below 2^22 elements apart. */
saki_status saki_linear_ce(const saki_head *head, const saki_ce_args *args, void *ws,
                           size_t ws_bytes, saki_stream_t stream);

/* Bytes of workspace of one saki_linear_ce call with this head (its pointers are not looked at); grads: 1 with
 * grad_hidden, 2 with grad_weight, 3 with both, 0 with neither.  0 for a head the call refuses. */
size_t saki_linear_ce_workspace_bytes(const saki_head *head, int32_t grads);

#ifdef __cplusplus
}
#endif

#endif /* SAKI_DISTILL_H */

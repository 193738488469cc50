/*
 * sk_layer.h -- C ABI of libsk_layer.so: what a decoder step of several tenants' models has beside its products (superkernel.h) and
 * its attention (sk_cache.h) (MI355X, gfx950).
 *
 *   sk_norm_*    norms before and after a block with its gate and scales: a block's output joins the residual stream, which is normalised
 *                for the next block
 *   sk_moe_*     a whole mixture-of-experts layer for the rows of a step: router, choice of experts, their products, weighted sum
 *   sk_verify_*  drafted tokens verified against the target's probabilities from given random numbers, and one more token sampled
 *
 * As with the other operators a list of problems, one per tenant, is planned once and launched step after step (arXiv 1901.10008,
 * Sections 1 and 5.3: independent operators of several streams in one launch).  Inference only: there are no gradients.
 *
 * General rules
 *   - Statuses, sk_strerror and sk_last_error are those of superkernel.h.  No C++ exception crosses this boundary.  On error the
 *     output arguments are left untouched and nothing is launched.
 *   - Pointers of problems are DEVICE pointers borrowed from the caller until the launches that use them have completed.  The
 *     arrays of problems themselves are copied.
 *   - Row strides are in elements; 0 means packed.  Pointers are multiples of their element's size unless stated otherwise.
 *   - n_rows (norm, moe): a number on the device, read by every launch; rows from it on are left as they are.  Values outside [0, rows]
 *     are cut to it; null means `rows`.  So a plan serves every step with up to `rows` rows, also out of a HIP graph.  Inputs have `rows` rows whatever
 *     the number is: those behind it may be read.
 *   - Norm plans have no workspace: their launches may overlap, and be made by several threads at once.  Plans of the other two own a workspace, so
 *     their launches must not: those on one stream are ordered by it, a launch on another stream gives SK_ERR_BUSY while the last one
 *     has not completed (best effort; launches of a graph are not tracked, and its replays are the caller's to order).
 *   - Outputs of a plan (of one problem or of several) whose spans from first to last element intersect give SK_ERR_OVERLAP.  What outputs may share with
 *     inputs stands with each operator.
 *   - Plans created host_only (1) are checked and planned without a device; their launches give SK_ERR_STATE.
 */
#ifndef SK_LAYER_H
#define SK_LAYER_H

#include "superkernel.h"

#ifdef __cplusplus
extern "C" {
#endif

/* z; 1 / (1 + e^-z); z / (1 + e^-z); tanh(z); z/2 (1 + tanh(sqrt(2/pi) (z + 0.044715 z^3))); max(z, 0) */
typedef enum { SK_ACT_NONE = 0, SK_ACT_SIGMOID = 1, SK_ACT_SILU = 2, SK_ACT_TANH = 3, SK_ACT_GELU = 4, SK_ACT_RELU = 5 } sk_act;

typedef struct {
  int32_t host_only;
  int32_t workgroups; /* workgroups at a time that the products of sk_moe are cut for; 0 = as many as the device holds (the other operators have no use for it) */
  int32_t reserved[2];
} sk_layer_params;

void sk_layer_params_default(sk_layer_params *params);

/* ---- norms around a block -----------------------------------------------------------------------------------------------
 *
 * For every row:
 *     u    = block                                     or, with post = 1, N(block) * post_weight + post_bias
 *     u    = u * act(gate)                             if there is a gate
 *     r    = residual_scale * residual + block_scale * u
 *     residual_out = r
 *     next = N(r) * pre_weight + pre_bias
 * N(x) = x / sqrt(mean(x^2) + eps) (SK_NORM_RMS), or (x - mean(x)) / sqrt(mean((x - mean(x))^2) + eps) (SK_NORM_LAYER).  Missing (null)
 * weights count as 1, biases as 0, a missing residual as 0; block or residual may be missing, not both; of residual_out and next one may be.
 * All of it is fp32, sums included; each output is rounded once (next is made from r before its rounding).  Squares are summed as
 * they are, which values beyond 2^59 in size overflow and, with eps = 0, values below 2^-60 may vanish in.
 * residual_out may be residual itself (same address, type and stride), next may be block itself; otherwise outputs must not touch inputs.
 */
typedef enum { SK_NORM_RMS = 0, SK_NORM_LAYER = 1 } sk_norm_kind;

typedef struct {
  int32_t dtype;          /* of block, gate, weights, biases and next: SK_F32, SK_BF16 or SK_F16     */
  int32_t residual_dtype; /* of residual and residual_out: dtype or SK_F32                            */
  int32_t kind;           /* sk_norm_kind                                                             */
  int32_t rows, dim;      /* dim 1 .. 32768                                                           */
  int32_t post;           /* 1: the block's output is normalised                                      */
  int32_t gate_act;       /* sk_act                                                                    */
  int32_t gate_rows;      /* 1: a gate for every row, 0: one for all                                   */
  float eps;
  float residual_scale, block_scale; /* 0 = 1 */
  int32_t reserved;                  /* 0     */
  int64_t block_stride, gate_stride, residual_stride, residual_out_stride, next_stride; /* between rows */
  const int32_t *n_rows;
  const void *block, *gate, *residual;
  const void *post_weight, *post_bias, *pre_weight, *pre_bias;
  void *residual_out, *next;
} sk_norm_problem;

typedef struct sk_norm_plan sk_norm_plan; /* opaque, owned by the library */

/*
 * Errors: SK_ERR_INVALID_ARG (null pointers, sizes < 1, fields outside their range, a stride below dim), SK_ERR_UNSUPPORTED (other
 * types, dim > 32768, pointers that are no multiples of their elements, rows beyond a launch's grid), SK_ERR_OVERLAP, SK_ERR_ALLOC, SK_ERR_HIP.
 */
sk_status sk_norm_plan_create(const sk_norm_problem *problems, int32_t n, const sk_layer_params *params, sk_norm_plan **out);
/* Waits for the device's work and frees the plan; null is accepted. */
sk_status sk_norm_plan_destroy(sk_norm_plan *plan);
/* One kernel launch for up to 16 problems of one kind of work (rows of up to 4096, 8192 or more elements; of 2048 rows or more up to 256, 1024 or 2048; all of
   them if they have 1024 rows or fewer). */
sk_status sk_norm_launch(sk_norm_plan *plan, void *hip_stream);

/* ---- mixture-of-experts layer -------------------------------------------------------------------------------------------
 *
 * For every row x of `dim` elements:
 *     l_e = x . router_e                                of every expert e
 *     s   = softmax(l)  (SK_MOE_SOFTMAX)   or   s_e = 1 / (1 + e^-l_e)  (SK_MOE_SIGMOID)
 *     the top_k experts with the largest s_e + router_bias_e (SK_MOE_SOFTMAX without bias: with the largest l_e, which is the same order but tells apart
 *     what the softmax rounds to the same), in that order; equal ones by their number; NaN below all others
 *     w_e = scale * s_e, with normalize = 1 divided by the sum of the chosen s_e
 *     h_e = act(gate_e . x) * (up_e . x),               without gate: act(up_e . x)
 *     out = sum over the chosen, w_e * (down_e . h_e), and the same of the shared expert, which every row passes, with w = 1
 * Scores are computed in 64 bits, so that the choice between experts whose scores are next to each other does not depend on the order of sums.
 * out may be x, or touch it: it is written when all of a plan's x have been read.  expert_ids and expert_weights must not touch inputs.
 * Products of the experts are summed in fp32, h is fp32 and not rounded to dtype, outputs are summed in fp32 and rounded once.  Each row's result depends on that row and the weights alone, up to the order of sums.
 * The weights are read once for up to 32 rows of an expert; made for the rows of decoder steps, it takes any number.  A row's sum goes over its experts
 * in the order in which they were chosen, the shared one last.
 */
typedef enum { SK_MOE_SOFTMAX = 0, SK_MOE_SIGMOID = 1 } sk_moe_scoring;

typedef struct {
  int32_t dtype;        /* SK_BF16 or SK_F16: x, experts' weights, out                             */
  int32_t router_dtype; /* dtype or SK_F32                                                         */
  int32_t rows, dim;    /* dim a multiple of 8                                                      */
  int32_t experts, top_k; /* 1 .. 512; 1 .. 32, at most `experts`                                   */
  int32_t ffn;          /* width of an expert, a multiple of 8                                      */
  int32_t shared_ffn;   /* width of the shared expert, a multiple of 8; 0 = none                    */
  int32_t act;          /* sk_act                                                                   */
  int32_t scoring;      /* sk_moe_scoring                                                           */
  int32_t normalize;    /* 0 or 1                                                                   */
  float scale;          /* 0 = 1                                                                    */
  int64_t x_stride, out_stride, router_stride;       /* between rows                                */
  int64_t up_expert_stride, down_expert_stride;      /* between experts (gate's is up's); 0 = packed */
  int64_t up_row_stride, down_row_stride;            /* between rows of weights (gate's is up's)     */
  const int32_t *n_rows;
  const void *x;
  const void *router;                                 /* [experts][dim]                             */
  const float *router_bias;                           /* [experts] or null                          */
  const void *gate, *up, *down;                       /* [experts][ffn][dim] (gate may be null), [experts][dim][ffn] */
  const void *shared_gate, *shared_up, *shared_down;  /* the same of the shared expert, packed; with a gate if the experts have one */
  void *out;
  int32_t *expert_ids;                                /* [rows][top_k], packed, or null             */
  float *expert_weights;                              /* [rows][top_k], packed, or null             */
} sk_moe_problem;

typedef struct sk_moe_plan sk_moe_plan; /* opaque, owned by the library */

/*
 * Errors as above; also SK_ERR_UNSUPPORTED: SK_F32, dim or widths that are no multiples of 8, x, weights, router and out or their strides
 * that are no multiples of 16 bytes, more than 512 experts or 32 chosen, dim or a stride of x from 2^21 on, widths beyond 2^24 or strides of
 * rows of weights from 2^26 on; SK_ERR_ALLOC also where the workspace does not fit the device.
 */
sk_status sk_moe_plan_create(const sk_moe_problem *problems, int32_t n, const sk_layer_params *params, sk_moe_plan **out);
/* Waits for the plan's launches and frees it; null is accepted. */
sk_status sk_moe_plan_destroy(sk_moe_plan *plan);
sk_status sk_moe_launch(sk_moe_plan *plan, void *hip_stream);
/* Kernel launches that sk_moe_launch makes, and bytes of the plan's workspace (either may be null). */
sk_status sk_moe_plan_info(const sk_moe_plan *plan, int32_t *launches, int64_t *workspace_bytes);

/* ---- verification of drafted tokens -------------------------------------------------------------------------------------
 *
 * Rows of logits belong to sequences as in sk_cache.h: sequence s has rows first_row[s] .. first_row[s+1]-1 (entries that do not decrease; none for a
 * sequence is fine; values are cut to [0, rows]).  Row first_row[s] + i gives the target's distribution of the token behind the sequence's i-th token of this step; drafted[row] is the
 * token that was drafted there, for all rows of the sequence but the last, which has no draft.  With one row a sequence this is plain sampling.
 *     p = softmax(logits / temperature), of the row
 *     q = softmax(draft_logits / temperature); without draft_logits the draft was certain of its token: q = 1 there, 0 elsewhere
 *     i = 0, 1, ..: a drafted token d is accepted while  accept_random[row] * q(d) < p(d)
 *     at the first row that does not accept: one more token is sampled from max(p - q, 0) (from p where that is 0 everywhere, or where d is no
 *     token); after the last accepted draft from p of the last row.
 * Sampling: the first token k with  sum_{j <= k} w_j > sample_random[s] * sum_j w_j  (the last with w > 0 if rounding leaves none).
 * Temperature 0 (or below, or NaN): p is 1 at the first of the largest logits, and the draft is certain of its token.
 * Outputs must not touch inputs of the plan, drafted among them (SK_ERR_OVERLAP): sequences and parts of a row are decided side by side.
 * Results: tokens[row] = accepted drafts, then the sampled token, then -1 up to the sequence's last row; accepted[s] = number of accepted
 * drafts.  Rows of no sequence are left as they are; a sequence without rows accepts 0.
 * A logit of -infinity is a token of probability 0.  A row of logits that holds NaN or +infinity, or -infinity only, has no distribution: it accepts
 * nothing, and its sampled token is -1.  A row of draft_logits without a distribution counts as certain.  Drafted numbers outside [0, vocab) are
 * rejected.  Random numbers are in [0, 1); others are cut to it, NaN to 0.
 * Probabilities and sums are computed in 64 bits, so that the tokens do not depend on the order of sums (up to errors of some 10^-12).
 */
typedef struct {
  int32_t dtype;     /* of logits and draft_logits: SK_F32, SK_BF16 or SK_F16 */
  int32_t sequences, rows;
  int32_t vocab;
  float temperature; /* where temperatures is null                             */
  int32_t reserved;  /* 0                                                      */
  int64_t logits_stride, draft_stride; /* between rows */
  const int32_t *first_row;    /* [sequences + 1] */
  const void *logits;          /* [rows][vocab]   */
  const int32_t *drafted;      /* [rows], or null: no row has a draft's token (all drafted numbers count as outside the vocabulary) */
  const void *draft_logits;    /* [rows][vocab] or null; the last row of a sequence is not read */
  const float *temperatures;   /* [sequences] or null */
  const float *accept_random;  /* [rows]; may be null if drafted is */
  const float *sample_random;  /* [sequences]     */
  int32_t *tokens;             /* [rows]          */
  int32_t *accepted;           /* [sequences]     */
} sk_verify_problem;

typedef struct sk_verify_plan sk_verify_plan; /* opaque, owned by the library */

sk_status sk_verify_plan_create(const sk_verify_problem *problems, int32_t n, const sk_layer_params *params, sk_verify_plan **out);
/* Waits for the plan's launches and frees it; null is accepted. */
sk_status sk_verify_plan_destroy(sk_verify_plan *plan);
sk_status sk_verify_launch(sk_verify_plan *plan, void *hip_stream);
/* Kernel launches that sk_verify_launch makes, and bytes of the plan's workspace (either may be null). */
sk_status sk_verify_plan_info(const sk_verify_plan *plan, int32_t *launches, int64_t *workspace_bytes);

#ifdef __cplusplus
}
#endif
#endif /* SK_LAYER_H */

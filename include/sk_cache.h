/*
 * sk_cache.h -- C ABI of libsk_cache.so: attention's side of decoder layers over paged key/value caches, for the models of
 * several tenants at once (MI355X, gfx950).
 *
 * superkernel.h runs the products of several streams' models in one launch (arXiv 1901.10008, Sections 1 and 5.3).  Between
 * two products of a decoder layer stand these operators, coalesced in the same way: a list of problems, one per tenant, is
 * planned once and launched step after step.
 *
 *   sk_attn_append  heads of queries and keys normalised and rotated to their positions, keys and values written to their pages
 *   sk_attn_launch  causal attention over the pages, with an optional sliding window and first tokens that stay visible (sinks);
 *                   prompts, chunks of prompts and single tokens may stand side by side in one problem
 *   sk_pages_*      which sequence holds which page: growing, forking (shared pages, copied when written), freeing, compacting;
 *                   and the copies of pages
 *
 * Inference only, like the rest of the framework: there are no gradients.
 *
 * General rules
 *   - Statuses, sk_strerror and sk_last_error are those of superkernel.h.  No C++ exception crosses this boundary.  On error the
 *     output arguments are left untouched and nothing is launched.
 *   - Pointers of sk_attn_problem are DEVICE pointers borrowed from the caller until the launches that use them have completed.
 *     The sk_attn_problem array itself is copied.
 *   - What changes from step to step is read on the device: the lengths, the rows of each sequence and the page table.  A
 *     plan therefore serves step after step, and its launches may be captured into a HIP graph (outside a capture an event
 *     is recorded with them).  The host states only upper bounds (rows, max_new, pages_per_sequence), which fix the grids.
 *   - A plan owns a workspace: its attention launches must not overlap.  Those on one stream are ordered by it; sk_attn_launch on
 *     another stream gives SK_ERR_BUSY while the last one has not completed (best effort; launches of a graph are not tracked).
 */
#ifndef SK_CACHE_H
#define SK_CACHE_H

#include "superkernel.h"

#ifdef __cplusplus
extern "C" {
#endif

/*
 * One tenant's layer: its cache, what is new in this step, and what is computed.
 *
 * Cache.  K and V are arrays of num_pages pages; a page holds page_tokens tokens of every key-value head.  Element e of token
 *   t of head h of page p stands at  p*page_stride + h*kv_head_stride + t*token_stride + e  elements behind k (and v).  All three
 *   strides 0: packed [page][head][token][dim].  Token i of sequence s lies in page page_table[s*pages_per_sequence + i / page_tokens],
 *   place i % page_tokens.  Entries of the table, and places of a page, behind a sequence's last token may hold anything.
 * Step.  lengths[s]: tokens of sequence s, those of this step included.  The new ones are the rows first_row[s] ..
 *   first_row[s+1]-1 of qkv, q and out (first_row has sequences + 1 entries that do not decrease; none for a sequence is fine), and
 *   the last ones of the sequence: row first_row[s] + t is the token at position lengths[s] - (first_row[s+1] - first_row[s]) + t.
 *   Values beyond the bounds given to the plan are cut to them on the device (lengths to pages_per_sequence * page_tokens, rows to
 *   `rows`); tokens whose page number is outside [0, num_pages) count as not there.  sk_attn_launch leaves the rows of new tokens beyond
 *   max_new of a sequence as they are; sk_attn_append, whose grid does not depend on max_new, appends all new tokens.
 *
 * sk_attn_append, for every new row x = qkv[row] (q_heads query heads, then kv_heads key heads, then kv_heads value heads, of
 *   head_dim elements each, rows qkv_row_stride elements apart, 0 = packed) at position p:
 *     y = x * w / sqrt(mean(x^2) + eps)           per head; queries with q_weight, keys with k_weight; null: y = x
 *     (a, b) -> (a*cos - b*sin, b*cos + a*sin)    for the pairs of the first rotary_dim elements: elements i and i + rotary_dim/2,
 *                                                 or with neighbours = 1 elements 2i and 2i+1, with cos = cos[p*rotary_dim/2 + i]
 *   Queries go to q, keys and values into their pages.  fp32 inside, one rounding at the end; the squares are summed in fp32 as they
 *   are, which elements beyond 2^59 in size overflow and, with eps = 0, elements below 2^-60 may vanish in.  cos and sin have `positions`
 *   rows, at least pages_per_sequence * page_tokens.  Rows at a position below 0 (more new rows than tokens) or in no page are
 *   not appended; their queries are rotated as at the nearest position.
 *
 * sk_attn_launch, for query head h (key-value head h / (q_heads / kv_heads)) of every new row at position p:
 *     out = sum_j softmax_j(scale * q.k_j) v_j    over the tokens j <= p with: window == 0, or p - j < window, or j < sinks
 *   A row that sees nothing gets zeros, and so does one all of whose scores are -infinity: such a score is a weight of zero, as one
 *   that is hidden.  Keys and values that a row does not see do not enter its result, whatever they hold.
 *   Scores, the softmax's running maximum and sum, and the output's sums are fp32; the softmax's weights are rounded to dtype
 *   for the matrix units (their sum is not).
 *
 * q and out: element e of head h of a row stands at row*row_stride + h*head_stride + e; both strides 0: packed [row][head][dim].
 * qkv may be null (then sk_attn_append gives SK_ERR_STATE), so may out (then sk_attn_launch does).
 */
typedef struct {
  int32_t dtype;                        /* SK_BF16 or SK_F16: queries, caches and outputs                       */
  int32_t q_heads, kv_heads, head_dim;  /* q_heads a multiple of kv_heads; head_dim a multiple of 8, 8 .. 256   */
  int32_t page_tokens;                  /* a power of two, 16 .. 65536                                           */
  int32_t num_pages;
  int32_t sequences, pages_per_sequence;
  int32_t rows;     /* rows that qkv, q and out have room for                                                   */
  int32_t max_new;  /* at most that many new rows for one sequence; 0 = rows                                    */
  int32_t window;   /* tokens a row sees back from itself, itself included; 0 = all                             */
  int32_t sinks;    /* first tokens that stay visible beyond the window                                         */
  int32_t rotary_dim;  /* even, 0 .. head_dim                                                                   */
  int32_t neighbours;  /* which elements are pairs, see above                                                   */
  int32_t positions;   /* rows of cos and sin                                                                   */
  float eps;
  float scale;         /* of the scores, up to 2.3e38; 0 = 1 / sqrt(head_dim)                                   */
  int32_t reserved;    /* 0                                                                                     */
  int64_t page_stride, kv_head_stride, token_stride;
  int64_t qkv_row_stride, q_row_stride, q_head_stride, out_row_stride, out_head_stride;
  void *k, *v;
  const int32_t *page_table; /* [sequences][pages_per_sequence] */
  const int32_t *lengths;    /* [sequences]                     */
  const int32_t *first_row;  /* [sequences + 1]                 */
  const void *qkv;
  const void *q_weight, *k_weight; /* head_dim elements of dtype, or null */
  const float *cos, *sin;          /* [positions][rotary_dim / 2]         */
  void *q;
  void *out;
} sk_attn_problem;

typedef struct {
  int32_t host_only;  /* 1: check and plan on the host only (launches then give SK_ERR_STATE)                     */
  int32_t workgroups; /* workgroups at a time that the work is split for; 0 = as many as the device holds         */
  int32_t reserved[2];
} sk_attn_params;

typedef struct sk_attn_plan sk_attn_plan; /* opaque, owned by the library */

void sk_attn_params_default(sk_attn_params *params);

/*
 * Plan for n problems (n = 0: launches do nothing).  Errors: SK_ERR_INVALID_ARG (null pointers, sizes < 1, strides that let
 * heads or tokens overlap, cos and sin with too few rows), SK_ERR_UNSUPPORTED (SK_F32; a head_dim that is no multiple of
 * 8 or larger than 256; page_tokens that is no power of two from 16 on; pointers or strides that are no multiples of 16 bytes;
 * sequences of 2^31 tokens and more; more than 2^20 sequences; more than 2^30 heads; a token_stride of 2^26 elements and more;
 * more units of work than the 2^24 - 1 workgroups of a launch), SK_ERR_OVERLAP (what q or out of two problems, or of
 * one, span from their first to their last element intersects), SK_ERR_ALLOC, SK_ERR_HIP.
 */
sk_status sk_attn_plan_create(const sk_attn_problem *problems, int32_t n, const sk_attn_params *params, sk_attn_plan **out);
/* Waits for the plan's launches and frees it; null is accepted. */
sk_status sk_attn_plan_destroy(sk_attn_plan *plan);
/* Norms, rotation and append of every problem: one kernel launch. */
sk_status sk_attn_append(sk_attn_plan *plan, void *hip_stream);
/* Attention of every problem: one kernel launch for all problems with heads of up to 128 elements, one for those with larger ones. */
sk_status sk_attn_launch(sk_attn_plan *plan, void *hip_stream);
/* Kernel launches that sk_attn_launch makes, and bytes of the plan's workspace (either may be null). */
sk_status sk_attn_plan_info(const sk_attn_plan *plan, int32_t *launches, int64_t *workspace_bytes);

/*
 * Pages: the host's account of which sequence holds which page of a set of arrays (all layers' K and V pages go together: a
 * page number means the same place in every array).
 *
 * sk_pages_create   an account of num_pages free pages for `sequences` sequences of at most pages_per_sequence pages.
 * sk_pages_resize   n sequences (no number twice) get room for tokens[i] tokens.  Growing takes the lowest free pages, sequence after
 *                   sequence; a last page that is not full and shared with another sequence is copied to a page of the sequence's own first,
 *                   since its next token will be written there.  Shrinking gives pages back (0: all of them).  If there are too few pages
 *                   SK_ERR_ALLOC, and nothing has changed.
 * sk_pages_fork     the n sequences to[] (empty, no number twice) become continuations of `from`: they share all of its pages.
 * sk_pages_compact  moves the pages in use to the lowest numbers.
 * sk_pages_apply    makes the device follow: the page copies that the calls since the last sk_pages_apply have called for, in every
 *                   array, in an order in which none overwrites what another still has to read; and the rows that have changed of
 *                   the device's page table, [sequences][pages_per_sequence] int32 with -1 where a sequence has no page.  Without a table
 *                   (null) the rows wait for a call that has one; without arrays the copies count as made.  One kernel launch
 *                   where no copy depends on another.  Asynchronous; not inside a stream capture (SK_ERR_STATE).  After SK_ERR_HIP
 *                   some of the copies may have been made and others not.
 * sk_pages_state    counts; row (of pages_per_sequence entries) and tokens of a sequence.  Any pointer may be null.
 * An account belongs to one host thread at a time.
 *
 * sk_pages_copy     the copies alone, for programs with an account of their own: page from[i] to page to[i] in every array, all
 *                   at once: no number may stand twice in to[], nor in both lists (SK_ERR_OVERLAP); from[i] may repeat.  May be captured.
 */
typedef struct {
  void *base;         /* device; a multiple of 16                                 */
  int64_t page_bytes; /* distance of two pages, and bytes of one; a multiple of 16, at most 2^38 */
} sk_page_array;

typedef struct sk_pages sk_pages; /* opaque, owned by the library */

sk_status sk_pages_create(int32_t num_pages, int32_t page_tokens, int32_t sequences, int32_t pages_per_sequence, sk_pages **out);
sk_status sk_pages_destroy(sk_pages *pages);
sk_status sk_pages_resize(sk_pages *pages, const int32_t *sequences, const int32_t *tokens, int32_t n);
sk_status sk_pages_fork(sk_pages *pages, int32_t from, const int32_t *to, int32_t n);
sk_status sk_pages_compact(sk_pages *pages);
sk_status sk_pages_apply(sk_pages *pages, const sk_page_array *arrays, int32_t n_arrays, int32_t *page_table, void *hip_stream);
sk_status sk_pages_state(const sk_pages *pages, int32_t *free_pages, int32_t *pending_copies, int32_t sequence, int32_t *tokens, int32_t *row);
sk_status sk_pages_copy(const sk_page_array *arrays, int32_t n_arrays, int32_t num_pages, const int32_t *from, const int32_t *to, int32_t n,
                        void *hip_stream);

#ifdef __cplusplus
}
#endif
#endif /* SK_CACHE_H */

/*
 * zo_forward.h -- operators of a forward point: what a decoder computes
 * between the weights that zo_perturb moves and the loss that zo_precondition
 * reads (Algorithm 1 evaluates L at theta, theta + eps z_k and theta - eps
 * z_k). The matrix products in between are the caller's.
 *
 *   zo_rotary_table      angles of every position, once per model
 *   zo_document_spans    the keys that each packed token sees, once per batch
 *   zo_rotate_heads      per-head norms and rotation of queries and keys; into a paged cache
 *   zo_attention         attention of packed documents
 *   zo_attention_decode  attention of one new token per sequence over a paged cache
 *   zo_token_loss        -log p of every target token, summed into a loss table
 *
 * Conventions are those of zo.h: device memory owned by the caller, calls that
 * only enqueue work on `stream` of the current device, zo_status returned,
 * argument errors found before anything is enqueued, nothing allocated and
 * nothing kept. The method estimates its gradient from losses, so there are
 * no backward passes.
 *
 * Data-dependent errors (a position outside the table, a page outside the
 * cache, a target outside the vocabulary) cannot be seen on the host: the
 * outputs that depend on them are NaN, so the loss is, zo_precondition
 * reports ZO_ERR_NONFINITE and the update is skipped. No access leaves the
 * given ranges.
 *
 * Arithmetic. Values are read as fp32; norms, scores, softmax statistics and
 * sums are fp32 (fp64 across tokens) and each output is rounded once. One
 * exception, in zo_attention and zo_attention_decode on 16-bit types: the
 * softmax's weights are rounded to that type for the tensor cores (in fp16 one
 * below 2^-21 of its row's largest loses bits, and one below 2^-32 is lost).
 *
 * Strides are in elements; the elements of one head are contiguous. An output
 * over an input or another output, or with rows or heads over one another, is
 * ZO_ERR_ARG as far as strides show it (layouts that interleave by unlike
 * strides are the caller's to keep apart).
 */
#ifndef ZO_FORWARD_H_
#define ZO_FORWARD_H_

#include "zo.h"

#ifdef __cplusplus
extern "C" {
#endif

/* Largest head size, and largest number of query heads. */
#define ZO_MAX_HEAD_DIM 256
#define ZO_MAX_HEADS 1024

/* Tokens of heads: element d of head h of token t at ptr[t * token + h * head + d]. */
typedef struct {
  void* ptr;
  int64_t token;
  int64_t head;
} zo_rows;

/* A paged cache: row r of page p, head h at ptr[p * page + r * token + h * head]. */
typedef struct {
  void* ptr;
  int64_t page;
  int64_t token;
  int64_t head;
} zo_pages;

/* ---------------------------------------------------------------------------
 * zo_rotary_table -- table[p][0..R/2) = magnitude cos(p w_i), table[p][R/2..R)
 * = magnitude sin(p w_i), i < R/2, for positions p < rows; fp64 inside, one
 * rounding. w_i = base^(-2i/R); with scale s > 1 for contexts s times the
 * `original` one, each frequency is interpolated by how many turns it makes
 * in the original context, t_i = original w_i / (2 pi):
 *   w_i <- w_i ((1 - g) / s + g),  g = clamp((t_i - low) / (high - low), 0, 1)
 * (interpolation by parts, Peng et al., "YaRN", arXiv 2309.00071, Sec. 3.2).
 * original = 0: every frequency is divided by s.
 *   table       fp32 [rows][rotary_dim]
 *   rotary_dim  R, even, 2 .. ZO_MAX_HEAD_DIM
 * ------------------------------------------------------------------------- */
int zo_rotary_table(float* table, int64_t rows, int32_t rotary_dim, double base, double scale, int64_t original,
                    double low, double high, double magnitude, void* stream);

/* ---------------------------------------------------------------------------
 * zo_document_spans -- which keys each query row sees, for documents packed
 * one after another.
 *   q_starts, k_starts  int32 [docs + 1], ascending: document i holds query
 *                       rows q_starts[i] .. q_starts[i+1] - 1 and keys
 *                       k_starts[i] .. (k_starts may be q_starts). Its queries
 *                       are its last keys: with more keys than queries the
 *                       first ones were there before, with fewer the first
 *                       rows see nothing.
 *   prefix              int32 [docs] or NULL: so many of a document's first
 *                       keys are seen from all of its rows; every other key
 *                       from its own row on (causal)
 *   spans               out, int32 [3][tokens]: first key, end of the keys, own
 *                       key. Rows in no document see nothing (0, 0, 0).
 * ------------------------------------------------------------------------- */
int zo_document_spans(const int32_t* q_starts, const int32_t* k_starts, const int32_t* prefix, int32_t docs,
                      int32_t* spans, int64_t tokens, void* stream);

/* ---------------------------------------------------------------------------
 * zo_rotate_heads -- for up to three parts (queries, keys, values) of one
 * fused projection, in one pass:
 *   y = x                                             without a weight
 *   y = x / sqrt(mean_d x^2 + eps) * weight           with one (per head)
 * then, with ZO_HEADS_ROTATE, the first R elements are turned in pairs by the
 * table's row of the token's position:
 *   (y_a, y_b) <- (y_a cos_i - y_b sin_i, y_b cos_i + y_a sin_i)
 * where pair i is (i, i + R/2) under ZO_ROTARY_HALF and (2i, 2i + 1) under
 * ZO_ROTARY_INTERLEAVED. With ZO_HEADS_SLOTTED token t goes to row slots[t] %
 * page_size of page slots[t] / page_size of `out` (nowhere if slots[t] is
 * negative or not below n_slots), else to row t (out_page is not used).
 * A part may be done in place (out = in, same strides; with slots each token to
 * its own row); else an output overlaps no input, and never another output.
 *   weight        one per element of a head, of type weight_dtype, or NULL
 *   positions, slots  int32 or int64 by index_bytes (4 or 8); needed by the
 *                 parts that rotate / are slotted
 *   table         fp32 [table_rows][rotary_dim], zo_rotary_table's layout
 * ------------------------------------------------------------------------- */
#define ZO_HEADS_ROTATE 1
#define ZO_HEADS_SLOTTED 2
#define ZO_ROTARY_HALF 0
#define ZO_ROTARY_INTERLEAVED 1

typedef struct {
  zo_rows in;
  zo_pages out;
  const void* weight;
  int32_t weight_dtype;
  int32_t heads;
  int32_t flags;
  int32_t reserved; /* 0 */
} zo_head_part;

int zo_rotate_heads(const zo_head_part* parts, int32_t n_parts, int64_t tokens, int32_t head_dim, int32_t dtype,
                    const float* table, int64_t table_rows, int32_t rotary_dim, int32_t layout, const void* positions,
                    const void* slots, int32_t index_bytes, int64_t n_slots, int64_t page_size, float eps,
                    void* stream);

/* ---------------------------------------------------------------------------
 * zo_attention -- for every query row i and head h, over the keys j in
 * [first_i, end_i) (clipped to the keys there are) of key-value head
 * h / (heads / kv_heads):
 *   s_j = scale q_i . k_j;  softcap > 0: s_j = softcap tanh(s_j / softcap)
 *   slopes given: s_j = s_j - slopes[h] |self_i - j|
 *   out_i = sum_j exp(s_j) v_j / sum_j exp(s_j);  lse_i = log sum_j exp(s_j)
 * A row that sees nothing, or only scores of -inf, gets out = 0 and lse = -inf.
 * What lies at keys that a row does not see (NaN, infinities, memory never
 * written) does not reach its result. A column of out in which a row sees a
 * value that is not finite is not finite; whether it is NaN or an infinity is
 * left open.
 *   spans   int32 [3][q_tokens], zo_document_spans's or the caller's own; the
 *           third row (self) is read with slopes only
 *   slopes  fp32 [heads] or NULL
 *   lse     fp32 [heads][q_tokens] or NULL
 * out overlaps no input.
 * ------------------------------------------------------------------------- */
int zo_attention(const zo_rows* q, const zo_rows* k, const zo_rows* v, const zo_rows* out, int64_t q_tokens,
                 int64_t k_tokens, int32_t heads, int32_t kv_heads, int32_t head_dim, int32_t dtype,
                 const int32_t* spans, float scale, float softcap, const float* slopes, float* lse, void* stream);

/* ---------------------------------------------------------------------------
 * zo_attention_decode -- zo_attention of one query row per sequence, over the
 * lengths[b] keys of sequence b, of which the last is the row's own: key t is
 * row t % page_size of page pages[b * pages_stride + t / page_size] of the
 * caches. A length of zero or less gives a row that sees nothing; a page
 * outside 0 .. n_pages - 1, or a length above max_pages * page_size (or 2^31 -
 * 65), NaN.
 * What lies in a page beyond the length does not reach the result.
 *   q, out  row b is sequence b's; out may be q (same strides) and overlaps
 *           nothing else
 *   lse     fp32 [batch][heads] or NULL
 * ------------------------------------------------------------------------- */
int zo_attention_decode(const zo_rows* q, const zo_pages* k, const zo_pages* v, const zo_rows* out, int64_t batch,
                        int32_t heads, int32_t kv_heads, int32_t head_dim, int32_t dtype, const int32_t* pages,
                        int64_t pages_stride, int64_t max_pages, int64_t n_pages, int32_t page_size,
                        const int32_t* lengths, float scale, float softcap, const float* slopes, float* lse,
                        void* stream);

/* ---------------------------------------------------------------------------
 * zo_token_loss -- nll_t = log sum_v exp(x_tv) - x_t,target_t and their sum
 * over the counted tokens (those whose target is not negative; the others have
 * nll 0 and their logits are not read). The sum is formed in fp64 in an order
 * that depends on `tokens` alone.
 *   logits, row  [tokens][vocab], `row` elements from one token to the next
 *   targets      int32 or int64 by target_bytes
 *   flags        ZO_LOSS_MEAN: the sum divided by the counted tokens (NaN if
 *                there are none); ZO_LOSS_ADD: added to *loss (Algorithm 1 sums
 *                over micro-batches); ZO_LOSS_F32: loss is fp32
 *   loss         one fp64 (or fp32) value, e.g. an entry of the K x 3 table
 *   nll          fp32 [tokens] or NULL
 *   workspace    zo_token_loss_workspace_size(tokens) bytes, 8-byte aligned
 * ------------------------------------------------------------------------- */
#define ZO_LOSS_MEAN 1
#define ZO_LOSS_ADD 2
#define ZO_LOSS_F32 4

int64_t zo_token_loss_workspace_size(int64_t tokens);
int zo_token_loss(const void* logits, int64_t row, int64_t tokens, int64_t vocab, int32_t dtype, const void* targets,
                  int32_t target_bytes, int32_t flags, void* loss, float* nll, void* workspace,
                  int64_t workspace_bytes, void* stream);

#ifdef __cplusplus
}
#endif

#endif /* ZO_FORWARD_H_ */

/*
 * asymspec_serving.h -- C ABI of the operators around the verification step.
 *
 * Between two calls of the step of asymspec.h a serving loop constrains the logits that
 * go into it (penalties for repeated tokens, biases, grammar masks), rolls its paged
 * key-value caches back to the accepted length and gets slots for the next round's
 * tokens, writes their keys and values there, and attends over the pages.  The
 * accepted lengths stay on the GPU: none of these calls needs the host to read them,
 * and a whole round can be captured in a CUDA graph.
 *
 * The conventions of asymspec.h hold: arrays are caller-owned device pointers that
 * the library never retains, structs are host memory read during the call, work
 * is enqueued on `stream` and nothing is allocated, host-detectable errors are returned
 * before anything is enqueued, and a problem in the data never traps: it sets a bit
 * of the optional device error word, and what it means for the result is stated below.
 * Error words are OR-ed into; the caller clears them.  Strides count elements.
 */
#ifndef ASYMSPEC_SERVING_H
#define ASYMSPEC_SERVING_H

#include "asymspec.h"

#ifdef __cplusplus
extern "C" {
#endif

/* ---- device error-word bits, beside those of asymspec.h --------------------- */
#define ASYMSPEC_DATA_BAD_PENALTY 0x40u /* a repetition penalty that is not finite and positive,
                                           or a frequency or presence penalty that is not finite */
#define ASYMSPEC_DATA_BAD_LENGTH 0x80u  /* a length or offset that is negative or past its array */
#define ASYMSPEC_DATA_BAD_INDEX 0x100u  /* a mask row, block or slot that does not exist */
#define ASYMSPEC_DATA_NO_BLOCKS 0x200u  /* a request that the pool had no blocks for */

/* ---- constrained logits ----------------------------------------------------
 * For each of B requests and P positions (a round's K drafts and its bonus position, P =
 * K + 1, or P = 1 for one drafted position), out[b][k][v] from logits[b][k][v]:
 *
 *   seen(v)  v is in the request's history (prompt or output) or among the drafts before k
 *   n(v)     how often v is in the output part of the history and among the drafts before k
 *   y  = x;  if seen(v): y = x > 0 ? x / repetition : x * repetition
 *   y -= frequency * n(v) + presence * [n(v) > 0]
 *   y += bias(v)
 *   out = allowed(v) ? y : mask_value
 *
 * computed in fp32 and rounded once, to `dtype`.  A finite logit stays finite (a result
 * beyond the type's range becomes its largest or lowest value), so that a logit masked
 * before at the lowest value stays there; a NaN or an infinity stays what it is, and a NaN
 * bias makes a NaN, unless the mask replaces it.  An entry that nothing changes is copied bit for bit.  The same
 * constraints belong on the step's three logit tensors and on the drafter's rows.
 * Every group of members may be absent (NULL).
 */
typedef struct {
  /* history: request b's tokens are history[b * history_ld + i], i < history_len[b]; the
   * first prompt_len[b] are the prompt (NULL: none), the others output.  history_width:
   * the entries a row holds.  A token outside [0, V) is left out (ASYMSPEC_DATA_BAD_TOKEN);
   * lengths are clamped to [0, history_width] and prompt lengths to [0, history_len[b]]
   * (ASYMSPEC_DATA_BAD_LENGTH). */
  const int32_t* history;
  int64_t history_ld;
  int32_t history_width;
  const int32_t* history_len;
  const int32_t* prompt_len;
  /* drafts[b * drafts_ld + j], j < P - 1: position k counts those with j < k as output; so P = 1
   * counts none, and a loop that drafts a position at a time has the drafts before it in the
   * history.  A token outside [0, V) is left out (ASYMSPEC_DATA_BAD_TOKEN). */
  const int32_t* drafts;
  int64_t drafts_ld;
  /* penalties [B] (NULL: 1, 0 and 0).  A request with a bad one is not penalised at all
   * (ASYMSPEC_DATA_BAD_PENALTY). */
  const float* repetition;
  const float* frequency;
  const float* presence;
  /* biases: request b's are the entries bias_offsets[b] to bias_offsets[b + 1] - 1 of
   * bias_tokens and bias_values, of bias_count; a token listed twice takes its last entry.
   * A token outside [0, V) is left out (ASYMSPEC_DATA_BAD_TOKEN), offsets are clamped to
   * [0, bias_count] (ASYMSPEC_DATA_BAD_LENGTH). */
  const int32_t* bias_offsets;
  const int32_t* bias_tokens;
  const float* bias_values;
  int32_t bias_count;
  /* masks: mask_count rows of bits, mask_ld words apart; bit v % 32 of word v / 32 is set
   * where token v is allowed.  Position (b, k) takes row mask_rows[b * P + k], or none where
   * that is -1; without mask_rows it takes row b * P + k.  A row that does not exist
   * allows nothing (ASYMSPEC_DATA_BAD_INDEX).  A mask that allows nothing leaves a row of
   * mask_value alone. */
  const uint32_t* mask;
  int64_t mask_ld;
  int32_t mask_count;
  const int32_t* mask_rows;
  /* What a masked logit becomes, clamped to the type's finite range: -FLT_MAX gives its
   * lowest value.  The drafter's draw and the step's streaming kernels take that; its staged
   * and generic kernels answer masks of about -1e30 and lower with ASYMSPEC_DATA_NONFINITE.
   * -1e4 serves everywhere. */
  float mask_value;
} asymspec_constraints;

/* logits, out: [B, P, V] of `dtype`, rows ld and out_ld elements apart (row b * P + k);
 * out may be logits with the same ld, or must not overlap it.  One launch.
 * ASYMSPEC_ERR_INVALID_ARG: a null pointer (a group given in part counts), B or P < 0, V <
 * 2, ld or out_ld < V, mask_ld * 32 < V, a negative width, count or stride, a mask value
 * that is not finite; without mask_rows, mask_count < B * P.  ASYMSPEC_ERR_UNSUPPORTED:
 * dtype.  ASYMSPEC_ERR_MISALIGNED.  ASYMSPEC_ERR_TOO_LARGE: P > ASYMSPEC_CONSTRAIN_MAX_P,
 * B > 65535 or V > 2^25.  B = 0 or P = 0 is a no-op. */
#define ASYMSPEC_CONSTRAIN_MAX_P 256
int asymspec_constrain_logits(const asymspec_constraints* c, const void* logits, int64_t ld,
                              void* out, int64_t out_ld, int B, int P, int V, int dtype,
                              uint32_t* out_error_word, void* stream);

/* ---- the paged cache: block tables and slot maps ------------------------------
 * A pool of num_blocks blocks of block_size tokens; request b's token i lies in block
 * block_tables[b][i / block_size] at i % block_size.  The free blocks are a stack,
 * free_list[0 .. *free_count - 1], its top last.  One call moves B requests on by a round:
 *
 *   keep    = lens[b] + accepted[b] + 1 (lens[b] without `accepted`): the tokens that stay.
 *             The verifying pass wrote the last emitted token and the K drafts from position
 *             lens[b] on, so the step's out_accept_len is what `accepted` takes (-1, a data
 *             error, keeps lens[b])
 *   grow    = grow[b], or grow_all without `grow`: tokens to make room for
 *   blocks  = ceil((keep + grow) / block_size)
 *   held    = held[b], the blocks the request has: entries 0 .. held - 1 of its table row
 *
 * Requests that hold more than `blocks` give the others back (lens, grow 0: all, the
 * request has ended): in the order of the requests and of the table they go on the
 * stack.  Then requests that hold fewer take theirs off its top, in the same order, as
 * long as they last: a request that needs blocks is served if it and all before it fit, and
 * gets none otherwise (ASYMSPEC_DATA_NO_BLOCKS; out_len tells which).  Outputs:
 *
 *   out_start [B] = keep;  out_len [B] = keep + grow, or keep where not served: what may be
 *       attended over, at most (the table's entries past it may be another request's blocks)
 *   out_held [B], *out_free_count: the state for the next call
 *   block_tables, free_list: updated in place; table entries from out_held[b] on are left
 *       as they are
 *   out_offsets [B + 1]: the prefix sums of grow.  Token i of request b's new ones is entry t =
 *       out_offsets[b] + i of
 *   out_slots [capacity]: block * block_size + keep % block_size ..., the place of position
 *       keep + i in the pool; -1 where not served and from the last token on
 *   out_positions [capacity] (or NULL): keep + i, or -1 likewise
 *
 * out_start may be lens, out_held held and out_free_count free_count.  Bad lengths (lens
 * or held negative, accepted below -1, grow negative, keep + grow beyond the table's width,
 * free_count outside [0, num_blocks]) are clamped into range (a request too long for its
 * table is not served) and tokens beyond `capacity` are dropped: ASYMSPEC_DATA_BAD_LENGTH.
 * A block outside [0, num_blocks) in the tables or the list gives slot -1
 * (ASYMSPEC_DATA_BAD_INDEX).  One launch.
 * ASYMSPEC_ERR_INVALID_ARG: a null pointer, B < 0, block_size < 1, num_blocks < 1,
 * table_width < 1, table_ld < table_width, capacity < 0, grow_all < 0 (without `grow`).
 * ASYMSPEC_ERR_TOO_LARGE: B > ASYMSPEC_CACHE_MAX_B, B * table_width, num_blocks *
 * block_size, table_width * block_size or capacity beyond 2^31 - 1. ASYMSPEC_ERR_MISALIGNED. */
#define ASYMSPEC_CACHE_MAX_B 8192
int asymspec_cache_plan(const int32_t* lens, const int32_t* accepted, const int32_t* grow,
                        int grow_all, int B, int block_size, int num_blocks,
                        int32_t* block_tables, int64_t table_ld, int table_width,
                        const int32_t* held, int32_t* free_list, const int32_t* free_count,
                        int32_t* out_start, int32_t* out_len, int32_t* out_held,
                        int32_t* out_free_count, int32_t* out_offsets, int64_t* out_slots,
                        int32_t* out_positions, int64_t capacity, uint32_t* out_error_word,
                        void* stream);

/* ---- the paged cache: its keys and values --------------------------------------
 * Key of block n, token i, kv head h: the head_dim consecutive elements from keys + n *
 * key_strides[0] + i * key_strides[1] + h * key_strides[2]; values likewise.  Any order of
 * the three axes in memory is a matter of the strides. */
typedef struct {
  void* keys;
  void* values;
  int64_t key_strides[3];   /* block, token, kv head */
  int64_t value_strides[3];
  int32_t num_blocks, block_size, kv_heads, head_dim;
  int32_t dtype;            /* asymspec_dtype_t */
} asymspec_cache;

/* Writes the keys and values of T tokens: k[t][h] (strides k_strides: token, head) goes to
 * slot slots[t] = block * block_size + token; a negative slot (the padding of a captured
 * batch) is skipped, one past the pool too (ASYMSPEC_DATA_BAD_INDEX).  Two tokens with one
 * slot leave either's key and value there.  One launch, any element-aligned pointers and
 * strides; 16-byte vectors where all of them allow it.  T = 0 is a no-op.
 * ASYMSPEC_ERR_INVALID_ARG: a null pointer, T < 0, a size < 1, a negative stride.
 * ASYMSPEC_ERR_UNSUPPORTED: dtype.  ASYMSPEC_ERR_MISALIGNED.  ASYMSPEC_ERR_TOO_LARGE:
 * num_blocks * block_size or kv_heads * head_dim beyond 2^31 - 1. */
int asymspec_cache_write(const asymspec_cache* cache, const void* k, const void* v,
                         const int64_t* k_strides, const int64_t* v_strides, const int64_t* slots,
                         int T, uint32_t* out_error_word, void* stream);

/* Attention of the last Q of each request's tokens over its cached ones (their own keys and
 * values written before).  For request b, query i and query head h, at position p = lens[b]
 * - Q + i, over the keys j of kv head h / (heads / kv_heads) with max(0, p - window + 1) <= j
 * <= p (window 0, or one that spans the whole table row: from 0 on):
 *
 *   s_j = scale * q . k_j,   lse = ln sum_j exp(s_j),   out = sum_j exp(s_j - lse) v_j
 *
 * Q = 1 is a decoded or drafted token, Q = K + 1 a round's verification.  A query without
 * keys (p < 0: a request that has ended or is shorter than Q) gets out = 0 and lse =
 * -infinity.  Keys and values that a query does not see never reach it, whatever is in
 * them (the rest of a block, a later token's).  Sums, maxima and the accumulated values
 * are fp32; out is rounded once.
 *   q [B, Q, heads, head_dim]: strides q_strides (request, query, head), out likewise; the
 *       cache's dtype, element-aligned.  out must not overlap q (whose queries are read
 *       until the call ends) nor anything else that the call reads
 *   block_tables [B, table_width] int32, rows table_ld apart; lens [B] int32
 *   out_lse: [B, Q, heads] fp32 contiguous, or NULL
 *   workspace: asymspec_cache_attend_workspace_bytes(...) bytes, 256-byte aligned; it needs
 *       no zeroing, serves any calls that it is large enough for, and must not be shared by
 *       calls in flight at the same time
 * A length below 0 counts as 0 and one beyond the table as the table's (ASYMSPEC_DATA_BAD_
 * LENGTH); keys in a block outside [0, num_blocks) are not seen (ASYMSPEC_DATA_BAD_INDEX; blocks
 * that lie before every query's window may be gone from the table).
 * B = 0 or Q = 0 is a no-op.  The work is split over the cached tokens of all requests
 * evenly, whatever their lengths, and the parts joined by a second launch; results do
 * not depend on the order in which the parts finish.
 * ASYMSPEC_ERR_INVALID_ARG: a null pointer, a size < 1 (B, Q < 0), heads not a multiple of
 * kv_heads, table_ld < table_width, a scale that is not finite, window < 0, a negative stride, a
 * stride of 0 along an axis of out that is longer than 1, out = q.
 * ASYMSPEC_ERR_UNSUPPORTED: dtype, head_dim > ASYMSPEC_CACHE_MAX_D.  ASYMSPEC_ERR_MISALIGNED:
 * an unaligned pointer; keys, values, their strides and head_dim must lie on 16-byte
 * boundaries.  ASYMSPEC_ERR_WORKSPACE.  ASYMSPEC_ERR_TOO_LARGE: B >
 * ASYMSPEC_CACHE_MAX_B, Q * heads > 2^20, num_blocks * block_size beyond 2^31 - 1 or
 * table_width * block_size beyond 2^30. */
#define ASYMSPEC_CACHE_MAX_D 256
size_t asymspec_cache_attend_workspace_bytes(int B, int Q, int heads, int kv_heads, int head_dim);
int asymspec_cache_attend(const asymspec_cache* cache, const void* q, const int64_t* q_strides,
                          int B, int Q, int heads, const int32_t* block_tables, int64_t table_ld,
                          int table_width, const int32_t* lens, float scale, int window, void* out,
                          const int64_t* out_strides, float* out_lse, void* workspace,
                          size_t workspace_bytes, uint32_t* out_error_word, void* stream);

#ifdef __cplusplus
}
#endif

#endif /* ASYMSPEC_SERVING_H */

/*
 * ltri_paged.h — C ABI of libltri, second part: a key-value cache in pages, the attention of new tokens over
 * it, and its eviction by accumulated attention weight, on one AMD MI355X (gfx950).
 *
 *   ltri_paged_append   write the rows of new tokens into the pages of their sequences;
 *   ltri_paged_attend   exact attention of each sequence's latest rows over all its tokens, the tokens' work shared
 *                       out over the whole chip whatever the lengths; optionally every token's weight becomes
 *                       decay * weight + the attention it received;
 *   ltri_paged_step     the two in one call (decoding);
 *   ltri_paged_evict    bring every sequence back to a budget: the first and the latest tokens stay, of the others
 *                       those of largest weight.
 *
 * The cache of one attention layer
 *   k_pages, v_pages  device [n_pages][n_kv_heads][page_tokens][head_dim] in the dtype, or any other order of the first
 *                     three (page_stride, head_stride, token_stride of ltri_paged_config);
 *   weight            device fp32 [n_pages][n_kv_heads][page_tokens]: attention weight received, per KV head (summed
 *                     over its query heads); pos: device int32, same shape: a token's position in its sequence.
 *                     Only with weights = 1, else both are NULL.
 * Which pages hold which sequence is the caller's business; every call is given, on the device,
 *   table             int32 [seq_count][table_pages]: page of the tokens p * page_tokens .. + page_tokens - 1;
 *                     entries behind a sequence's last page are not read;
 *   lens              int32 [seq_count]: tokens the sequence holds, the call's new ones among them;
 *   seen              int32 [seq_count]: tokens the sequence has taken in (lens, if nothing was ever evicted): the
 *                     newest token has position seen - 1. Read only with weights = 1, else it may be NULL.
 * They are read when the work runs, not when it is enqueued, and grids do not depend on them, so a captured call can
 * be replayed with other lengths and tables. A sequence of length 0 is padding: it takes no rows, its outputs are 0 and
 * -infinity, its eviction does nothing.
 * Sequences may share pages for reading. Where a call writes (appended rows, weights, evictions), the written tokens'
 * pages belong to one sequence of the call only, and with weights no page is named twice in a call.
 *
 * Conventions are those of ltri.h: statuses, caller-owned buffers (alive until the work on them is done), work enqueued on
 * the handle's stream without waiting. A call runs on the device that was current at creation, whatever is current when it is made. Calls on one
 * handle must not overlap; handles may share a scratch buffer if their calls do not overlap. k/v pages and rows, q and
 * out are 16-byte aligned (EINVAL else). What only the device can see is reported by ltri_paged_sync_status(): a length
 * beyond the table's capacity (LTRI_ECAPACITY; the sequence is taken as length 0), a page outside [0, n_pages)
 * (LTRI_EINVAL; its tokens are not attended and not written, and its sequence is not evicted) and, where weights are written
 * or tokens evicted, sequences that together hold more tokens than the pool, be it by a page named twice or by pages outside it
 * (LTRI_ECAPACITY; the attention is whole, but sequences that found no room in scratch may keep their weights or stay unevicted).
 */
#ifndef LTRI_PAGED_H
#define LTRI_PAGED_H

#include "ltri.h"

#ifdef __cplusplus
extern "C" {
#endif

#define LTRI_PAGED_MAX_SEQS  4096   /* most sequences one call can take                  */
#define LTRI_PAGED_MAX_ROWS  64     /* most query rows per sequence                      */

typedef struct ltri_paged ltri_paged;

typedef struct {
  int32_t n_q_heads, n_kv_heads, head_dim;   /* head_dim 64 or 128; at most 4096 query heads, 128 per KV head */
  int32_t dtype;                             /* LTRI_F32 | LTRI_BF16                       */
  int32_t page_tokens;                       /* a power of two, 1 to 4096                  */
  int32_t n_pages;                           /* pages in the pool                          */
  int32_t table_pages;                       /* entries in a sequence's row of the table; table_pages *
                                                page_tokens <= 2^30 tokens                 */
  int32_t max_seqs;                          /* most sequences in one call                 */
  int32_t rows_max;                          /* most query rows per sequence in one call   */
  int32_t weights;                           /* 1: weights and positions are kept          */
  /* Elements from a page, KV head, token to the next (the last at most 2^24), multiples of 16 bytes; keys and values alike. All 0: dense
   * [n_pages][n_kv_heads][page_tokens][head_dim]. Different (page, head, token) must not overlap. */
  int64_t page_stride, head_stride, token_stride;
} ltri_paged_config;

/* Bytes of the two device buffers of a handle: `state` (counters, the device's error word; as long as the handle
 * lives; ltri_paged_create enqueues a kernel that clears it) and `scratch` (temporaries of a call: partial results;
 * with weights also lists of moves, 4 to 12 bytes, and scores, 4 min(rows_max n_q_heads / n_kv_heads, 31) bytes, for every token of the pool and
 * KV head: 8 KV heads of 4, a pool of 1M tokens, rows_max 1: 151 MB, 7: 974 MB). EINVAL on an unsupported configuration. */
int32_t ltri_paged_workspace_bytes(const ltri_paged_config* cfg, size_t* state_bytes, size_t* scratch_bytes);

/* All pointers are device memory of the current device and the caller's; state and scratch 256-byte aligned. */
int32_t ltri_paged_create(const ltri_paged_config* cfg, void* k_pages, void* v_pages, float* weight, int32_t* pos,
                          void* state, void* scratch, void* hip_stream, ltri_paged** out);
/* Without device buffers: calls check their arguments and enqueue nothing. */
int32_t ltri_paged_create_dry(const ltri_paged_config* cfg, ltri_paged** out);
int32_t ltri_paged_destroy(ltri_paged* c);
/* Stream of the following calls. Ordering it behind the old one's work, ltri_paged_create's included, is the caller's business (events). */
int32_t ltri_paged_set_stream(ltri_paged* c, void* hip_stream);

/* k_new, v_new: device [seq_count][n_kv_heads][n_new][head_dim]. Row i of sequence s goes to place lens[s] - n_new + i
 * (rows whose place is negative are dropped), with position seen[s] - n_new + i and weight
 * w_new[s][kv head][i] (device fp32, NULL = 0). n_new >= 1; beyond table_pages * page_tokens ECAPACITY. */
int32_t ltri_paged_append(ltri_paged* c, int32_t seq_count, const int32_t* table, const int32_t* lens,
                          const int32_t* seen, const void* k_new, const void* v_new, const float* w_new, int32_t n_new);

/* q: device [seq_count][n_q][n_q_heads][head_dim], out the same, in the dtype, not overlapping; lse: device fp32
 * [seq_count][n_q][n_q_heads] or NULL (natural-log sum of exponentials of the scaled scores). Row i attends the tokens
 * 0 .. lens - n_q + i, with weights softmax(q.k / sqrt(head_dim)); a row that sees no token, or whose scores are all
 * -infinity, gives 0 and -infinity. Rows of tokens it does not see have no influence, whatever they hold; an infinity or NaN in
 * a value row that it does see makes that column infinite or NaN.
 * decay >= 0 (weights = 1 only): every token's weight becomes decay * weight + the sum of its attention weights over
 * the rows and the KV head's query heads; a weight that is not read (decay = 0) may hold anything. decay < 0: weights
 * stay as they are.
 * Rounding: fp32 sums and exponentials; bf16 probabilities enter the products as the sum of two bf16 parts (2^-17),
 * so only the result is rounded to the dtype. How a sequence's tokens are shared out depends on the call's lengths, so
 * a row can differ in its last bits between calls with other sequences beside it; the same call repeats itself bit for
 * bit. */
int32_t ltri_paged_attend(ltri_paged* c, int32_t seq_count, const int32_t* table, const int32_t* lens, const void* q,
                          int32_t n_q, void* out, float* lse, float decay);

/* ltri_paged_append (weights of new tokens 0) and ltri_paged_attend of the same n_new rows, n_new <= rows_max: the same results. */
int32_t ltri_paged_step(ltri_paged* c, int32_t seq_count, const int32_t* table, const int32_t* lens, const int32_t* seen,
                        const void* k_new, const void* v_new, const void* q, int32_t n_new, void* out, float* lse,
                        float decay);

/* Per sequence of more than `keep` tokens and KV head (weights = 1 only): tokens are ordered by (protected first, weight
 * descending, place ascending), where the protected ones have a position below n_sink or among the last n_recent of
 * seen; the first `keep` stay. Kept tokens at places >= keep move, in order, to the places < keep that became free, with
 * row, weight and position; nothing else is written, and lens becomes keep. A NaN weight counts as lowest, -0 as 0.
 * EINVAL unless keep >= 1 and n_sink + n_recent <= keep. Pages behind the new length are the caller's to reuse. */
int32_t ltri_paged_evict(ltri_paged* c, int32_t seq_count, const int32_t* table, int32_t* lens, const int32_t* seen,
                         int32_t keep, int32_t n_sink, int32_t n_recent);

/* Synchronises the stream: LTRI_OK or the first error the device raised since the last call, which is then forgotten. */
int32_t ltri_paged_sync_status(ltri_paged* c);
const char* ltri_paged_last_error(const ltri_paged* c);

#ifdef __cplusplus
}
#endif
#endif /* LTRI_PAGED_H */

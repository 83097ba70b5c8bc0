/*
 * kara_evict.h -- eviction from the paged cache by accumulated attention weight.
 *
 * Every cached token has, per layer and KV head, an accumulator: the sum over
 * the queries seen so far of the softmax weight they gave it, over the G query
 * heads of its KV head.  A decoding step adds to it as it attends
 * (kara_evict_attention), a prompt's or a window's queries are added afterwards
 * (kara_evict_observe), and kara_evict_tokens cuts a sequence to a budget: its
 * first and last tokens and those of the largest accumulators stay.
 *
 * Accumulators live in pages like the keys, `weights` of a layer being fp32
 * [num_pages][n_kv_heads][block_size]: they follow a page wherever a block table
 * puts it.  Those of the n_new newest positions of a sequence start from zero in
 * the call that first counts them, so pages need no clearing.
 *
 * Every page below the seq_len of a sequence that a call lists must be that
 * sequence's alone among the listed ones, and in its table once (not checked):
 * accumulators are added to without atomics, in one order, so that results are the
 * same bits every time, and two sequences at one page would lose weights.  Sequences that share a prefix are
 * listed in calls of their own, one after the other; their weights then add up in
 * the shared accumulators, n_new counting each one's own positions.  Before
 * kara_evict_tokens, which moves rows, a page belongs to one sequence of all.
 *
 * The cache is either rows of p->dtype (kara.h; k_scales and v_scales NULL) or
 * held in 4 bits (kara_q4.h; both given, p->dtype the type of q).
 *
 * Infinite and NaN elements of keys and queries enter the logits as they are: a
 * logit of -inf is a weight of 0, one of +inf or NaN makes the weights that its
 * query gives NaN.  A query whose every logit is -inf gives no weights.
 *
 * Conventions are those of kara.h and kara_harness.h: device pointers unless
 * stated (pool arrays: host arrays of n_layers device pointers, 1 <= n_layers <=
 * 64), the caller owns all memory, nothing synchronises or allocates,
 * host-checkable argument errors come back as KARA_ERR_* with nothing enqueued.
 * The window-related fields of p must be valid but are not used.  max_len and keep
 * are 2^30 at most.  Alignment, checked: that of kara_q4.h, rows 16 bytes, accumulators
 * 16 where block_size is a multiple of 4, else 4.
 */
#ifndef KARA_EVICT_H
#define KARA_EVICT_H

#include "kara.h"

#ifdef __cplusplus
extern "C" {
#endif

/* Bytes of device workspace kara_evict_attention needs for n sequences of at most
 * max_len tokens and n_layers layers (written to *bytes, a HOST pointer); it is
 * enough for fewer and shorter ones.  Every logit of the call passes through it: 4
 * bytes a layer, sequence, query head and key, and a record of head_dim + 2 fp32 per
 * 256 keys (64 sequences of 32K tokens, 40 heads: 0.5 GB a layer).  A program with
 * many layers passes them in groups of a few, which share one workspace. */
kara_status_t kara_evict_attention_workspace_size(const kara_params_t* p, int32_t n, int32_t n_layers,
                                                  int32_t max_len, size_t* bytes);

/*
 * kara_harness_decode_attention (one query per layer, sequence and query head
 * over the whole cache, G <= KARA_HARNESS_MAX_GROUP; out fp32) that also adds
 * each key's weight, summed over the group's query heads, to its accumulator:
 * positions below seq_len - n_new are added to, the last n_new are set.  The output
 * row of a query that gives no weights is zero.  A sequence listed more than once is
 * counted once, by its first listing.  Longer
 * sequences than max_len, empty ones and indices outside [0, n_seqs) give zero
 * output rows and leave their accumulators alone.  The block table must map
 * every position below seq_len, to pages of no other listed sequence; a position on
 * no page leaves the sequence's output unspecified, and nothing outside the pools is
 * read or written.
 */
kara_status_t kara_evict_attention(const kara_params_t* p, int32_t n, const int32_t* seqs, int32_t n_layers,
                                   const void* q, const void* const* k_pools, const void* const* v_pools,
                                   const void* const* k_scales, const void* const* v_scales,
                                   float* const* weights, const int32_t* block_table, const int32_t* seq_lens,
                                   int32_t n_new, int32_t max_len, float* out, void* workspace,
                                   size_t workspace_bytes, void* stream);

/* Bytes of device workspace kara_evict_observe needs (written to *bytes, a HOST
 * pointer). */
kara_status_t kara_evict_observe_workspace_size(const kara_params_t* p, int32_t n, int32_t n_layers,
                                                int32_t n_query, int32_t max_len, size_t* bytes);

/*
 * Adds to the accumulators the weights that the last n_query tokens of each
 * listed sequence give: query t, at position i = seq_lens[s] - n_query + t, spreads
 * a weight of one per query head over positions [0, i] (softmax of scale * q . K).
 * q: [n_layers][n][n_query][n_q_heads][head_dim] (p->dtype).  The last n_new
 * positions are set, those before are added to (n_new = n_query for a prompt just
 * appended, n_new >= seq_len for all).  Queries before the sequence's start
 * (n_query > seq_len) do not count.  Listings, lengths and pages, one sequence's
 * alone, as in kara_evict_attention.
 */
kara_status_t kara_evict_observe(const kara_params_t* p, int32_t n, const int32_t* seqs, int32_t n_layers,
                                 int32_t n_query, const void* q, const void* const* k_pools,
                                 const void* const* k_scales, float* const* weights, const int32_t* block_table,
                                 const int32_t* seq_lens, int32_t n_new, int32_t max_len, void* workspace,
                                 size_t workspace_bytes, void* stream);

/* Bytes of device workspace kara_evict_tokens needs (written to *bytes, a HOST
 * pointer); 4 n of them where the caller takes the kept positions. */
kara_status_t kara_evict_workspace_size(const kara_params_t* p, int32_t n, int32_t n_layers, int32_t keep,
                                        size_t* bytes);

/*
 * Cuts every listed sequence longer than `keep` to `keep` tokens in n_layers
 * layers.  Per layer and KV head the first n_sink and the last n_recent positions
 * stay, and of those between the keep - n_sink - n_recent with the largest
 * accumulators (ties to the lower position; NaN below every number).  Rows of K,
 * V and accumulators move in place to positions 0 .. keep - 1, in order; rows
 * from there on are left as they were.  Sequences of at most `keep` tokens are
 * left alone.
 *   kept     [n_layers][n][n_kv_heads][keep] int32, ascending positions, -1 past
 *            the end of a shorter sequence; NULL: held in the workspace
 *   commit   non-zero: seq_lens[s] = keep, and the blocks past it released as in
 *            kara_commit_tables (freed [n][max_blocks_per_seq], n_freed [n]), by the
 *            last launch, with the rows: where a launch fails, lengths and tables stay.
 *            Zero: lengths and tables stay, for a caller that passes its layers in
 *            several calls and commits with the last; freed, n_freed are not used.
 *   status   KARA_SEQ_* bits: BAD_INDEX, DUP_TRIGGER, BAD_WINDOW (seq_len negative,
 *            over max_len or past the table), BAD_PAGE (a block of [0, seq_len) on no
 *            page of the pool), DUP_PAGE (a page twice among them).  Flagged sequences
 *            are left alone; their kept entries are -1, n_freed 0.
 * 1 <= keep, 0 <= n_sink, 0 <= n_recent, n_sink + n_recent <= keep.  Pages must
 * belong to one sequence alone, as in kara.h.
 */
kara_status_t kara_evict_tokens(const kara_params_t* p, int32_t n, const int32_t* seqs, int32_t n_layers,
                                int32_t keep, int32_t n_sink, int32_t n_recent, void* const* k_pools,
                                void* const* v_pools, void* const* k_scales, void* const* v_scales,
                                float* const* weights, int32_t* block_table, int32_t* seq_lens, int32_t max_len,
                                int32_t commit, int32_t* kept, int32_t* freed, int32_t* n_freed, int32_t* status,
                                void* workspace, size_t workspace_bytes, void* stream);

#ifdef __cplusplus
}
#endif

#endif /* KARA_EVICT_H */

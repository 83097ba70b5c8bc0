/*
 * kara_q4.h -- a paged K/V cache held in 4 bits, beside the rows of kara.h:
 * tokens quantised as they are appended, read back, and attended over.
 *
 * Format.  A row of head_dim values is cut into blocks of 32.  A block is 32
 * codes of 4 bits -- the e2m1 values 0, 0.5, 1, 1.5, 2, 3, 4, 6 (codes 0..7)
 * and their negatives (8..15) -- and one scale byte b: a code stands for its
 * value times 2^(b - 127).  For a block whose largest finite magnitude is top,
 *   e = floor(log2(top)) - 2, one more where top > 7 * 2^e,
 * held to [-125, 125]; b = e + 127; each code is x / 2^e rounded to the
 * nearest value, ties to the even code, magnitudes past 6 to 6.  (7 is where
 * rounding down to 6 errs as much as the doubled step does.)  A NaN is stored
 * as 0 and an infinity as 6 * 2^e with its sign, so that what is read is always
 * finite; the append reports both (KARA_SEQ_NONFINITE).  Every value is exact in
 * bf16 and fp32.
 *
 * Pools, per layer (PAGES of kara.h, the same block table and lengths):
 *   k_pools, v_pools     codes  [num_pages][n_kv_heads][block_size][head_dim / 2]
 *                        uint8, element 2i in the low half of byte i
 *   k_scales, v_scales   scales [num_pages][n_kv_heads][block_size][head_dim / 32]
 *                        uint8
 * 68 bytes a row at head_dim 128 where bf16 takes 256.
 *
 * Alignment, checked: codes, k_new, v_new, q, k_out, v_out, out and workspaces 16
 * bytes, scales those of a row (head_dim / 32), int32 arrays 4.
 *
 * Conventions are those of kara.h and kara_harness.h: device pointers unless
 * stated (pool arrays: host arrays of n_layers device pointers, 1 <= n_layers
 * <= 64), the caller owns all memory, nothing synchronises or allocates,
 * host-checkable argument errors come back as KARA_ERR_* with nothing
 * enqueued.  p->dtype is the type of k_new, v_new, q, k_out, v_out and out; the
 * window-related fields of p must be valid but are not used.
 */
#ifndef KARA_Q4_H
#define KARA_Q4_H

#include "kara.h"

#ifdef __cplusplus
extern "C" {
#endif

/* Status bit of kara_q4_append: a new row held a NaN or an infinity.  Alone it
 * is a report: the sequence was appended. */
#define KARA_SEQ_NONFINITE 64

/*
 * Appends n_new tokens to each of the n sequences seqs[0..n) (distinct) in every
 * one of n_layers layers, quantised: row of token i, KV head h, layer l from
 * k_new / v_new [n_layers][n][n_new][n_kv_heads][head_dim] (p->dtype) to logical
 * position seq_lens[s] + i of sequence s = seqs[j].  Then seq_lens[s] += n_new.
 * The caller maps the blocks covering the new positions beforehand, to pages that
 * no other sequence maps.  status[j]
 * as in kara_harness_kv_append (BAD_INDEX, DUP_TRIGGER, BAD_WINDOW, BAD_PAGE;
 * such sequences are not written), or KARA_SEQ_NONFINITE.
 */
kara_status_t kara_q4_append(const kara_params_t* p, int32_t n, const int32_t* seqs, int32_t n_new,
                             int32_t n_layers, const void* k_new, const void* v_new, void* const* k_pools,
                             void* const* v_pools, void* const* k_scales, void* const* v_scales,
                             const int32_t* block_table, int32_t* seq_lens, int32_t* status, void* stream);

/*
 * Reads n_rows rows from logical position start[s] on (start: [n_seqs]) of each
 * listed sequence s = seqs[j] into k_out / v_out [n_layers][n][n_rows]
 * [n_kv_heads][head_dim] (p->dtype), exactly.  Positions outside [0, seq_lens[s])
 * or on no page of the pool, and sequence indices outside [0, n_seqs), read as
 * zeros.
 */
kara_status_t kara_q4_read(const kara_params_t* p, int32_t n, const int32_t* seqs, const int32_t* start,
                           int32_t n_rows, int32_t n_layers, const void* const* k_pools,
                           const void* const* v_pools, const void* const* k_scales,
                           const void* const* v_scales, const int32_t* block_table, const int32_t* seq_lens,
                           void* k_out, void* v_out, void* stream);

/*
 * Bytes of device workspace kara_q4_attention needs for n sequences of at most
 * max_len tokens (2^30 at most), n_layers layers and n_query queries each (written
 * to *bytes, a HOST pointer).  It is enough for fewer sequences and layers and for
 * shorter ones, not for fewer queries: few queries split their keys further, so a
 * decoding step may need more than a prompt's chunk (100 sequences of 32000 tokens,
 * 32/8 heads, one layer: 208 MB for one query, 34 for 300).  A workspace for calls
 * of several n_query is the largest of their sizes.
 */
kara_status_t kara_q4_attention_workspace_size(const kara_params_t* p, int32_t n, int32_t n_layers,
                                               int32_t n_query, int32_t max_len, size_t* bytes);

/*
 * Causal attention of the last n_query tokens of each listed sequence over its
 * cache: query t of sequence s = seqs[j], at position i = seq_lens[s] - n_query +
 * t, gives
 *   out[l][j][t][hq][:] = sum_k w_k V_k,  w = softmax over k in [0, i] of
 *                         scale * q . K_k,  KV head hq / G.
 * n_query = 1 is a decoding step.  q, out: [n_layers][n][n_query][n_q_heads]
 * [head_dim] (p->dtype).  Rows before the sequence's start (n_query > seq_len),
 * sequences longer than max_len, sequence indices outside [0, n_seqs) and queries
 * whose every logit is -inf give zeros; a logit of +inf or NaN gives NaN.  The block table must map every position below seq_len to a page of the
 * pool; where it does not, the sequence's output is unspecified, and nothing
 * outside the pools is read.  Softmax statistics and sums are fp32; bf16 calls
 * round each weight to bf16 before it meets V (the same rounded weights make up
 * its sum), fp32 calls keep it whole.  Results are the same bits from call to
 * call; they may differ in the last ones with n, n_layers, n_query and max_len,
 * which decide how keys are split.
 */
kara_status_t kara_q4_attention(const kara_params_t* p, int32_t n, const int32_t* seqs, int32_t n_layers,
                                int32_t n_query, const void* q, const void* const* k_pools,
                                const void* const* v_pools, const void* const* k_scales,
                                const void* const* v_scales, const int32_t* block_table,
                                const int32_t* seq_lens, int32_t max_len, void* out, void* workspace,
                                size_t workspace_bytes, void* stream);

#ifdef __cplusplus
}
#endif

#endif /* KARA_Q4_H */

/*
 * kara_q8.h -- a paged K/V cache held in 8 bits with a scale for each page and KV
 * head, beside the rows of kara.h and the 4-bit codes of kara_q4.h: tokens
 * quantised as they are appended, read back, and attended over.
 *
 * Format.  The rows of one page and KV head are a block: e4m3 codes (1 sign, 4
 * exponent and 3 mantissa bits, bias 7, largest value 448, no infinities) and one
 * scale byte b: a code stands for its value times 2^(b - 127).  For a block whose
 * largest finite magnitude is top, e is the smallest whole number with
 * top <= 448 * 2^e, held to [-117, 119]; b = e + 127; each code is x / 2^e rounded to
 * the nearest value, ties to the even code, magnitudes past 448 to 448.  A NaN is
 * stored as 0 and an infinity as 448 * 2^e with its sign, so that what is read is always
 * finite; the append reports both (KARA_SEQ_NONFINITE).  Every value is exact in
 * bf16 and fp32.
 *
 * A block's scale never falls while its page fills: tokens that join older ones in a
 * page take the larger of its scale and their own, and where that grows the older codes
 * are rounded to it.  Codes are floating, so that this changes their exponents alone,
 * exactly, down to 2^-6 of the new scale; smaller ones lose bits.  The first token of a
 * page (a position that is a multiple of block_size) starts its scale anew.
 *
 * The calls of this header, kara_rope_append and kara_window_attention are all that take
 * this cache: compression, eviction and the helpers of kara_harness.h do not.
 *
 * Pools, per layer (PAGES of kara.h, the same block table and lengths):
 *   k_pools, v_pools     codes  [num_pages][n_kv_heads][block_size][head_dim] uint8
 *   k_scales, v_scales   scales [num_pages][n_kv_heads] uint8
 *
 * Alignment, checked: codes, k_new, v_new, q, k_out, v_out, out and workspaces 16
 * bytes, int32 arrays 4.
 *
 * Conventions are those of kara.h and kara_harness.h: device pointers unless
 * stated (pool arrays: host arrays of n_layers device pointers, 1 <= n_layers
 * <= 64), the caller owns all memory, nothing synchronises or allocates,
 * host-checkable argument errors come back as KARA_ERR_* with nothing
 * enqueued.  p->dtype is the type of k_new, v_new, q, k_out, v_out and out; the
 * window-related fields of p must be valid but are not used.
 */
#ifndef KARA_Q8_H
#define KARA_Q8_H

#include "kara_q4.h" /* KARA_SEQ_NONFINITE */

#ifdef __cplusplus
extern "C" {
#endif

/*
 * Appends n_new tokens to each of the n sequences seqs[0..n) (distinct) in every
 * one of n_layers layers, quantised: row of token i, KV head h, layer l from
 * k_new / v_new [n_layers][n][n_new][n_kv_heads][head_dim] (p->dtype) to logical
 * position seq_lens[s] + i of sequence s = seqs[j].  Then seq_lens[s] += n_new.
 * The caller maps the blocks covering the new positions beforehand, to pages that
 * no other sequence maps.  status[j] as in kara_harness_kv_append (BAD_INDEX,
 * DUP_TRIGGER, BAD_WINDOW, BAD_PAGE; such sequences are not written), or
 * KARA_SEQ_NONFINITE.
 */
kara_status_t kara_q8_append(const kara_params_t* p, int32_t n, const int32_t* seqs, int32_t n_new,
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
kara_status_t kara_q8_read(const kara_params_t* p, int32_t n, const int32_t* seqs, const int32_t* start,
                           int32_t n_rows, int32_t n_layers, const void* const* k_pools,
                           const void* const* v_pools, const void* const* k_scales,
                           const void* const* v_scales, const int32_t* block_table, const int32_t* seq_lens,
                           void* k_out, void* v_out, void* stream);

/*
 * Bytes of device workspace kara_q8_attention needs for n sequences of at most
 * max_len tokens (2^30 at most), n_layers layers and n_query queries each (written
 * to *bytes, a HOST pointer).  It is enough for fewer sequences and layers and for
 * shorter ones, not for fewer queries, as in kara_q4_attention_workspace_size.
 */
kara_status_t kara_q8_attention_workspace_size(const kara_params_t* p, int32_t n, int32_t n_layers,
                                               int32_t n_query, int32_t max_len, size_t* bytes);

/*
 * Causal attention of the last n_query tokens of each listed sequence over its
 * cache: kara_window_attention (kara_window.h) without a window.  n_query = 1 is a
 * decoding step.  q, out: [n_layers][n][n_query][n_q_heads][head_dim] (p->dtype).
 */
kara_status_t kara_q8_attention(const kara_params_t* p, int32_t n, const int32_t* seqs, int32_t n_layers,
                                int32_t n_query, const void* q, const void* const* k_pools,
                                const void* const* v_pools, const void* const* k_scales,
                                const void* const* v_scales, const int32_t* block_table,
                                const int32_t* seq_lens, int32_t max_len, void* out, void* workspace,
                                size_t workspace_bytes, void* stream);

#ifdef __cplusplus
}
#endif

#endif /* KARA_Q8_H */

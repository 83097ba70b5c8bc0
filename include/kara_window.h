/*
 * kara_window.h -- causal attention within a sliding window, with the first tokens
 * of a sequence always visible, over paged rows or 8-bit codes.
 *
 * Conventions are those of kara.h and kara_q8.h.
 */
#ifndef KARA_WINDOW_H
#define KARA_WINDOW_H

#include "kara_q8.h"

#ifdef __cplusplus
extern "C" {
#endif

/*
 * Bytes of device workspace kara_window_attention needs (written to *bytes, a HOST
 * pointer) for n sequences of at most max_len tokens (2^30 at most), n_layers layers and
 * n_query queries each; as for kara_q8_attention it is enough for fewer sequences and
 * layers and for a smaller max_len, not for other values of n_query, window and n_sink,
 * nor of p.
 *
 * It covers a cache of either kind.  fp32 calls over rows keep a record (head_dim + 2
 * floats) for each row of output and part of the keys, of 4608 keys at most: 4.4 GB for
 * one prompt of 32K queries of 32 heads of 128 and one layer, 136 MB for 4 x 1024 queries
 * over 8.7K tokens.  fp32 calls over 8 bits and bf16 ones of many queries need 34 to 68 MB
 * (d = 128), so that an fp32 program whose cache is in 8 bits is told more than it needs
 * here; without a window kara_q8_attention_workspace_size is exact for it.
 */
kara_status_t kara_window_attention_workspace_size(const kara_params_t* p, int32_t n, int32_t n_layers,
                                                   int32_t n_query, int32_t window, int32_t n_sink,
                                                   int32_t max_len, size_t* bytes);

/*
 * Attention of the last n_query tokens of each listed sequence: query t of sequence s
 * = seqs[j], at position i = seq_lens[s] - n_query + t, sees the keys
 *   k <= i  with  k > i - window  or  k < n_sink
 * (itself, the window - 1 before it and the first n_sink; window = 0: all up to i) and
 * gives out[l][j][t][hq][:] = sum_k w_k V_k, w = softmax over them of scale * q . K_k,
 * KV head hq / G.  q, out: [n_layers][n][n_query][n_q_heads][head_dim] (p->dtype).
 *
 * The cache is rows of p->dtype (kara.h; k_scales and v_scales NULL) or held in 8 bits
 * (both given).  Keys and values that a query does not see do not reach its result,
 * whatever they hold.  Blocks of which no query sees a token are not needed: their
 * entries of the block table may be -1 or name pages that others own by now, so that a
 * program may take back the pages between the first tokens and the window.  Visible
 * positions must be mapped to pages of the pool; where they are not, the sequence's
 * output is unspecified, and nothing outside the pools is read.
 *
 * Rows before the sequence's start (n_query > seq_len), sequences longer than max_len,
 * sequence indices outside [0, n_seqs) and queries whose every visible logit is -inf
 * give zeros; a visible logit of +inf or NaN gives NaN, and a visible infinite or NaN
 * value enters the sum as it is (an infinite one of a weight that is 0 in 32 bits: itself or
 * NaN).  Softmax statistics and sums are fp32.  fp32 calls, and bf16 ones over rows where a
 * KV head has few query rows (G * n_query at most 64), keep all 24 bits of a weight; bf16
 * calls of few rows over 8 bits hold it in 16 (two bf16 terms), and those of more rows round
 * it to bf16; the same held weights make up its sum.  Results are the same bits from call to
 * call; they may differ in the last ones with n, n_layers, n_query and max_len, which decide
 * how keys are split.
 *
 * KARA_ERR_UNSUPPORTED past what one launch holds, also where the workspace's size is given.
 * With U = n_layers * n * n_kv_heads and R = G * n_query it holds, of few rows (R at most 64,
 * and all fp32 calls over rows), U * ceil(R / 16) times the parts of the keys up to 2^24, and
 * 2^26 rows of output where there is more than one part; of more rows U * ceil(R / 128) up to
 * 2^23.
 */
kara_status_t kara_window_attention(const kara_params_t* p, int32_t n, const int32_t* seqs, int32_t n_layers,
                                    int32_t n_query, int32_t window, int32_t n_sink, const void* q,
                                    const void* const* k_pools, const void* const* v_pools,
                                    const void* const* k_scales, const void* const* v_scales,
                                    const int32_t* block_table, const int32_t* seq_lens, int32_t max_len, void* out,
                                    void* workspace, size_t workspace_bytes, void* stream);

#ifdef __cplusplus
}
#endif

#endif /* KARA_WINDOW_H */

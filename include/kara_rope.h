/*
 * kara_rope.h -- tokens appended to the paged cache with the position rotation
 * applied on the way.
 *
 * The rotation is the rotate-half form of kara_recompute.h over a head's first r =
 * dim elements (the others stay): for i < r/2 the pair (x_i, x_{i + r/2}) turns by
 * the angle pos * f_i,
 *   x_i' = x_i cos - x_{i+r/2} sin,   x_{i+r/2}' = x_{i+r/2} cos + x_i sin,
 * f_i = theta^(-2i/r), or inv_freq[i] where the caller gives its own frequencies.
 * Angles are formed and reduced in fp64, the products are fp32, and the result is
 * rounded once, to p->dtype or to 8-bit codes.
 *
 * Conventions are those of kara.h and kara_q8.h.
 */
#ifndef KARA_ROPE_H
#define KARA_ROPE_H

#include "kara_q8.h"

#ifdef __cplusplus
extern "C" {
#endif

typedef struct kara_rope {
  int32_t dim;           /* elements of a head that turn: a multiple of 16, head_dim at most; 0: head_dim */
  float theta;           /* base of the frequencies, finite and > 0; not used with inv_freq */
  const float* inv_freq; /* device, [dim / 2], 4-byte aligned, or NULL */
} kara_rope_t;

/*
 * Appends n_new tokens to each of the n sequences seqs[0..n) (distinct) in n_layers
 * layers, keys turned: rows k_new / v_new [n_layers][n][n_new][n_kv_heads][head_dim]
 * (p->dtype) of sequence s = seqs[j] go to its positions pos0 .. pos0 + n_new - 1, into
 * rows of p->dtype (k_scales and v_scales NULL) or 8-bit codes (both given).  Queries
 * q [n_layers][n][n_new][n_q_heads][head_dim], where given, are turned into q_out (the
 * same shape; it may be q, or else must not overlap it; both or neither).
 *
 *   counted  0: pos0 = seq_lens[s], and the call ends with seq_lens[s] += n_new and
 *               rope_pos[s] += n_new.
 *            1: the tokens are counted already, by the call of an earlier layer of the
 *               same step: pos0 = seq_lens[s] - n_new, the rotary positions begin
 *               at rope_pos[s] - n_new, and neither array changes.  A program that
 *               forms a layer's keys from the layer before passes its first layer
 *               with 0 and the others with 1.
 *   rope_pos [n_seqs] rotary position of each sequence's next token; NULL: its position
 *            in the cache.  (After compression or eviction a token's position counts
 *            what was cut; the cache's does not.  A cache in 8 bits is neither compressed nor evicted from.)
 *   status   as in kara_q8_append, KARA_SEQ_NONFINITE from 8-bit caches alone;
 *            BAD_WINDOW too where counted tokens are more than the sequence's.
 *            Flagged sequences' cache, lengths and q_out rows are left as they were.
 */
kara_status_t kara_rope_append(const kara_params_t* p, const kara_rope_t* rope, int32_t n, const int32_t* seqs,
                               int32_t n_new, int32_t n_layers, const void* q, const void* k_new, const void* v_new,
                               void* q_out, void* const* k_pools, void* const* v_pools, void* const* k_scales,
                               void* const* v_scales, const int32_t* block_table, int32_t* seq_lens,
                               int32_t* rope_pos, int32_t counted, int32_t* status, void* stream);

#ifdef __cplusplus
}
#endif

#endif /* KARA_ROPE_H */

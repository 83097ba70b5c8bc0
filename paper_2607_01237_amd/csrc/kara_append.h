// The check of a listed sequence before tokens are appended to it, shared by
// the appends of rows (kara_harness.hip), of 4-bit codes (kara_q4.hip) and with a
// rotation or into 8 bits (kara_store.hip).
#pragma once

#include "kara_internal.h"

namespace kara {
namespace {

constexpr int kAppendThreads = 256;

// Status of listed sequence j, by all threads of a workgroup; the same value
// in each.  counted: seq_lens holds the new tokens already.
template <class G>   // Geom, or its fields named here
__device__ inline int append_status(const G& g, int n, const int32_t* __restrict__ seqs, int n_new,
                             const int32_t* __restrict__ bt, const int32_t* __restrict__ seq_lens, int j, bool counted = false) {
  const int s = seqs[j];
  if (s < 0 || s >= g.n_seqs) return KARA_SEQ_BAD_INDEX;
  int dup = 0;
  for (int o = threadIdx.x; o < n; o += kAppendThreads) dup |= o != j && seqs[o] == s;
  const int64_t len = (int64_t)seq_lens[s] - (counted ? n_new : 0);
  const int64_t new_len = len + n_new;
  const bool fits = len >= 0 && new_len <= (int64_t)g.max_blocks * g.bs;
  int bad = 0;
  if (fits) {
    const int32_t* row = bt + (int64_t)s * g.max_blocks;
    for (int b = (int)(len / g.bs) + threadIdx.x; b < (int)((new_len + g.bs - 1) / g.bs); b += kAppendThreads) {
      const int pg = row[b];
      bad |= pg < 0 || pg >= g.num_pages;
    }
  }
  const int any = __syncthreads_or(dup | (bad << 1));
  // (the two flags come back as one "any": told apart by a second vote only
  // when something is wrong)
  if (!any) return fits ? KARA_SEQ_OK : KARA_SEQ_BAD_WINDOW;
  const int d = __syncthreads_or(dup) ? KARA_SEQ_DUP_TRIGGER : 0;
  const int p = __syncthreads_or(bad) ? KARA_SEQ_BAD_PAGE : 0;
  return d | p | (fits ? 0 : KARA_SEQ_BAD_WINDOW);
}

}  // namespace
}  // namespace kara

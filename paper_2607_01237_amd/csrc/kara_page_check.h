// The check of a sequence's pages before rows move in place, shared by window
// compaction (kara_pages.hip) and eviction (kara_evict.hip).
#pragma once

#include "kara_internal.h"

namespace kara {
namespace {

constexpr int kValidateThreads = 256;
// One buffer of LDS words, used as a bitmap of the pool's pages when it has
// that many bits (a duplicate is a bit already set: one pass over the row;
// 1,100 blocks 42 -> 6 us against the pairwise scan), else as a copy of the
// table row for the pairwise scan when the row fits, else not at all.
constexpr int kValidateLds = 8192;

// By all threads of a workgroup, the same value in each: KARA_SEQ_BAD_PAGE if
// one of the blocks [b0, b1) of a table row is on no page of the pool,
// KARA_SEQ_DUP_PAGE if one of them shares its page with another of [0, b1).
__device__ inline int pages_status(const int32_t* __restrict__ row, int b0, int b1, int num_pages,
                                   uint32_t (&lds)[kValidateLds]) {
  const int tid = threadIdx.x;
  int bad = 0, twice = 0;
  const int n_words = (num_pages + 31) / 32;
  if (n_words <= kValidateLds) {
    for (int i = tid; i < n_words; i += kValidateThreads) lds[i] = 0;
    __syncthreads();
    for (int b = tid; b < b0; b += kValidateThreads) {
      const int pg = row[b];
      if (pg >= 0 && pg < num_pages) atomicOr(&lds[pg >> 5], 1u << (pg & 31));
    }
    __syncthreads();
    for (int b = b0 + tid; b < b1; b += kValidateThreads) {
      const int pg = row[b];
      if (pg < 0 || pg >= num_pages) bad = 1;
      else twice |= (atomicOr(&lds[pg >> 5], 1u << (pg & 31)) >> (pg & 31)) & 1;
    }
  } else {
    const bool in_lds = b1 <= kValidateLds;
    if (in_lds)
      for (int b = tid; b < b1; b += kValidateThreads) lds[b] = (uint32_t)row[b];
    __syncthreads();
    for (int b = b0 + tid; b < b1; b += kValidateThreads) {
      const int pg = in_lds ? (int)lds[b] : row[b];
      if (pg < 0 || pg >= num_pages) {
        bad = 1;
        continue;
      }
      if (in_lds) {
        for (int c = 0; c < b; ++c) twice |= (int)lds[c] == pg;
      } else {
        for (int c = 0; c < b; ++c) twice |= row[c] == pg;
      }
    }
  }
  return (__syncthreads_or(bad) ? KARA_SEQ_BAD_PAGE : 0) | (__syncthreads_or(twice) ? KARA_SEQ_DUP_PAGE : 0);
}

}  // namespace
}  // namespace kara

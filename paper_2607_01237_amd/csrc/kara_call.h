// What the serving operators' launches pass to their kernels beside their own arguments.
#pragma once

#include "kara_internal.h"

namespace kara {

// The geometry that they use, and the pools of up to NL layers.  A launch passes its
// arguments by value and takes longer for more of them (a launch of 80, 270 and 1040 to 4000
// bytes: 2.9, 3.6 and 4.5 us of host time), so calls of two layers or fewer pass two.
struct Dims {
  int Hq, Hkv, G, bs, num_pages, max_blocks, n_seqs;
  float scale;
};
inline Dims dims_of(const Geom& g) { return {g.Hq, g.Hkv, g.G, g.bs, g.num_pages, g.max_blocks, g.n_seqs, g.scale}; }
constexpr int kFewLayers = 2;
template <int NL>
struct Pools {
  void* p[NL];
};

template <int NL>
void set_pools(Pools<NL>* x, const void* const* pools, int n_layers) {
  for (int i = 0; pools && i < n_layers; ++i) x->p[i] = const_cast<void*>(pools[i]);
}

}  // namespace kara

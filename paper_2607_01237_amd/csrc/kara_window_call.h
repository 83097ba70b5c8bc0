// Attention within a sliding window and the first tokens (include/kara_window.h): what
// the kernels of few query rows (kara_window.hip) and of many (kara_window_chunk.hip)
// share.
#pragma once

#include "kara_call.h"

namespace kara {

struct WindowHead {
  Dims g;
  int n, n_layers;
  int T;                      // queries per sequence, its last T positions
  int window, sink;           // at most kMaxLen; no window: kMaxLen
  int n_rt;                   // tiles of query rows of a (layer, sequence, KV head)
  int split_keys, n_splits, max_len;
  int run;                    // log2 of the keys that lie in one page wherever they start
  const int32_t *seqs, *bt, *seq_lens;
  const void* q;              // [n_layers][n][T][Hq][d]
  float *rec_o, *rec_ml;      // records [n_layers][n][T][Hq][n_splits]: o[d]; m, l
  void* out;                  // [n_layers][n][T][Hq][d]
};

template <int NL>
struct WindowCallOf : WindowHead {
  Pools<NL> kp, vp, ksp, vsp;   // rows, or codes and scales
};
using WindowCall = WindowCallOf<kMaxLayersPerLaunch>;

// Keys that a tile of query rows sees, numbered without the gap: key v is at position
// v while v < head, else at v + gap.  The numbers 0 .. n - 1 hold all of them, and a few
// that no row sees: both parts begin and the first ends at a multiple of 16, so that runs
// of up to 16 keys from a multiple of their length lie in one page wherever the block
// size allows it.
//
// In these numbers a query at position i sees v where
//   v <= i - gap  and  (v > i - gap - window  or  v < sink):
// with a gap, head is sink rounded up and lies below every row's window.
struct Span {
  int i0, i1;                 // first and last position of the rows
  int head, gap, n;
  __host__ __device__ int position(int v) const { return v < head ? v : v + gap; }
};

// rows [row0, row1) of queries at the last T of len positions, G rows a query
__host__ __device__ inline Span span_of(int len, int T, int G, int row0, int row1, int window, int sink) {
  Span s;
  s.i0 = len - T + row0 / G;
  s.i1 = len - T + (row1 - 1) / G;
  s.head = s.gap = 0;
  s.n = s.i1 + 1 > 0 ? s.i1 + 1 : 0;
  const int lo = (s.i0 - window + 1) & ~15;       // (negative: no gap)
  const int head = (sink + 15) & ~15;
  if (lo > head) {
    s.head = head;
    s.gap = lo - head;
    s.n -= s.gap;
  }
  return s;
}

// The most keys a tile's span holds.
inline int span_most(int T, int G, int rows, int window, int sink, int max_len) {
  const int64_t positions = ((int64_t)rows + G - 2) / G + 1 < T ? ((int64_t)rows + G - 2) / G + 1 : T;
  const int64_t most = (int64_t)window + positions - 1 + 15 + ((sink + 15) & ~15);
  return most < max_len ? (int)most : max_len;
}

// Many query rows over 8 bits or bf16 rows (kara_window_chunk.hip): bytes of workspace, and
// the launches.
struct WindowChunkPlan {
  int qt, rows_wg, n_rb;      // tiles of a wave, rows of a workgroup, row blocks of a unit
  bool split;                 // whether long sequences' keys may be split
  int64_t blocks;             // row blocks of the call
};
WindowChunkPlan window_chunk_plan(const Geom& g, int n, int n_layers, int T);
size_t window_chunk_workspace(const Geom& g, int n, int n_layers, int T);
hipError_t launch_window_chunk(const Geom& g, const WindowCall& a, const WindowChunkPlan& x, bool q8, void* workspace,
                               hipStream_t stream);

}  // namespace kara

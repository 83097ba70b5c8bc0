// Attention within a sliding window and the first tokens (include/kara_window.h) of few
// query rows, with the keys split over workgroups, and over rows of fp32; the 8-bit
// cache's attention (include/kara_q8.h), which is the same without a window.
#include <algorithm>
#include <type_traits>

#include "kara_lds.h"
#include "kara_q8_device.h"
#include "kara_window.h"
#include "kara_window_call.h"

namespace kara {
namespace {

constexpr float kLog2e = 1.4426950408889634f;
constexpr float kNegInf = -__builtin_huge_valf();
// Lower end of a running maximum: finite, so that a logit of -inf weighs 0.
constexpr float kMaxFloor = -3.402823466e38f;

constexpr int kThreads = 256;
constexpr int kWaves = kThreads / 64;
constexpr int kSplitMin = 512;       // keys per split, at least (of a span of more)
constexpr int kSplitMax = 4608;      // at most
constexpr int kSplitRuns = 1024;     // runs of keys a split's LDS table holds
constexpr int kWgsAtOnce = 512;      // workgroups that run at once, two to a CU

enum Cache { kRowsBf16, kRowsF32, kCodes };

template <Cache CT, int D, int QT>
struct WinCfg {
  static constexpr int kTB = CT == kRowsF32 ? 1 : 2;               // tiles of 16 keys per block
  static constexpr int kBlock = 16 * kTB;
  static constexpr int kRow = D * (CT == kRowsF32 ? 4 : CT == kRowsBf16 ? 2 : 1);
  static constexpr int kKC = kRow / 64;                            // 16-byte pieces of a key in a lane
  static constexpr int kE = D / 16;                                // columns of a lane
  static constexpr int kVB = kRow / 16;                            // bytes of a value row in a lane
  static constexpr int kVW = kVB / 4;
  // Blocks of values held: wide rows would take more registers than there are (spilled, they
  // cost a quarter of a long decoding step).  Then a block's values are on their way while
  // its logits are formed, the next block's keys behind them.
  static constexpr int kVBuf = kRow >= 256 ? 1 : 2;
  // With two tiles of rows its keys too are asked for behind the products of the present ones.
  static constexpr int kKBuf = kRow >= 256 && QT == 2 ? 1 : 2;
};

// One workgroup of four waves per (layer, sequence, KV head, tile of 16 QT query rows,
// split of split_keys keys of the tile's span): for the tile's rows, the split's maximum m,
// exponential sum l and unnormalised output o, in log2 units and fp32.  Rows of a (layer,
// sequence, KV head) run over (query, head in group).
//
// The pool rows of the split's keys go to LDS first; the four waves then take its blocks
// of 32 keys (16 of fp32) in turn, each with the next block on its way into registers
// while it works on the present one, straight from the pages in the layout of the matrix
// operands: S^T = K Q^T with a lane's pieces of one key as they lie (the query's pieces
// are taken the same way), and V as rows, d/16 columns of a key per lane.  A lane so holds
// four keys of one query per tile, and its weights are the B operand of O^T += V^T P^T as
// they stand; of 16-bit values, pairs of columns are put together to pairs of keys by
// byte permutes.
//
// Bound by the bytes where there are many: 96 sequences of 7-8.2K tokens, 2 layers, 40/8
// heads, d = 128: over codes 525 us for 2.99 GB, 5.7 TB/s; in a window of 4096 over rows 543
// us for 3.23 GB, 6.0 TB/s (the counters hold 3.05 and 3.24 GB).  A small batch is bound by the
// loads that wait for one another (list, length, table, keys): 8 sequences of 300-4000 tokens
// 15.8 us and the join 4.4.
//
// Rows of fp32 go through the fp32 matrix instructions, and are bound by those where queries
// are many: 6 x 101 queries of 16 heads, d = 64, in a window of 777, 28-32 us, 1.5 GFLOP (the
// card's fp32 rate in a large library product is 154 TFLOP/s).  NT: bf16 terms of a query over codes
// (3 where p->dtype is fp32: 24 bits; codes are exact in one).  NP: bf16 terms of a weight: 3,
// all its bits, but for bf16 calls over codes, where the third would cost what it does not over
// rows: 2.  In us with 2 and 3: over rows, a step of 8 sequences 16.1, 16.3; 96 x 2 layers of 8K
// in a window of 4096 543, 542; 5 queries there, no window, 1090, 1089.  Over codes, in the same
// order, no window, 19.4, 20.1; 528, 531; 617, 650.  (A weight rounded to bf16 would leave an
// output of flat weights 2.3e-3 off, two terms 1.66e-3, which is its own rounding.)
template <Cache CT, int NT, int NP, int D, int QT, int NL>
__global__ __launch_bounds__(kThreads, 2) void window_split_kernel(WindowCallOf<NL> a) {
  using C = WinCfg<CT, D, QT>;
  constexpr int kTileRows = 16 * QT;
  constexpr int TB = C::kTB, KC = C::kKC, E = C::kE, VW = C::kVW;
  constexpr bool F32 = CT == kRowsF32;
  constexpr bool kOutBf16 = !F32 && NT == 1;
  constexpr int KS = D / 32;                       // bf16 products per dot product
  struct Table {
    uint32_t row[kSplitRuns];                      // pool rows of runs of keys
    uint32_t scale[CT == kCodes ? kSplitRuns : 1]; // K's scale byte, V's above it
  };
  __shared__ __attribute__((aligned(16))) union {
    Table t;
    float o[kWaves][kTileRows][D];
  } lds;
  __shared__ float red_m[kWaves][kTileRows], red_l[kWaves][kTileRows];
  Table& tab = lds.t;

  const Dims& g = a.g;
  const int tid = threadIdx.x;
  const int lane = tid & 63;
  const int wave = __builtin_amdgcn_readfirstlane(tid >> 6);
  const int gq = lane >> 4, li = lane & 15;
  uint32_t rest = blockIdx.x;
  // (blocks go round the 8 XCDs: the splits of eight units in a row fall to the same ones,
  // those of the next eight are shifted, so that no XCD gets all the short last ones)
  const uint32_t unit8 = rest / ((uint32_t)a.n_splits * 8);
  const int split = (rest + unit8) % (uint32_t)a.n_splits;
  rest /= (uint32_t)a.n_splits;
  const int rt = rest % (uint32_t)a.n_rt;
  rest /= (uint32_t)a.n_rt;
  const int h = rest % (uint32_t)g.Hkv;
  rest /= (uint32_t)g.Hkv;
  const int j = rest % (uint32_t)a.n;
  const int l = rest / (uint32_t)a.n;
  const int s = a.seqs[j];
  const int G = g.G, T = a.T, R = G * T;
  const int len = s >= 0 && s < g.n_seqs ? a.seq_lens[s] : 0;
  // row r of the unit: output row orow + (r / G) * Hq + r % G
  const int64_t orow = ((int64_t)l * a.n + j) * T * g.Hq + h * G;
  const int row0 = rt * kTileRows;
  const int rows = min(kTileRows, R - row0);
  const bool none = len <= 0 || len > a.max_len;
  const Span sp = span_of(none ? 0 : len, T, G, row0, row0 + rows, a.window, a.sink);
  const int k0 = split * a.split_keys;
  if (none || k0 >= sp.n) {
    // no keys: zero rows, or a record marked so where the combine kernel follows
    if (a.n_splits > 1) {
      if (tid < rows) {
        const int r = row0 + tid;
        *(floatx2*)(a.rec_ml + 2 * ((orow + (int64_t)(r / G) * g.Hq + r % G) * a.n_splits + split)) = floatx2{kNegInf, 0.f};
      }
      return;
    }
    for (int i = tid; i < rows * D; i += kThreads) {
      const int r = row0 + i / D;
      const int64_t at = (orow + (int64_t)(r / G) * g.Hq + r % G) * D + i % D;
      if constexpr (kOutBf16) ((__bf16*)a.out)[at] = (__bf16)0.f;
      else ((float*)a.out)[at] = 0.f;
    }
    return;
  }
  const int nk = min(sp.n - k0, a.split_keys);                // keys of this split
  const float c = g.scale * kLog2e;
  const int nblk = (nk + C::kBlock - 1) / C::kBlock;

  // lane (gq, li): its pieces of query row li of each tile, and the keys that the row sees
  int qhi[QT], qlo[QT];                        // (sinks not counted; none: of a row that is not there)
  uint4 qraw[QT][F32 || NT > 1 ? D / 16 : KS];
#pragma unroll
  for (int qt = 0; qt < QT; ++qt) {
    const bool there = qt * 16 + li < rows;
    const int r = row0 + (there ? qt * 16 + li : 0);
    const int t = T == 1 ? 0 : r / G;
    qhi[qt] = there ? len - T + t - sp.gap : -1;
    qlo[qt] = there ? qhi[qt] - a.window + 1 : 0;
    const char* src = (const char*)a.q + (orow + (int64_t)t * g.Hq + (r - t * G)) * D * (kOutBf16 ? 2 : 4);
    if constexpr (F32) {
#pragma unroll
      for (int x = 0; x < KC; ++x) qraw[qt][x] = *(const uint4*)(src + (gq + 4 * x) * 16);
    } else if constexpr (CT == kRowsBf16) {
#pragma unroll
      for (int x = 0; x < KS; ++x) qraw[qt][x] = *(const uint4*)(src + (gq + 4 * x) * 16);
    } else {
      // (octet x lies in 16 codes: those of piece x / 2)
#pragma unroll
      for (int x = 0; x < KS; ++x) {
        const int at = (gq + 4 * (x >> 1)) * 16 + (x & 1) * 8;
        if constexpr (NT == 1) {
          qraw[qt][x] = *(const uint4*)(src + at * 2);
        } else {
          qraw[qt][2 * x] = *(const uint4*)(src + at * 4);
          qraw[qt][2 * x + 1] = *(const uint4*)(src + at * 4 + 16);
        }
      }
    }
  }
  // Pool rows of the split's keys: runs of 2^run keys lie in one page, an entry each.
  // (Keys that no row sees may be on no page: any row of the pool stands for them.)  The
  // scales go to LDS behind the first block's loads.
  const int run = a.run;
  const int runs = (nblk * C::kBlock) >> run;
  constexpr int kEntries = kSplitRuns / kThreads;
  uint32_t scale_pair[kEntries];
  {
    const int32_t* row_pages = a.bt + (int64_t)s * g.max_blocks;
#pragma unroll
    for (int k = 0; k < kEntries; ++k) {
      const int i = tid + k * kThreads;
      if (i < runs) {
        const int pos = sp.position(k0 + min(i << run, (nk - 1) >> run << run));
        const int b = pos / g.bs;
        const int page = min(max(row_pages[b], 0), g.num_pages - 1);
        const uint32_t unit = (uint32_t)page * (uint32_t)g.Hkv + (uint32_t)h;
        tab.row[i] = unit * (uint32_t)g.bs + (uint32_t)(pos - b * g.bs);
        if constexpr (CT == kCodes)
          scale_pair[k] = (uint32_t)((const uint8_t*)a.ksp.p[l])[unit] | (uint32_t)((const uint8_t*)a.vsp.p[l])[unit] << 16;
      }
    }
  }
  lds_barrier();
  const char* kbase = (const char*)a.kp.p[l] + gq * 16;
  const char* vbase = (const char*)a.vp.p[l] + li * (C::kVB < 16 ? C::kVB : 16);
  const int run_mask = (1 << run) - 1;
  // (padding keys past the last one repeat it)
  auto row_of = [&](int key) __attribute__((always_inline)) {
    key = min(key, nk - 1);
    return tab.row[key >> run] + (uint32_t)(key & run_mask);
  };
  auto scale_of = [&](int key) __attribute__((always_inline)) { return tab.scale[min(key, nk - 1) >> run]; };
  uint4 kb[C::kKBuf][TB][KC];
  uint32_t vb[C::kVBuf][TB][4][VW];
  auto load_k = [&](int blk, int b) __attribute__((always_inline)) {
    uint64_t kat[TB];
#pragma unroll
    for (int t = 0; t < TB; ++t) kat[t] = (uint64_t)row_of(blk * C::kBlock + t * 16 + li) * C::kRow;
#pragma unroll
    for (int t = 0; t < TB; ++t)
#pragma unroll
      for (int x = 0; x < KC; ++x) kb[b][t][x] = *(const uint4*)(kbase + kat[t] + x * 64);
  };
  auto load_v = [&](int blk, int b) __attribute__((always_inline)) {
    uint64_t vat[TB][4];
#pragma unroll
    for (int t = 0; t < TB; ++t)
#pragma unroll
      for (int r = 0; r < 4; ++r) vat[t][r] = (uint64_t)row_of(blk * C::kBlock + t * 16 + 4 * gq + r) * C::kRow;
#pragma unroll
    for (int t = 0; t < TB; ++t)
#pragma unroll
      for (int r = 0; r < 4; ++r) {
        const char* src = vbase + vat[t][r];
        if constexpr (VW == 1) {
          vb[b][t][r][0] = *(const uint32_t*)src;
        } else if constexpr (VW == 2) {
          const uint2 v = *(const uint2*)src;
          vb[b][t][r][0] = v.x, vb[b][t][r][1] = v.y;
        } else {
          // (fp32 at d = 128: columns 4li.. and 64 + 4li..)
#pragma unroll
          for (int y = 0; y < VW / 4; ++y) {
            const uint4 v = *(const uint4*)(src + y * 256);
            vb[b][t][r][4 * y] = v.x, vb[b][t][r][4 * y + 1] = v.y, vb[b][t][r][4 * y + 2] = v.z, vb[b][t][r][4 * y + 3] = v.w;
          }
        }
      }
  };

  constexpr int V1 = C::kVBuf - 1;
  if (wave < nblk) {
    load_k(wave, 0);
    if constexpr (V1) load_v(wave, 0);
  }
  if constexpr (CT == kCodes) {
#pragma unroll
    for (int k = 0; k < kEntries; ++k)
      if (tid + k * kThreads < runs) tab.scale[tid + k * kThreads] = scale_pair[k];
    lds_barrier();
  }
  bf16x8 qa[QT][F32 ? 1 : NT][KS];
#pragma unroll
  for (int qt = 0; qt < QT; ++qt) {
    const bool there = qt * 16 + li < rows;
    if constexpr (!F32) {
#pragma unroll
      for (int x = 0; x < KS; ++x) {
        if constexpr (NT == 1) {
          qa[qt][0][x] = __builtin_bit_cast(bf16x8, there ? qraw[qt][x] : uint4{0, 0, 0, 0});
        } else {
          const floatx4 u = __builtin_bit_cast(floatx4, qraw[qt][2 * x]);
          const floatx4 v = __builtin_bit_cast(floatx4, qraw[qt][2 * x + 1]);
          uint32_t w[4][NT];
#pragma unroll
          for (int i = 0; i < 4; ++i) {
            const float x0 = i < 2 ? u[2 * i] : v[2 * i - 4], x1 = i < 2 ? u[2 * i + 1] : v[2 * i - 3];
            bf16_term_pairs<true>(there ? x0 : 0.f, there ? x1 : 0.f, w[i]);
          }
#pragma unroll
          for (int y = 0; y < NT; ++y) qa[qt][y][x] = __builtin_bit_cast(bf16x8, uint4{w[0][y], w[1][y], w[2][y], w[3][y]});
        }
      }
    } else {
#pragma unroll
      for (int x = 0; x < KC; ++x) qraw[qt][x] = there ? qraw[qt][x] : uint4{0, 0, 0, 0};
    }
  }
  float m[QT], lsum[QT];             // query li's reference, and this lane's part of its sum
  floatx4 lones[QT];                 // bf16: the sum, in every element
  floatx4 o[QT][E];                  // query li, column e of lanes 4gq + r
#pragma unroll
  for (int qt = 0; qt < QT; ++qt) {
    m[qt] = kMaxFloor, lsum[qt] = 0.f;
    lones[qt] = floatx4{0.f, 0.f, 0.f, 0.f};
#pragma unroll
    for (int e = 0; e < E; ++e) o[qt][e] = floatx4{0.f, 0.f, 0.f, 0.f};
  }
  bf16x8 ones;
#pragma unroll
  for (int i = 0; i < 8; ++i) ones[i] = (__bf16)1.f;

  // keys that some row sees, and that every row sees (sinks not counted)
  const int any_lo = sp.i0 - a.window + 1 - sp.gap, any_hi = sp.n - 1;
  const int all_lo = sp.i1 - a.window + 1 - sp.gap, all_hi = sp.i0 - sp.gap;
  auto in = [&](int v, int lo, int hi) __attribute__((always_inline)) { return v <= hi && (v >= lo || v < a.sink); };

  bool careful = false;              // (rows) whether infinite and NaN values are taken apart
  // block blk, its keys in buffer b and values in vbuf; next: the block whose keys follow
  // into one buffer
  auto work = [&](int blk, int b, int vbuf, int next) __attribute__((always_inline)) {
    floatx4 sv[QT][TB];
#pragma unroll
    for (int t = 0; t < TB; ++t) {
#pragma unroll
      for (int qt = 0; qt < QT; ++qt) sv[qt][t] = floatx4{0.f, 0.f, 0.f, 0.f};
      if constexpr (F32) {
#pragma unroll
        for (int x = 0; x < KC; ++x) {
          const floatx4 ka = __builtin_bit_cast(floatx4, kb[b][t][x]);
#pragma unroll
          for (int i = 0; i < 4; ++i)
#pragma unroll
            for (int qt = 0; qt < QT; ++qt)
              sv[qt][t] = __builtin_amdgcn_mfma_f32_16x16x4f32(ka[i], __builtin_bit_cast(floatx4, qraw[qt][x])[i], sv[qt][t], 0, 0, 0);
        }
      } else {
        float scale = 0.f;
        if constexpr (CT == kCodes) scale = q8_scale(scale_of(blk * C::kBlock + t * 16 + li) & 255);
#pragma unroll
        for (int x = 0; x < KS; ++x) {
          bf16x8 ka;
          if constexpr (CT == kCodes) {
            const uint4 w = kb[b][t][x >> 1];
            ka = x & 1 ? q8_octet(w.z, w.w, scale) : q8_octet(w.x, w.y, scale);
          } else {
            ka = __builtin_bit_cast(bf16x8, kb[b][t][x]);
          }
#pragma unroll
          for (int y = NT - 1; y >= 0; --y)
#pragma unroll
            for (int qt = 0; qt < QT; ++qt) sv[qt][t] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(ka, qa[qt][y][x], sv[qt][t], 0, 0, 0);
        }
      }
    }
    // Wait states between the last product and the first read of its result, which lies
    // past a branch: the compiler does not count across it.
#pragma unroll
    for (int t = 0; t < TB; ++t)
#pragma unroll
      for (int qt = 0; qt < QT; ++qt) asm volatile("s_nop 7\n\ts_nop 3" : "+v"(sv[qt][t]));
    if constexpr (C::kKBuf == 1)
      if (next < nblk) load_k(next, 0);
    // values as the second products take them: of 16 bits, pairs of columns
    constexpr int VP = F32 ? E : E / 2;
    uint32_t pv[TB * 4][VP];
#pragma unroll
    for (int t = 0; t < TB; ++t)
#pragma unroll
      for (int r = 0; r < 4; ++r) {
        if constexpr (CT == kCodes) {
          const float scale = q8_scale(scale_of(blk * C::kBlock + t * 16 + 4 * gq + r) >> 16);
#pragma unroll
          for (int y = 0; y < VW; ++y) {
            pv[4 * t + r][2 * y] = q8_pair<false>(vb[vbuf][t][r][y], scale);
            pv[4 * t + r][2 * y + 1] = q8_pair<true>(vb[vbuf][t][r][y], scale);
          }
        } else {
#pragma unroll
          for (int y = 0; y < VP; ++y) pv[4 * t + r][y] = vb[vbuf][t][r][y];
        }
      }
    const int v0 = k0 + blk * C::kBlock;
    bool odd_values = false;
    const bool masked = v0 < all_lo || v0 + C::kBlock - 1 > all_hi;
    if (masked) {
#pragma unroll
      for (int t = 0; t < TB; ++t)
#pragma unroll
        for (int r = 0; r < 4; ++r) {
          const int v = v0 + t * 16 + 4 * gq + r;
#pragma unroll
          for (int qt = 0; qt < QT; ++qt)
            if (!in(v, qlo[qt], qhi[qt])) sv[qt][t][r] = kNegInf;
          // what no row sees may be anything: its weights are 0, its values must be finite
          if (!in(v, any_lo, any_hi))
#pragma unroll
            for (int y = 0; y < VP; ++y) pv[4 * t + r][y] = 0;
        }
    }
    if (CT != kCodes && careful) {
      uint32_t hit = 0;
#pragma unroll
      for (int i = 0; i < TB * 4; ++i)
#pragma unroll
        for (int y = 0; y < VP; ++y) {
          if constexpr (F32) hit |= (pv[i][y] & 0x7fffffffu) >= 0x7f800000u;
          else hit |= ((pv[i][y] & 0x7fff7fffu) + 0x00800080u) & 0x80008000u;
        }
      odd_values = __ballot(hit != 0) != 0ull;
      if (odd_values) {
#pragma unroll
        for (int i = 0; i < TB * 4; ++i)
#pragma unroll
          for (int y = 0; y < VP; ++y) {
            if constexpr (F32) {
              if ((pv[i][y] & 0x7fffffffu) >= 0x7f800000u) pv[i][y] = 0;
            } else {
              if ((pv[i][y] & 0x7f80u) == 0x7f80u) pv[i][y] &= 0xffff0000u;
              if ((pv[i][y] & 0x7f800000u) == 0x7f800000u) pv[i][y] &= 0xffffu;
            }
          }
      }
    }
    bf16x8 pb[QT][F32 ? 1 : NP];           // terms of the lane's eight weights
    float p[QT][TB][4];
#pragma unroll
    for (int qt = 0; qt < QT; ++qt) {
      float mx = sv[qt][0][0];
#pragma unroll
      for (int t = 0; t < TB; ++t)
#pragma unroll
        for (int r = 0; r < 4; ++r) mx = fmaxf(mx, sv[qt][t][r]);
      // The reference m, one for the four lanes of a query, is raised only where a
      // logit passes it by more than 2^8: no exchange between lanes before that.
      if (__ballot(mx * c > m[qt] + 8.f) != 0ull) {
        mx = fmaxf(mx, __shfl_xor(mx, 16, 64));
        mx = fmaxf(mx, __shfl_xor(mx, 32, 64)) * c;
        const float mn = fmaxf(m[qt], mx);
        const float f = __builtin_amdgcn_exp2f(m[qt] - mn);
        m[qt] = mn;
        lsum[qt] *= f;
        lones[qt] *= f;
#pragma unroll
        for (int e = 0; e < E; ++e) o[qt][e] *= f;
      }
#pragma unroll
      for (int t = 0; t < TB; ++t)
#pragma unroll
        for (int r = 0; r < 4; ++r) p[qt][t][r] = __builtin_amdgcn_exp2f(fmaf(sv[qt][t][r], c, -m[qt]));
      if constexpr (F32) {
#pragma unroll
        for (int r = 0; r < 4; ++r) lsum[qt] += p[qt][0][r];
      } else {
        uint32_t pw[NP][4];                  // in pairs
#pragma unroll
        for (int t = 0; t < 2; ++t)
#pragma unroll
          for (int r = 0; r < 4; r += 2) {
            if constexpr (!kOutBf16) lsum[qt] += p[qt][t][r] + p[qt][t][r + 1];
            uint32_t w[NP];
            bf16_term_pairs<false>(p[qt][t][r], p[qt][t][r + 1], w);
#pragma unroll
            for (int y = 0; y < NP; ++y) pw[y][2 * t + (r >> 1)] = w[y];
          }
#pragma unroll
        for (int y = 0; y < NP; ++y) pb[qt][y] = __builtin_bit_cast(bf16x8, uint4{pw[y][0], pw[y][1], pw[y][2], pw[y][3]});
        // (of bf16 calls the sum is one more product, with ones, of the weights as they are held)
        if constexpr (kOutBf16)
#pragma unroll
          for (int y = NP - 1; y >= 0; --y)
            lones[qt] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(ones, pb[qt][y], lones[qt], 0, 0, 0);
      }
    }
    if constexpr (F32) {
#pragma unroll
      for (int r = 0; r < 4; ++r)
#pragma unroll
        for (int e = 0; e < E; ++e)
#pragma unroll
          for (int qt = 0; qt < QT; ++qt)
            o[qt][e] = __builtin_amdgcn_mfma_f32_16x16x4f32(__uint_as_float(pv[r][e]), p[qt][0][r], o[qt][e], 0, 0, 0);
    } else {
#pragma unroll
      for (int e = 0; e < E; ++e) {
        const uint32_t sel = (e & 1) ? 0x07060302u : 0x05040100u;
        const uint4 va = {__builtin_amdgcn_perm(pv[1][e >> 1], pv[0][e >> 1], sel),
                          __builtin_amdgcn_perm(pv[3][e >> 1], pv[2][e >> 1], sel),
                          __builtin_amdgcn_perm(pv[5][e >> 1], pv[4][e >> 1], sel),
                          __builtin_amdgcn_perm(pv[7][e >> 1], pv[6][e >> 1], sel)};
#pragma unroll
        for (int y = NP - 1; y >= 0; --y)
#pragma unroll
          for (int qt = 0; qt < QT; ++qt)
            o[qt][e] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(__builtin_bit_cast(bf16x8, va), pb[qt][y], o[qt][e], 0, 0, 0);
      }
    }
    if constexpr (CT != kCodes) {
      if (odd_values) {
        // infinite and NaN values, taken out above: added where they are seen (a weight
        // is positive), key by key, the rows read again
#pragma unroll
        for (int qt = 0; qt < QT; ++qt)
#pragma unroll
          for (int e = 0; e < E; ++e) asm volatile("s_nop 7\n\ts_nop 3" : "+v"(o[qt][e]));
        for (int key = 0; key < C::kBlock; ++key) {
          if (!in(v0 + key, any_lo, any_hi)) continue;
          const char* row = (const char*)a.vp.p[l] + (uint64_t)row_of(blk * C::kBlock + key) * C::kRow;
#pragma unroll
          for (int r = 0; r < 4; ++r)
#pragma unroll
            for (int e = 0; e < E; ++e) {
              const int col = F32 && E == 8 ? (e >> 2) * 64 + 4 * (4 * gq + r) + (e & 3) : E * (4 * gq + r) + e;
              uint32_t x;
              if constexpr (F32) x = ((const uint32_t*)row)[col];
              else x = (uint32_t)((const uint16_t*)row)[col] << 16;
              if ((x & 0x7fffffffu) >= 0x7f800000u)
#pragma unroll
                for (int qt = 0; qt < QT; ++qt)
                  if (in(v0 + key, qlo[qt], qhi[qt])) o[qt][e][r] += __uint_as_float(x);
            }
        }
      }
    }
  };
  // the next block's keys after this block's values, so that waiting for the values
  // leaves the keys on their way
  // the wave's blocks, the first one's loads made
  for (;;) {
    if constexpr (C::kKBuf == 1) {
      for (int blk = wave; blk < nblk; blk += kWaves) {
        load_v(blk, 0);
        work(blk, 0, 0, blk + kWaves);
      }
    } else if (wave < nblk) {
      int blk = wave;
      for (;;) {
        const int n1 = blk + kWaves;
        if constexpr (!V1) load_v(blk, 0);
        if (n1 < nblk) {
          load_k(n1, 1);
          if constexpr (V1) load_v(n1, 1);
        }
        work(blk, 0, 0, 0);
        if (n1 >= nblk) break;
        blk = n1 + kWaves;
        if constexpr (!V1) load_v(n1, 0);
        if (blk < nblk) {
          load_k(blk, 0);
          if constexpr (V1) load_v(blk, 0);
        }
        work(n1, 1, V1, 0);
        if (blk >= nblk) break;
      }
    }
    // An infinite or NaN value that a row does not see has met its weight of 0 in the
    // products, and one that it sees a later term of its weight, which may be 0: where a
    // result is not finite (codes are), the wave's blocks again with such values apart.
    if (CT == kCodes || careful) break;
    floatx4 zero = {0.f, 0.f, 0.f, 0.f};
#pragma unroll
    for (int qt = 0; qt < QT; ++qt)
#pragma unroll
      for (int e = 0; e < E; ++e) {
        asm volatile("s_nop 7\n\ts_nop 3" : "+v"(o[qt][e]));
#pragma unroll
        for (int r = 0; r < 4; ++r) zero[r] = fmaf(o[qt][e][r], 0.f, zero[r]);
      }
    if (__ballot(!(zero[0] + zero[1] + zero[2] + zero[3] == 0.f)) == 0ull) break;
    careful = true;
#pragma unroll
    for (int qt = 0; qt < QT; ++qt) {
      m[qt] = kMaxFloor, lsum[qt] = 0.f;
      lones[qt] = floatx4{0.f, 0.f, 0.f, 0.f};
#pragma unroll
      for (int e = 0; e < E; ++e) o[qt][e] = floatx4{0.f, 0.f, 0.f, 0.f};
    }
    load_k(wave, 0);                 // (a wave without blocks has sums of 0)
    if constexpr (V1) load_v(wave, 0);
  }

  // ---- the waves' sums ----
#pragma unroll
  for (int qt = 0; qt < QT; ++qt) {
#pragma unroll
    for (int e = 0; e < E; ++e) asm volatile("s_nop 7\n\ts_nop 3" : "+v"(o[qt][e]));   // (as above, past the loop's branch)
    if constexpr (kOutBf16) {
      asm volatile("s_nop 7\n\ts_nop 3" : "+v"(lones[qt]));
      lsum[qt] = lones[qt][0];
    } else {
      lsum[qt] += __shfl_xor(lsum[qt], 16, 64);
      lsum[qt] += __shfl_xor(lsum[qt], 32, 64);
    }
    if (gq == 0) {
      red_m[wave][qt * 16 + li] = m[qt];
      red_l[wave][qt * 16 + li] = lsum[qt];
    }
  }
  __syncthreads();   // the table is no longer read
#pragma unroll
  for (int qt = 0; qt < QT; ++qt)
#pragma unroll
    for (int r = 0; r < 4; ++r)
#pragma unroll
      for (int e = 0; e < E; e += 4) {
        const int col = F32 && E == 8 ? (e >> 2) * 64 + 4 * (4 * gq + r) : E * (4 * gq + r) + e;
        *(floatx4*)&lds.o[wave][qt * 16 + li][col] = floatx4{o[qt][e][r], o[qt][e + 1][r], o[qt][e + 2][r], o[qt][e + 3][r]};
      }
  __syncthreads();
  const bool direct = a.n_splits == 1;
  for (int x = tid; x < rows * D; x += kThreads) {
    const int i = x / D, e = x - i * D;
    // (a wave without keys left its start: a maximum below all, sums of 0)
    float wm[kWaves], M = kMaxFloor, L = 0.f, O = 0.f;
#pragma unroll
    for (int w = 0; w < kWaves; ++w) M = fmaxf(M, wm[w] = red_m[w][i]);
#pragma unroll
    for (int w = 0; w < kWaves; ++w) {
      const float f = __builtin_amdgcn_exp2f(wm[w] - M);
      L = fmaf(red_l[w][i], f, L);
      O = fmaf(lds.o[w][i][e], f, O);
    }
    const int r = row0 + i, t = T == 1 ? 0 : r / G;
    const int64_t at = orow + (int64_t)t * g.Hq + (r - t * G);
    if (direct) {
      const float v = L == 0.f ? 0.f : O / L;   // (a row that sees no key)
      if constexpr (kOutBf16) ((__bf16*)a.out)[at * D + e] = (__bf16)v;
      else ((float*)a.out)[at * D + e] = v;
    } else {
      const int64_t rec = at * a.n_splits + split;
      if (e == 0) a.rec_ml[2 * rec] = M, a.rec_ml[2 * rec + 1] = L;
      a.rec_o[rec * D + e] = O;
    }
  }
}

// One wave per output row: its splits' records joined, but those without keys (a maximum of
// -inf; their sums were not written).  A record of weights that are all 0 is joined: its
// values may not be finite, which a row of one split would show.  Nothing is looked up but the records, and those of up to
// eight splits are all asked for at once: a launch of a few rows takes as long as its loads
// that wait for others.
template <int D, bool OUT_BF16>
__global__ __launch_bounds__(256) void window_combine_kernel(const float* __restrict__ rec_o, const float* __restrict__ rec_ml,
                                                             void* __restrict__ out, int n_splits, int64_t n_rows) {
  constexpr int kDPerLane = D / 64, kAtOnce = 8;
  typedef float floatd __attribute__((ext_vector_type(kDPerLane)));
  const int lane = threadIdx.x & 63;
  const int64_t row = (int64_t)blockIdx.x * 4 + (threadIdx.x >> 6);   // (l, j, t, hq)
  if (row >= n_rows) return;
  const floatx2* ml = (const floatx2*)rec_ml + row * n_splits;
  const float* v = rec_o + row * n_splits * D + lane * kDPerLane;
  auto load = [&](int from, floatd (&x)[kAtOnce]) __attribute__((always_inline)) {
#pragma unroll
    for (int i = 0; i < kAtOnce; ++i) __builtin_memcpy(&x[i], v + (int64_t)min(from + i, n_splits - 1) * D, sizeof(x[i]));
  };
  floatd x[kAtOnce];
  load(0, x);
  // lane i: split i's maximum and sum, 64 at a time, the first kept
  const floatx2 first = lane < n_splits ? ml[lane] : floatx2{kNegInf, 0.f};
  float M = first[0];
  for (int i = lane + 64; i < n_splits; i += 64) M = fmaxf(M, ml[i][0]);
#pragma unroll
  for (int i = 1; i < 64; i <<= 1) M = fmaxf(M, __shfl_xor(M, i, 64));
  float L = 0.f, acc[kDPerLane] = {};
  for (int s0 = 0; s0 < n_splits; s0 += 64) {
    const floatx2 mine = s0 == 0 ? first : s0 + lane < n_splits ? ml[s0 + lane] : floatx2{kNegInf, 0.f};
    const float f = __builtin_amdgcn_exp2f(mine[0] - M), lf = mine[1] * f;
    const int cnt = min(64, n_splits - s0);
    for (int i0 = 0; i0 < cnt; i0 += kAtOnce) {
      if (s0 + i0 > 0) load(s0 + i0, x);
#pragma unroll
      for (int i = 0; i < kAtOnce; ++i) {
        const float fi = __shfl(f, i0 + i, 64), li = __shfl(lf, i0 + i, 64);
        const bool in = i0 + i < cnt && __shfl(mine[0], i0 + i, 64) != kNegInf;
        if (in) {
          L += li;
#pragma unroll
          for (int e = 0; e < kDPerLane; ++e) acc[e] = fmaf(x[i][e], fi, acc[e]);
        }
      }
    }
  }
#pragma unroll
  for (int e = 0; e < kDPerLane; ++e) {
    const float y = L == 0.f ? 0.f : acc[e] / L;   // (a row that sees no key)
    if constexpr (OUT_BF16) ((__bf16*)out)[row * D + lane * kDPerLane + e] = (__bf16)y;
    else ((float*)out)[row * D + lane * kDPerLane + e] = y;
  }
}

int run_of(int bs) { return std::min(4, __builtin_ctz((unsigned)bs)); }

// Splits of a span into parts of one length, a multiple of 64: as many as run at once with
// the other tiles', each of 512 keys at least, or as the longest parts make where there are
// more tiles than that.  Parts of 256, 512, 1K, 2K keys, us: 8 sequences of 300-4000 tokens,
// 64 tiles 29.9, 22.7, 22.5, 28.9; 13 x 5 queries of 16 heads, 78 tiles 24.4, 21.4, 23.0,
// 30.2.  Parts of 1K, 2K, 4.1K, whole: 96 x 2 layers of 8K, 1536 tiles 566, 539, 532, 516; a
// window of 4096 there 577, 561, 541; of 64 sequences, 512 tiles 138, 132, 124.  (Whole
// sequences of all lengths would end with the longest.)
int split_most(int bs) { return std::min(kSplitMax, kSplitRuns << run_of(bs)); }
int split_keys_of(int bs, int64_t tiles, int span) {
  const int64_t longest = split_most(bs), few = ((int64_t)span + kSplitMin - 1) / kSplitMin;
  const int64_t n = std::min(few, std::max((span + longest - 1) / longest, (kWgsAtOnce + tiles - 1) / tiles));
  return (int)(((span + n - 1) / n + 63) / 64 * 64);
}

// Up to this many query rows per (layer, sequence, KV head) go through the split kernel,
// 16 or 32 a workgroup, and all over rows of fp32; more through the chunk kernel.  From 33 to
// 64 rows a tile of the two passes the keys on its own, where the chunk kernel would pass them
// once but hold a weight in one bf16 term: 96 x 2 layers of 8K, 40 and 60 rows, rows 1670 and
// 1695 us, there 1300; codes 1030 and 1080, there 1030; 16 of 300-4000 tokens, one layer, rows 69
// and 71, there 52, codes 55 and 56, there 53; in a window of 1024 of 96 x 2 rows 255 and 263,
// there 263.  The weights' bits decided.
constexpr int kFewRows = 64;
bool splits(const Geom& g, int T, bool q8) { return (int64_t)g.G * T <= kFewRows || (g.dtype == KARA_F32 && !q8); }

// a grid of one dimension, of 256 threads a block: HIP counts its threads in 32 bits
bool grid_ok(int64_t blocks) { return blocks > 0 && blocks < ((int64_t)1 << 24); }

bool layers_ok(int32_t n, int32_t n_layers) { return n >= 0 && n_layers >= 1 && n_layers <= kMaxLayersPerLaunch; }

template <int NL>
void set_pools(WindowCallOf<NL>* a, const void* const* k, const void* const* v, const void* const* ks, const void* const* vs) {
  set_pools(&a->kp, k, a->n_layers);
  set_pools(&a->vp, v, a->n_layers);
  set_pools(&a->ksp, ks, a->n_layers);
  set_pools(&a->vsp, vs, a->n_layers);
}

template <Cache CT, int NT, int NP, int QT, int NL>
void launch_split(int d, const WindowCallOf<NL>& a, int64_t blocks, hipStream_t s) {
  if (d == 128) hipLaunchKernelGGL((window_split_kernel<CT, NT, NP, 128, QT, NL>), dim3((unsigned)blocks), dim3(kThreads), 0, s, a);
  else hipLaunchKernelGGL((window_split_kernel<CT, NT, NP, 64, QT, NL>), dim3((unsigned)blocks), dim3(kThreads), 0, s, a);
}
template <int NL>
hipError_t launch_split(const Geom& g, bool q8, int rows, const WindowCallOf<NL>& a, int64_t blocks, hipStream_t s) {
  if (g.dtype == KARA_F32) {
    if (q8) launch_split<kCodes, 3, 3, 1>(g.d, a, blocks, s);
    else launch_split<kRowsF32, 1, 1, 1>(g.d, a, blocks, s);
  } else if (rows == 16) {
    if (q8) launch_split<kCodes, 1, 2, 1>(g.d, a, blocks, s);
    else launch_split<kRowsBf16, 1, 3, 1>(g.d, a, blocks, s);
  } else {
    if (q8) launch_split<kCodes, 1, 2, 2>(g.d, a, blocks, s);
    else launch_split<kRowsBf16, 1, 3, 2>(g.d, a, blocks, s);
  }
  return hipGetLastError();
}

// Query rows of a workgroup.  bf16: 32 where there are more than 16, so that the keys pass
// once, but in small launches: 96 x 5 queries x 2 layers of 8K, 25 rows a KV head: rows 1667
// -> 1088 us, codes 858 -> 623; 8 x 5 over 300-4000 tokens, 128 tiles of 16: 28.1, 29.9 so; 8
// x 16, 256 tiles 41.7, 39.0 so.  fp32 is bound by its products, and workgroups of 32 rows are
// fewer: 6 x 101 queries of 16 heads 32 us, 44 so.
int tile_rows(const Geom& g, int n, int n_layers, int T) {
  const int64_t tiles = (int64_t)n_layers * n * g.Hkv * (((int64_t)g.G * T + 15) / 16);
  return (int64_t)g.G * T <= 16 || g.dtype == KARA_F32 || tiles < 256 ? 16 : 32;
}

// q8: whether the cache is of codes (the size over either is the same where it says nothing)
kara_status_t workspace_size(const kara_params_t* p, int32_t n, int32_t n_layers, int32_t n_query, int32_t window,
                             int32_t n_sink, int32_t max_len, bool q8, size_t* bytes) {
  Geom g;
  const kara_status_t st = make_geom(p, n, &g);
  if (st != KARA_OK) return st;
  if (!bytes || !layers_ok(n, n_layers) || n_query < 1 || window < 0 || n_sink < 0 || max_len < 1 ||
      (int64_t)max_len > (int64_t)g.max_blocks * g.bs || (int64_t)n_query * g.Hq > INT32_MAX / 4)
    return KARA_ERR_INVALID_ARG;
  if (max_len > kMaxLen) return KARA_ERR_UNSUPPORTED;
  const int w = window == 0 ? kMaxLen : std::min(window, kMaxLen), sink = std::min(n_sink, kMaxLen);
  const size_t rec = (g.d + 2) * sizeof(float);
  const int64_t rows = (int64_t)n_layers * n * n_query * g.Hq;
  if (splits(g, n_query, q8)) {
    const int tile = tile_rows(g, n, n_layers, n_query);
    const int span = span_most(n_query, g.G, tile, w, sink, max_len);
    // (a tile has no more than `few` splits, and no more than the longest ones make or
    // kWgsAtOnce over the tiles: either way their records grow with the tiles)
    const int64_t longest = split_most(g.bs), few = ((int64_t)span + kSplitMin - 1) / kSplitMin;
    const int64_t tiles = (int64_t)n_layers * n * g.Hkv * (((int64_t)g.G * n_query + tile - 1) / tile);
    const int64_t many = std::max(rows * (((int64_t)span + longest - 1) / longest), (kWgsAtOnce + tiles) * tile);
    *bytes = few == 1 ? 0 : (size_t)std::min(rows * few, many) * rec;
  } else {
    *bytes = window_chunk_workspace(g, n, n_layers, n_query);
  }
  return KARA_OK;
}

kara_status_t attend(const kara_params_t* p, int32_t n, const int32_t* seqs, int32_t n_layers, int32_t n_query,
                     int32_t window, int32_t n_sink, const void* q, const void* const* k_pools,
                     const void* const* v_pools, const void* const* k_scales, const void* const* v_scales,
                     const int32_t* block_table, const int32_t* seq_lens, int32_t max_len, void* out, void* workspace,
                     size_t workspace_bytes, void* stream) {
  if ((k_scales == nullptr) != (v_scales == nullptr)) return KARA_ERR_INVALID_ARG;
  const bool q8 = k_scales != nullptr;
  size_t need = 0;
  kara_status_t st = workspace_size(p, n, n_layers, n_query, window, n_sink, max_len, q8, &need);
  if (st != KARA_OK) return st;
  if (n == 0) return KARA_OK;
  if (!seqs || !q || !block_table || !seq_lens || !out || !pools_ok(k_pools, n_layers) || !pools_ok(v_pools, n_layers) ||
      (q8 && (!pools_ok(k_scales, n_layers) || !pools_ok(v_scales, n_layers))))
    return KARA_ERR_INVALID_ARG;
  if (need && (!workspace || workspace_bytes < need)) return KARA_ERR_WORKSPACE;
  if (!aligned(16, {q, out, need ? workspace : nullptr}) || !aligned(4, {seqs, block_table, seq_lens}) ||
      !pools_aligned(16, k_pools, n_layers) || !pools_aligned(16, v_pools, n_layers))
    return KARA_ERR_INVALID_ARG;
  Geom g;
  st = make_geom(p, n, &g);
  if (st != KARA_OK) return st;
  WindowHead a{};
  a.g = dims_of(g);
  a.n = n;
  a.n_layers = n_layers;
  a.T = n_query;
  a.window = window == 0 ? kMaxLen : std::min(window, kMaxLen);
  a.sink = std::min(n_sink, kMaxLen);
  a.run = run_of(g.bs);
  a.max_len = max_len;
  const bool few = splits(g, n_query, q8), f32 = g.dtype == KARA_F32;
  const int tile = tile_rows(g, n, n_layers, n_query);
  const int64_t rows = (int64_t)n_layers * n * n_query * g.Hq;
  WindowChunkPlan plan{};
  int64_t blocks;
  if (few) {
    a.n_rt = (int)(((int64_t)g.G * n_query + tile - 1) / tile);
    const int64_t tiles = (int64_t)n_layers * n * g.Hkv * a.n_rt;
    const int span = span_most(n_query, g.G, tile, a.window, a.sink, max_len);
    a.split_keys = split_keys_of(g.bs, tiles, span);
    a.n_splits = (span + a.split_keys - 1) / a.split_keys;
    blocks = tiles * a.n_splits;
  } else {
    plan = window_chunk_plan(g, n, n_layers, n_query);
    a.n_rt = plan.n_rb;
    a.n_splits = 1;
    blocks = 2 * plan.blocks;           // (of 512 threads)
  }
  // (the launch that joins records takes four output rows a workgroup)
  if (!grid_ok(blocks) || (a.n_splits > 1 && !grid_ok((rows + 3) / 4))) return KARA_ERR_UNSUPPORTED;
  a.seqs = seqs;
  a.bt = block_table;
  a.seq_lens = seq_lens;
  a.q = q;
  a.rec_o = (float*)workspace;
  a.rec_ml = a.rec_o + rows * a.n_splits * g.d;
  a.out = out;
  hipStream_t s = (hipStream_t)stream;
  hipError_t e = hipSuccess;
  if (few && n_layers <= kFewLayers) {
    WindowCallOf<kFewLayers> c{a, {}, {}, {}, {}};
    set_pools(&c, k_pools, v_pools, k_scales, v_scales);
    e = launch_split(g, q8, tile, c, blocks, s);
  } else {
    WindowCall c{a, {}, {}, {}, {}};
    set_pools(&c, k_pools, v_pools, k_scales, v_scales);
    e = few ? launch_split(g, q8, tile, c, blocks, s) : launch_window_chunk(g, c, plan, q8, workspace, s);
  }
  if (e != hipSuccess || a.n_splits == 1) return hip_status(e);
  const dim3 grid((unsigned)((rows + 3) / 4));
#define KARA_WINDOW_COMBINE(D, B)                                                                               \
  hipLaunchKernelGGL((window_combine_kernel<D, B>), grid, dim3(256), 0, s, (const float*)a.rec_o, (const float*)a.rec_ml, \
                     out, a.n_splits, rows)
  if (g.d == 128) {
    if (f32) KARA_WINDOW_COMBINE(128, false);
    else KARA_WINDOW_COMBINE(128, true);
  } else {
    if (f32) KARA_WINDOW_COMBINE(64, false);
    else KARA_WINDOW_COMBINE(64, true);
  }
#undef KARA_WINDOW_COMBINE
  return hip_status(hipGetLastError());
}

}  // namespace
}  // namespace kara

using namespace kara;

extern "C" {

kara_status_t kara_window_attention_workspace_size(const kara_params_t* p, int32_t n, int32_t n_layers, int32_t n_query,
                                                   int32_t window, int32_t n_sink, int32_t max_len, size_t* bytes) {
  // (for a cache of either kind: over rows of fp32 all queries take the split kernel)
  size_t rows = 0, codes = 0;
  kara_status_t st = workspace_size(p, n, n_layers, n_query, window, n_sink, max_len, false, bytes ? &rows : nullptr);
  if (st == KARA_OK) st = workspace_size(p, n, n_layers, n_query, window, n_sink, max_len, true, &codes);
  if (st == KARA_OK) *bytes = std::max(rows, codes);
  return st;
}

kara_status_t kara_window_attention(const kara_params_t* p, int32_t n, const int32_t* seqs, int32_t n_layers,
                                    int32_t n_query, int32_t window, int32_t n_sink, const void* q,
                                    const void* const* k_pools, const void* const* v_pools, const void* const* k_scales,
                                    const void* const* v_scales, const int32_t* block_table, const int32_t* seq_lens,
                                    int32_t max_len, void* out, void* workspace, size_t workspace_bytes, void* stream) {
  return attend(p, n, seqs, n_layers, n_query, window, n_sink, q, k_pools, v_pools, k_scales, v_scales, block_table,
                seq_lens, max_len, out, workspace, workspace_bytes, stream);
}

kara_status_t kara_q8_attention_workspace_size(const kara_params_t* p, int32_t n, int32_t n_layers, int32_t n_query,
                                               int32_t max_len, size_t* bytes) {
  return workspace_size(p, n, n_layers, n_query, 0, 0, max_len, true, bytes);
}

kara_status_t kara_q8_attention(const kara_params_t* p, int32_t n, const int32_t* seqs, int32_t n_layers,
                                int32_t n_query, const void* q, const void* const* k_pools, const void* const* v_pools,
                                const void* const* k_scales, const void* const* v_scales, const int32_t* block_table,
                                const int32_t* seq_lens, int32_t max_len, void* out, void* workspace,
                                size_t workspace_bytes, void* stream) {
  if (n > 0 && (!k_scales || !v_scales)) return KARA_ERR_INVALID_ARG;
  return attend(p, n, seqs, n_layers, n_query, 0, 0, q, k_pools, v_pools, k_scales, v_scales, block_table, seq_lens,
                max_len, out, workspace, workspace_bytes, stream);
}

}  // extern "C"

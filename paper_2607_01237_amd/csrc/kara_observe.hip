// kara_evict_observe: the softmax weights that many queries give to the cached
// keys, summed per key (include/kara_evict.h).  Two sweeps over q . k, as the
// weights need the rows' sums first: row statistics (each row's maximum and sum of
// exponentials), then column sums with K held and the queries streamed.  No V, no
// atomics: every key's sum is formed by one workgroup, in row order (or in a few parts
// that a last launch adds in order).  Few rows have kernels of their own in either sweep.
//
// Bound by the vector work on the logits, 3 operations and an exponential for each in
// either sweep, beside the matrix products: 2 prompts of 2048 queries over 2048 and
// 4001 tokens, 32/8 heads, d = 128: statistics 104 us, sums 110, 67 GFLOP
// each.
#include <type_traits>

#include "kara_evict.h"
#include "kara_q4_device.h"

namespace kara {
namespace {

constexpr float kLog2e = 1.4426950408889634f;
constexpr float kNegInf = -__builtin_huge_valf();
constexpr float kMaxFloor = -3.402823466e38f;

typedef uint32_t u32x4 __attribute__((ext_vector_type(4)));

// what a stream of rows is made of
enum { kBf16Rows, kF32Rows, kCodeRows };

// Unit and piece of a block, the pieces of all units in turn and the longest first: the
// last ones fill what is left.  Blocks go round the 8 XCDs, and an XCD's round its four
// shader engines.
struct Order {
  // The second half backwards: where all blocks are placed at once, two to a CU, long
  // ones then share a CU with short ones (2 prompts of 2048 queries over 2048 and 4001
  // tokens: 260 -> 200 us).
  int back;
  // Units moved on by `shift` from piece to piece, or from every second one to the next.
  // With eight KV heads a unit's pieces stay on one XCD, whose L2 then holds its rows, and
  // each XCD has heads of every sequence; an even number of sequences is shifted there,
  // or each engine would keep its own (8 prompts: 787 -> 710 us).  With other counts an
  // XCD might get all the pieces of a long sequence.
  uint32_t shift, half;
};
constexpr int kCUs = 256;
Order order_of(const Geom& g, int64_t units, int64_t blocks, bool pairs) {
  const bool back = pairs && blocks <= 2 * kCUs;
  if (g.Hkv % 8 != 0) return {back, 1, 0};
  const int64_t each = units / 8;        // of an XCD
  return {back, back || each % 2 != 0 ? 0u : 8u, each % 4 != 0};
}

struct ObserveArgs {
  Geom g;
  int n, T, n_new, max_len;
  uint32_t units;                       // (layer, sequence, KV head)
  Order order;                          // of the blocks
  int row_blocks, splits, split_keys;   // row statistics (split_keys: column sums of few rows, too)
  int bs_shift;                         // log2(bs) when bs is a power of two, else -1
  int key_blocks, parts, part_rows;     // column sums: the rows of a unit in parts
  const int32_t *seqs, *bt, *seq_lens;
  const void* q;                        // [n_layers][n][T][Hq][d]
  PoolPtrs k, ks;
  float* w[kMaxLayersPerLaunch];
  floatx2* stats;                       // [n_layers][n][Hkv][T * G][splits]: maximum (log2 units), sum
  float* sums;                          // [n_layers][n][Hkv][parts][ld] (parts > 1)
  int64_t ld;
};

// Eight values of a row as loaded, and as NT bf16 terms.
template <int SRC>
struct Octet {
  u32x4 v[SRC == kF32Rows ? 2 : 1];
  __device__ __forceinline__ void load(const void* base, const void* scales, uint64_t row, int o, int D) {
    if constexpr (SRC == kCodeRows) {
      v[0][0] = *(const uint32_t*)((const char*)base + row * (D / 2) + o * 4);
      v[0][1] = *((const uint8_t*)scales + row * (D / kQ4Block) + (o >> 2));
    } else if constexpr (SRC == kF32Rows) {
      const u32x4* p = (const u32x4*)((const char*)base + row * (D * 4) + o * 32);
      v[0] = p[0];
      v[1] = p[1];
    } else {
      v[0] = *(const u32x4*)((const char*)base + row * (D * 2) + o * 16);
    }
  }
  __device__ __forceinline__ void zero() {
#pragma unroll
    for (auto& x : v) x = u32x4{0, 0, 0, 0};
  }
  template <int NT>
  __device__ __forceinline__ void terms(bf16x8 (&t)[NT]) const {
    if constexpr (SRC == kCodeRows) {
      static_assert(NT == 1, "codes are exact in bf16");
      t[0] = q4_octet(v[0][0], q4_scale(v[0][1]));
    } else if constexpr (SRC == kBf16Rows) {
      static_assert(NT == 1, "bf16 rows");
      t[0] = __builtin_bit_cast(bf16x8, v[0]);
    } else {
      uint32_t w[4][NT];
#pragma unroll
      for (int i = 0; i < 4; ++i)
        bf16_term_pairs<true>(__uint_as_float(v[i >> 1][2 * i & 3]), __uint_as_float(v[i >> 1][(2 * i & 3) + 1]), w[i]);
#pragma unroll
      for (int y = 0; y < NT; ++y) t[y] = __builtin_bit_cast(bf16x8, uint4{w[0][y], w[1][y], w[2][y], w[3][y]});
    }
  }
};

// LDS rows of D bf16, 16-byte chunks XOR-swizzled so that 16 rows read at one chunk
// each fall in different banks (the pattern of the recompute attention's keys)
template <int D>
__device__ __forceinline__ int swz(int row) {
  if constexpr (D == 128) return ((row & 3) << 2) | ((row >> 2) & 3);
  return ((row & 3) << 1) | ((row >> 2) & 1);
}

struct Piece {
  uint32_t unit, piece;
};
__device__ __forceinline__ Piece piece_of(uint32_t units, const Order& o) {
  uint32_t block = blockIdx.x;
  if (o.back && block >= kCUs) block = gridDim.x - 1 - (block - kCUs);
  const uint32_t piece = block / units, at = block - piece * units;
  return {o.shift == 0 ? at : (at + o.shift * (piece >> o.half)) % units, piece};
}

constexpr int kObsThreads = 512;
constexpr int kObsWaves = kObsThreads / 64;
constexpr int kChunk = 64;                  // rows staged at a time
constexpr int kMaxSplits = 16;              // of a row's keys, or parts of a key's rows

template <int NT, int D>
struct ChunkLds {
  __attribute__((aligned(16))) char b[2][NT][kChunk * D * 2];
};

// q . k of a 16-row A tile against a 16-row B tile: products of terms i, j with i +
// j below the larger count (fp32 on both sides: 24 of 24 bits)
template <int NA, int NB, int KS>
__device__ __forceinline__ floatx4 dot_tile(const bf16x8 (&a)[NA][KS], const bf16x8 (&b)[NB][KS]) {
  floatx4 acc = {0.f, 0.f, 0.f, 0.f};
  constexpr int most = NA > NB ? NA : NB;
#pragma unroll
  for (int sum = most - 1; sum >= 0; --sum)
#pragma unroll
    for (int i = 0; i < NA; ++i)
#pragma unroll
      for (int j = 0; j < NB; ++j)
        if (i + j == sum)
#pragma unroll
          for (int x = 0; x < KS; ++x) acc = __builtin_amdgcn_mfma_f32_16x16x32_bf16(a[i][x], b[j][x], acc, 0, 0, 0);
  return acc;
}

template <int NT, int D>
__device__ __forceinline__ void read_tile(const char (&b)[NT][kChunk * D * 2], int row0, int gq, int li,
                                          bf16x8 (&t)[NT][D / 32]) {
#pragma unroll
  for (int y = 0; y < NT; ++y)
#pragma unroll
    for (int x = 0; x < D / 32; ++x)
      __builtin_memcpy(&t[y][x], &b[y][(row0 + li) * D * 2 + (((gq * (D / 32) + x) ^ swz<D>(li)) * 16)], 16);
}

// Unit and sequence of a workgroup; false: nothing to do there.
struct Unit {
  int l, j, h, s, len;
};
__device__ __forceinline__ bool unit_of(const ObserveArgs& a, uint32_t u, Unit* x) {
  const Geom& g = a.g;
  x->h = u % (uint32_t)g.Hkv;
  u /= (uint32_t)g.Hkv;
  x->j = u % (uint32_t)a.n;
  x->l = u / (uint32_t)a.n;
  x->s = a.seqs[x->j];
  x->len = x->s >= 0 && x->s < g.n_seqs ? a.seq_lens[x->s] : 0;
  return x->len > 0 && x->len <= a.max_len;
}

__device__ __forceinline__ uint64_t key_row(const Geom& g, const int32_t* row_pages, int h, int pos) {
  const int b = pos / g.bs;
  const int page = min(max(row_pages[b], 0), g.num_pages - 1);
  return (uint64_t)(((int64_t)page * g.Hkv + h) * g.bs + (pos - b * g.bs));
}

// A lane's maximum and sum of its rows, over the logits of two 16-key tiles.  The
// reference is raised only where a logit passes it by more than 2^8.
template <int QT>
__device__ __forceinline__ void add_logits(const floatx4 (&sv)[2][QT], float c, float (&m)[QT], float (&sum)[QT]) {
  float over = kNegInf, mx[QT];
#pragma unroll
  for (int t = 0; t < QT; ++t) {
    mx[t] = sv[0][t][0];
#pragma unroll
    for (int y = 0; y < 2; ++y)
#pragma unroll
      for (int r = 0; r < 4; ++r) mx[t] = fmaxf(mx[t], sv[y][t][r]);
    over = fmaxf(over, fmaf(mx[t], c, -m[t]));
  }
  if (__ballot(over > 8.f) != 0ull) {
#pragma unroll
    for (int t = 0; t < QT; ++t) {
      const float mn = fmaxf(m[t], mx[t] * c);
      sum[t] *= __builtin_amdgcn_exp2f(m[t] - mn);
      m[t] = mn;
    }
  }
#pragma unroll
  for (int t = 0; t < QT; ++t)
#pragma unroll
    for (int y = 0; y < 2; ++y) {
      const float e0 = __builtin_amdgcn_exp2f(fmaf(sv[y][t][0], c, -m[t])), e1 = __builtin_amdgcn_exp2f(fmaf(sv[y][t][1], c, -m[t]));
      const float e2 = __builtin_amdgcn_exp2f(fmaf(sv[y][t][2], c, -m[t])), e3 = __builtin_amdgcn_exp2f(fmaf(sv[y][t][3], c, -m[t]));
      sum[t] += (e0 + e1) + (e2 + e3);
    }
}

// ---- row statistics: one workgroup per (unit, 128 QT query rows, split of the
// keys); a wave holds 16 QT rows, the keys pass through LDS 64 at a time.  A lane
// keeps a maximum and a sum of its own -- of the keys 4gq + r -- and the four of a
// row meet at the end.
template <int KSRC, int NK, int QSRC, int NQ, int D, int QT>
__global__ __launch_bounds__(kObsThreads, NK * NQ == 1 ? 4 : 2) void observe_stats_kernel(ObserveArgs a) {
  constexpr int KS = D / 32, kOct = D / 8, kPer = kChunk * kOct / kObsThreads;
  __shared__ ChunkLds<NK, D> lds;
  const Geom& g = a.g;
  const int tid = threadIdx.x, lane = tid & 63;
  const int wave = __builtin_amdgcn_readfirstlane(tid >> 6);
  const int gq = lane >> 4, li = lane & 15;
  const Piece pc = piece_of(a.units, a.order);
  const uint32_t u = pc.unit;
  const int split = pc.piece % (uint32_t)a.splits;
  const int rb = a.row_blocks - 1 - (int)(pc.piece / (uint32_t)a.splits);     // rows that see most keys first
  Unit x;
  if (!unit_of(a, u, &x)) return;
  const int G = g.G, R = G * a.T;
  const int row0 = rb * kObsWaves * 16 * QT;
  const int first = x.len - a.T;                       // position of query 0
  const int last_pos = first + (min(row0 + kObsWaves * 16 * QT, R) - 1) / G;
  const int k_lo = split * a.split_keys;
  const int k_hi = min(min(x.len, last_pos + 1), k_lo + a.split_keys);
  const int32_t* row_pages = a.bt + (int64_t)x.s * g.max_blocks;
  const int wrow0 = row0 + wave * 16 * QT;
  const int wfirst = first + min(wrow0, R - 1) / G, wlast = wrow0 < R ? first + min(wrow0 + 16 * QT - 1, R - 1) / G : -1;

  bf16x8 qa[QT][NQ][KS];
  int qpos[QT];
#pragma unroll
  for (int t = 0; t < QT; ++t) {
    const int r = min(wrow0 + t * 16 + li, R - 1);
    const int qt = r / G;
    qpos[t] = first + qt;
    const uint64_t row = (((uint64_t)x.l * a.n + x.j) * a.T + qt) * g.Hq + x.h * G + (r - qt * G);
#pragma unroll
    for (int y = 0; y < KS; ++y) {
      Octet<QSRC> o;
      o.load(a.q, nullptr, row, gq * KS + y, D);
      bf16x8 tt[NQ];
      o.terms(tt);
#pragma unroll
      for (int z = 0; z < NQ; ++z) qa[t][z][y] = tt[z];
    }
  }
  float m[QT], sum[QT];
#pragma unroll
  for (int t = 0; t < QT; ++t) m[t] = kMaxFloor, sum[t] = 0.f;
  const float c = g.scale * kLog2e;

  // A thread's kPer octets are one column of rows kObsThreads / kOct apart.  Their
  // pages are read a chunk before the octets.  (Past the end: the last key, masked.)
  const int srow = tid / kOct, soct = tid % kOct;
  Octet<KSRC> pre[kPer];
  int page[kPer], slot[kPer];
  auto look = [&](int k0) __attribute__((always_inline)) {
#pragma unroll
    for (int i = 0; i < kPer; ++i) {
      const int pos = min(k0 + srow + i * (kObsThreads / kOct), k_hi - 1);
      const int b = a.bs_shift >= 0 ? pos >> a.bs_shift : pos / g.bs;
      slot[i] = pos - b * g.bs;
      page[i] = row_pages[b];
    }
  };
  // (a pool has fewer than 2^32 rows)
  const void *const kbase = a.k.p[x.l], *const sbase = a.ks.p[x.l];
  const uint32_t page_rows = (uint32_t)g.Hkv * g.bs, head_row = (uint32_t)x.h * g.bs;
  auto fetch = [&]() __attribute__((always_inline)) {
#pragma unroll
    for (int i = 0; i < kPer; ++i) {
      const uint32_t p = min(max(page[i], 0), g.num_pages - 1);
      pre[i].load(kbase, sbase, p * page_rows + (head_row + slot[i]), soct, D);
    }
  };
  // two 16-key tiles against the wave's rows
  auto tiles = [&](const char (&b)[NK][kChunk * D * 2], int kt, int k0, auto masked) __attribute__((always_inline)) {
    floatx4 sv[2][QT];
#pragma unroll
    for (int y = 0; y < 2; ++y) {
      bf16x8 ka[NK][KS];
      read_tile<NK, D>(b, (kt + y) * 16, gq, li, ka);
#pragma unroll
      for (int t = 0; t < QT; ++t) sv[y][t] = dot_tile<NK, NQ, KS>(ka, qa[t]);
    }
    if constexpr (decltype(masked)::value) {
#pragma unroll
      for (int t = 0; t < QT; ++t) {
        const int sees = min(k_hi, qpos[t] + 1) - (k0 + kt * 16 + 4 * gq);
#pragma unroll
        for (int y = 0; y < 2; ++y)
#pragma unroll
          for (int r = 0; r < 4; ++r)
            if (y * 16 + r >= sees) sv[y][t][r] = kNegInf;
      }
    }
    add_logits(sv, c, m, sum);
  };
  if (k_lo < k_hi) {
    look(k_lo);
    fetch();
    look(k_lo + kChunk);
    int buf = 0;
    for (int k0 = k_lo; k0 < k_hi; k0 += kChunk, buf ^= 1) {
#pragma unroll
      for (int i = 0; i < kPer; ++i) {
        const int row = srow + i * (kObsThreads / kOct);
        bf16x8 t[NK];
        pre[i].terms(t);
#pragma unroll
        for (int y = 0; y < NK; ++y)
          __builtin_memcpy(&lds.b[buf][y][row * D * 2 + ((soct ^ swz<D>(row & 15)) * 16)], &t[y], 16);
      }
      if (k0 + kChunk < k_hi) {
        fetch();
        look(k0 + 2 * kChunk);
      }
      __syncthreads();
      if (k0 > wlast) continue;
      if (k0 + kChunk > min(k_hi, wfirst + 1)) {
#pragma unroll 1
        for (int kt = 0; kt < 4; kt += 2) tiles(lds.b[buf], kt, k0, std::true_type{});
      } else {
#pragma unroll 1
        for (int kt = 0; kt < 4; kt += 2) tiles(lds.b[buf], kt, k0, std::false_type{});
      }
    }
  }
#pragma unroll
  for (int t = 0; t < QT; ++t) {
    float M = fmaxf(m[t], __shfl_xor(m[t], 16, 64));
    M = fmaxf(M, __shfl_xor(M, 32, 64));
    float L = sum[t] * __builtin_amdgcn_exp2f(m[t] - M);
    L += __shfl_xor(L, 16, 64);
    L += __shfl_xor(L, 32, 64);
    const int r = wrow0 + t * 16 + li;
    if (gq == 0 && r < R) a.stats[((int64_t)u * R + r) * a.splits + split] = floatx2{M, L};
  }
}

// The same for few query rows: a workgroup of four waves per (unit, 32 rows, split of the
// keys).  The waves take 32 keys each in turn, straight from the pages to registers, the
// next ones on their way, without barriers: staged, most waves would have no rows.
constexpr int kFewThreads = 256;
constexpr int kFewWaves = kFewThreads / 64;
constexpr int kFewRows = 32;                // of a workgroup

// a lane's part of 16 keys as loaded: values gq * D / 4 .. of key li
template <int KSRC, int D>
struct KeyPart {
  static constexpr int KS = D / 32;
  uint32_t v[KSRC == kCodeRows ? KS + 1 : 4 * KS];
  __device__ __forceinline__ void load(const void* base, const void* scales, uint64_t row, int gq) {
    if constexpr (KSRC == kCodeRows) {
      __builtin_memcpy(v, (const char*)base + row * (D / 2) + gq * (D / 8), D / 8);
      v[KS] = ((const uint8_t*)scales)[row * (D / kQ4Block) + gq * KS / 4];
    } else {
      __builtin_memcpy(v, (const char*)base + row * (D * 2) + gq * (D / 2), D / 2);
    }
  }
  __device__ __forceinline__ void operand(bf16x8 (&t)[1][KS]) const {
    if constexpr (KSRC == kCodeRows) {
      const float scale = q4_scale(v[KS]);
#pragma unroll
      for (int x = 0; x < KS; ++x) t[0][x] = q4_octet(v[x], scale);
    } else {
      __builtin_memcpy(t, v, sizeof(v));
    }
  }
};

template <int KSRC, int QSRC, int NQ, int D>
__global__ __launch_bounds__(kFewThreads, 2) void observe_few_kernel(ObserveArgs a) {
  constexpr int KS = D / 32, QT = kFewRows / 16;
  __shared__ floatx2 part[kFewWaves][kFewRows];
  const Geom& g = a.g;
  const int tid = threadIdx.x, lane = tid & 63;
  const int wave = __builtin_amdgcn_readfirstlane(tid >> 6);
  const int gq = lane >> 4, li = lane & 15;
  const Piece pc = piece_of(a.units, a.order);
  const uint32_t u = pc.unit;
  const int split = pc.piece / (uint32_t)a.row_blocks;
  const int row0 = (a.row_blocks - 1 - (int)(pc.piece % (uint32_t)a.row_blocks)) * kFewRows;
  Unit x;
  if (!unit_of(a, u, &x)) return;
  const int G = g.G, R = G * a.T;
  const int first = x.len - a.T;                       // position of query 0
  const int first_pos = first + row0 / G, last_pos = first + (min(row0 + kFewRows, R) - 1) / G;
  const int k_lo = split * a.split_keys;
  const int k_hi = min(min(x.len, last_pos + 1), k_lo + a.split_keys);
  const int32_t* row_pages = a.bt + (int64_t)x.s * g.max_blocks;

  // this wave's keys k0 .. k0 + 31 (past the end: the last key, masked), their pages
  // looked up a step before they are read
  const void *const kbase = a.k.p[x.l], *const sbase = a.ks.p[x.l];
  const uint32_t page_rows = (uint32_t)g.Hkv * g.bs, head_row = (uint32_t)x.h * g.bs;
  int page[2], slot[2];
  auto look = [&](int k0) __attribute__((always_inline)) {
#pragma unroll
    for (int y = 0; y < 2; ++y) {
      const int pos = min(k0 + y * 16 + li, k_hi - 1);
      const int b = a.bs_shift >= 0 ? pos >> a.bs_shift : pos / g.bs;
      slot[y] = pos - b * g.bs;
      page[y] = row_pages[b];
    }
  };
  KeyPart<KSRC, D> keys[2];
  auto fetch = [&]() __attribute__((always_inline)) {
#pragma unroll
    for (int y = 0; y < 2; ++y) {
      const uint32_t p = min(max(page[y], 0), g.num_pages - 1);
      keys[y].load(kbase, sbase, p * page_rows + (head_row + slot[y]), gq);
    }
  };
  constexpr int kStep = kFewWaves * 32;
  const int k_wave = k_lo + wave * 32;
  if (k_wave < k_hi) look(k_wave);

  bf16x8 qa[QT][NQ][KS];
  int qpos[QT];
#pragma unroll
  for (int t = 0; t < QT; ++t) {
    const int r = min(row0 + t * 16 + li, R - 1);
    const int qt = r / G;
    qpos[t] = first + qt;
    const uint64_t row = (((uint64_t)x.l * a.n + x.j) * a.T + qt) * g.Hq + x.h * G + (r - qt * G);
#pragma unroll
    for (int y = 0; y < KS; ++y) {
      Octet<QSRC> o;
      o.load(a.q, nullptr, row, gq * KS + y, D);
      bf16x8 tt[NQ];
      o.terms(tt);
#pragma unroll
      for (int z = 0; z < NQ; ++z) qa[t][z][y] = tt[z];
    }
  }
  float m[QT], sum[QT];
#pragma unroll
  for (int t = 0; t < QT; ++t) m[t] = kMaxFloor, sum[t] = 0.f;
  const float c = g.scale * kLog2e;
  if (k_wave < k_hi) {
    fetch();
    look(k_wave + kStep);
    for (int k0 = k_wave; k0 < k_hi; k0 += kStep) {
      bf16x8 ka[2][1][KS];
#pragma unroll
      for (int y = 0; y < 2; ++y) keys[y].operand(ka[y]);
      if (k0 + kStep < k_hi) {
        fetch();
        look(k0 + 2 * kStep);
      }
      floatx4 sv[2][QT];
#pragma unroll
      for (int y = 0; y < 2; ++y)
#pragma unroll
        for (int t = 0; t < QT; ++t) sv[y][t] = dot_tile<1, NQ, KS>(ka[y], qa[t]);
      // (wait states before the products' results are read past the branch)
#pragma unroll
      for (int t = 0; t < QT; ++t) asm volatile("s_nop 7\n\ts_nop 3" : "+v"(sv[0][t]), "+v"(sv[1][t]));
      if (k0 + 32 > min(k_hi, first_pos + 1)) {
#pragma unroll
        for (int t = 0; t < QT; ++t) {
          const int sees = min(k_hi, qpos[t] + 1) - (k0 + 4 * gq);
#pragma unroll
          for (int y = 0; y < 2; ++y)
#pragma unroll
            for (int r = 0; r < 4; ++r)
              if (y * 16 + r >= sees) sv[y][t][r] = kNegInf;
        }
      }
      add_logits(sv, c, m, sum);
    }
  }
#pragma unroll
  for (int t = 0; t < QT; ++t) {
    float M = fmaxf(m[t], __shfl_xor(m[t], 16, 64));
    M = fmaxf(M, __shfl_xor(M, 32, 64));
    float L = sum[t] * __builtin_amdgcn_exp2f(m[t] - M);
    L += __shfl_xor(L, 16, 64);
    L += __shfl_xor(L, 32, 64);
    if (gq == 0) part[wave][t * 16 + li] = floatx2{M, L};
  }
  __syncthreads();
  if (tid < kFewRows && row0 + tid < R) {
    float M = kMaxFloor, L = 0.f;
#pragma unroll
    for (int w = 0; w < kFewWaves; ++w) M = fmaxf(M, part[w][tid][0]);
#pragma unroll
    for (int w = 0; w < kFewWaves; ++w) L += part[w][tid][1] * __builtin_amdgcn_exp2f(part[w][tid][0] - M);
    a.stats[((int64_t)u * R + row0 + tid) * a.splits + split] = floatx2{M, L};
  }
}

// A row's maximum and sum from its splits'.
__device__ __forceinline__ floatx2 join_splits(const floatx2* st, int splits) {
  float M = kMaxFloor, L = 0.f;
#pragma unroll 4
  for (int i = 0; i < splits; ++i) M = fmaxf(M, st[i][0]);
#pragma unroll 4
  for (int i = 0; i < splits; ++i) L += st[i][1] * __builtin_amdgcn_exp2f(st[i][0] - M);
  return floatx2{M, L};
}

// A row's splits joined into the first: a thread per row.  (Few rows are joined by the
// workgroups that read them.)
__global__ __launch_bounds__(256) void observe_join_kernel(floatx2* stats, int splits, int64_t rows) {
  const int64_t r = (int64_t)blockIdx.x * 256 + threadIdx.x;
  if (r >= rows) return;
  stats[r * splits] = join_splits(stats + r * splits, splits);
}

// The 16 lanes of a row of the wave hold parts of the same 8 sums: reduced and dealt out,
// lanes li and li ^ 1 end with sum (t, r) = (li >> 3, (li >> 1) & 3).
__device__ __forceinline__ float deal_sums(const floatx4 (&acc)[2], int li) {
  auto half = [&](float lo, float hi, int bit) __attribute__((always_inline)) {
    const bool up = li & bit;
    return (up ? hi : lo) + __shfl_xor(up ? lo : hi, bit, 64);
  };
  const float a0 = half(acc[0][0], acc[1][0], 8), a1 = half(acc[0][1], acc[1][1], 8);
  const float a2 = half(acc[0][2], acc[1][2], 8), a3 = half(acc[0][3], acc[1][3], 8);
  const float v = half(half(a0, a2, 4), half(a1, a3, 4), 2);
  return v + __shfl_xor(v, 1, 64);
}

// ---- column sums: one workgroup per (unit, 128 KT keys, part of the rows); a wave
// holds 16 KT keys, the query rows that see them pass through LDS 64 at a time with
// their maxima and reciprocal sums.
template <int KSRC, int NK, int QSRC, int NQ, int D, int KT>
__global__ __launch_bounds__(kObsThreads, NK * NQ == 1 ? 4 : 2) void observe_sum_kernel(ObserveArgs a) {
  constexpr int KS = D / 32, kOct = D / 8, kPer = kChunk * kOct / kObsThreads;
  __shared__ ChunkLds<NQ, D> lds;
  __shared__ floatx2 row_stat[2][kChunk];              // maximum and reciprocal sum
  const Geom& g = a.g;
  const int tid = threadIdx.x, lane = tid & 63;
  const int wave = __builtin_amdgcn_readfirstlane(tid >> 6);
  const int gq = lane >> 4, li = lane & 15;
  const Piece pc = piece_of(a.units, a.order);
  const uint32_t u = pc.unit;
  const int part = a.parts - 1 - (int)(pc.piece % (uint32_t)a.parts);
  const int kb = pc.piece / (uint32_t)a.parts;         // the first keys are seen by most rows
  Unit x;
  if (!unit_of(a, u, &x)) return;
  const int key0 = kb * kObsWaves * 16 * KT;
  if (key0 >= x.len) return;
  if (a.parts == 1) {
    int dup = 0;
    for (int o = tid; o < x.j; o += kObsThreads) dup |= a.seqs[o] == x.s;
    if (__syncthreads_or(dup)) return;                 // an earlier listing counts
  }
  const int G = g.G, R = G * a.T;
  const int first = x.len - a.T;
  const int32_t* row_pages = a.bt + (int64_t)x.s * g.max_blocks;
  const int wkey0 = key0 + wave * 16 * KT;

  bf16x8 ka[KT][NK][KS];
#pragma unroll
  for (int t = 0; t < KT; ++t) {
    const uint64_t row = key_row(g, row_pages, x.h, min(wkey0 + t * 16 + li, x.len - 1));
#pragma unroll
    for (int y = 0; y < KS; ++y) {
      Octet<KSRC> o;
      o.load(a.k.p[x.l], a.ks.p[x.l], row, gq * KS + y, D);
      bf16x8 tt[NK];
      o.terms(tt);
#pragma unroll
      for (int z = 0; z < NK; ++z) ka[t][z][y] = tt[z];
    }
  }
  floatx4 acc[KT];
#pragma unroll
  for (int t = 0; t < KT; ++t) acc[t] = floatx4{0.f, 0.f, 0.f, 0.f};
  const float c = g.scale * kLog2e;
  // the part's rows that see this workgroup's first key
  const int r_lo = max(max(0, key0 - first) * G, part * a.part_rows);
  const int r_hi = min(R, (part + 1) * a.part_rows);

  // A thread's octets are one column of rows kObsThreads / kOct apart; their queries
  // are stepped from chunk to chunk, without a division.
  const int srow = tid / kOct, soct = tid % kOct;
  Octet<QSRC> pre[kPer];
  floatx2 st = {0.f, 1.f};
  uint32_t qrow[kPer];                                 // row of q, and head in group, of the next chunk's rows
  int qg[kPer];
  const int step_g = kChunk % G, step = kChunk / G * g.Hq + step_g;
#pragma unroll
  for (int i = 0; i < kPer; ++i) {
    const int r = r_lo + srow + i * (kObsThreads / kOct);
    qg[i] = r % G;
    qrow[i] = (uint32_t)(r / G) * g.Hq + qg[i];
  }
  const char* const qbase = (const char*)a.q + (((uint64_t)x.l * a.n + x.j) * a.T * g.Hq + x.h * G) * (D * (QSRC == kF32Rows ? 4 : 2));
  const floatx2* const ustats = a.stats + (int64_t)u * R * a.splits;
  auto fetch = [&](int r0) __attribute__((always_inline)) {
#pragma unroll
    for (int i = 0; i < kPer; ++i) {
      pre[i].zero();
      if (r0 + srow + i * (kObsThreads / kOct) < r_hi)
        pre[i].load(qbase, nullptr, qrow[i], soct, D);
      qrow[i] += step;
      qg[i] += step_g;
      if (qg[i] >= G) qg[i] -= G, qrow[i] += g.Hq - G;
    }
    if (tid < kChunk && r0 + tid < r_hi) st = ustats[(int64_t)(r0 + tid) * a.splits];
  };
  // one 16-row tile against the wave's keys
  auto tile = [&](int buf, int rt, int r0, auto masked) __attribute__((always_inline)) {
    bf16x8 qb[NQ][KS];
    read_tile<NQ, D>(lds.b[buf], rt * 16, gq, li, qb);
    const floatx2 stat = row_stat[buf][rt * 16 + li];
    const float rm = stat[0], ri = stat[1];
    floatx4 sv[KT];
#pragma unroll
    for (int t = 0; t < KT; ++t) sv[t] = dot_tile<NK, NQ, KS>(ka[t], qb);
    // (past the last row: sees none)
    const int pos = !decltype(masked)::value ? 0 : r0 + rt * 16 + li < r_hi ? first + (r0 + rt * 16 + li) / G : -1;
#pragma unroll
    for (int t = 0; t < KT; ++t)
#pragma unroll
      for (int r = 0; r < 4; ++r) {
        const float p = __builtin_amdgcn_exp2f(fmaf(sv[t][r], c, -rm));
        // (dropped, not multiplied by 0: against the maximum of a row that sees no key it may be infinite)
        if constexpr (decltype(masked)::value) acc[t][r] += wkey0 + t * 16 + 4 * gq + r > pos ? 0.f : p * ri;
        else acc[t][r] = fmaf(p, ri, acc[t][r]);
      }
  };
  if (r_lo < r_hi) {
    fetch(r_lo);
    int buf = 0;
    for (int r0 = r_lo; r0 < r_hi; r0 += kChunk, buf ^= 1) {
#pragma unroll
      for (int i = 0; i < kPer; ++i) {
        const int row = srow + i * (kObsThreads / kOct);
        bf16x8 t[NQ];
        pre[i].terms(t);
#pragma unroll
        for (int y = 0; y < NQ; ++y)
          __builtin_memcpy(&lds.b[buf][y][row * D * 2 + ((soct ^ swz<D>(row & 15)) * 16)], &t[y], 16);
      }
      // (a sum of 0: every logit of the row is -inf, or it sees no key)
      if (tid < kChunk) row_stat[buf][tid] = floatx2{st[0], st[1] == 0.f ? 0.f : 1.f / st[1]};
      if (r0 + kChunk < r_hi) fetch(r0 + kChunk);
      __syncthreads();
      if (wkey0 >= x.len || first + (min(r0 + kChunk, r_hi) - 1) / G < wkey0) continue;     // (uniform in the wave)
      if (r0 + kChunk > r_hi || first + r0 / G < wkey0 + 16 * KT - 1) {
#pragma unroll 1
        for (int rt = 0; rt < 4; ++rt) tile(buf, rt, r0, std::true_type{});
      } else {
#pragma unroll 2
        for (int rt = 0; rt < 4; ++rt) tile(buf, rt, r0, std::false_type{});
      }
    }
  }
  static_assert(KT == 2, "eight sums to sixteen lanes");
  const float v = deal_sums(acc, li);
  const int pos = wkey0 + (li >> 3) * 16 + 4 * gq + ((li >> 1) & 3);
  if ((li & 1) || pos >= x.len) return;
  if (a.parts > 1) {
    a.sums[((int64_t)u * a.parts + part) * a.ld + pos] = v;
    return;
  }
  const int b = pos / g.bs, page = row_pages[b];
  if (page < 0 || page >= g.num_pages) return;
  float* to = a.w[x.l] + ((int64_t)page * g.Hkv + x.h) * g.bs + (pos - b * g.bs);
  *to = pos >= x.len - a.n_new ? v : *to + v;
}

// The same for few query rows, all in LDS with their statistics: a workgroup of four
// waves per (unit, split_keys keys), the waves taking 32 keys each in turn as in
// observe_few_kernel, without the prologue that a workgroup of observe_sum_kernel has for
// each 256 keys (45 sequences of 2.6-3.8K tokens, 32/8 heads, codes, 28 rows: 96 -> 68 us a
// call, 128 rows 152 -> 148, fp32 with 64 rows 203 -> 154).
template <int KSRC, int QSRC, int NQ, int D>
__global__ __launch_bounds__(kFewThreads, 2) void observe_few_sum_kernel(ObserveArgs a) {
  constexpr int KS = D / 32, kOct = D / 8, kMost = (NQ == 1 ? 4 : 2) * kFewRows;
  __shared__ __attribute__((aligned(16))) char rows[NQ][kMost * D * 2];
  __shared__ floatx2 row_stat[kMost];                  // maximum and reciprocal sum
  const Geom& g = a.g;
  const int tid = threadIdx.x, lane = tid & 63;
  const int wave = __builtin_amdgcn_readfirstlane(tid >> 6);
  const int gq = lane >> 4, li = lane & 15;
  const Piece pc = piece_of(a.units, a.order);
  const uint32_t u = pc.unit;
  Unit x;
  if (!unit_of(a, u, &x)) return;
  const int k_lo = pc.piece * a.split_keys, k_hi = min(x.len, k_lo + a.split_keys);
  if (k_lo >= k_hi) return;
  const int G = g.G, R = G * a.T, R16 = (R + 15) & ~15;
  const int first = x.len - a.T;                       // position of query 0
  const int32_t* row_pages = a.bt + (int64_t)x.s * g.max_blocks;
  const void *const kbase = a.k.p[x.l], *const sbase = a.ks.p[x.l];
  float* const wbase = a.w[x.l];
  const uint32_t page_rows = (uint32_t)g.Hkv * g.bs, head_row = (uint32_t)x.h * g.bs;

  // A wave's keys k0 .. k0 + 31 (past the end: the last one, dropped), and the
  // accumulator that a lane writes, that of key (li >> 3) * 16 + 4 gq + ((li >> 1) & 3); pages are
  // looked up a step before.
  const int mine = (li >> 3) * 16 + 4 * gq + ((li >> 1) & 3);
  int page[3], slot[3];
  auto look = [&](int k0) __attribute__((always_inline)) {
#pragma unroll
    for (int y = 0; y < 3; ++y) {
      const int pos = min(k0 + (y < 2 ? y * 16 + li : mine), k_hi - 1);
      const int b = a.bs_shift >= 0 ? pos >> a.bs_shift : pos / g.bs;
      slot[y] = pos - b * g.bs;
      page[y] = row_pages[b];
    }
  };
  KeyPart<KSRC, D> keys[2];
  float was = 0.f;
  float* to = nullptr;
  auto fetch = [&]() __attribute__((always_inline)) {
#pragma unroll
    for (int y = 0; y < 2; ++y) {
      const uint32_t p = min(max(page[y], 0), g.num_pages - 1);
      keys[y].load(kbase, sbase, p * page_rows + (head_row + slot[y]), gq);
    }
    const bool mapped = page[2] >= 0 && page[2] < g.num_pages;
    to = mapped ? wbase + (uint64_t)((uint32_t)page[2] * page_rows + (head_row + slot[2])) : nullptr;
    was = mapped ? *to : 0.f;
  };
  constexpr int kStep = kFewWaves * 32;
  const int k_wave = k_lo + wave * 32;
  if (k_wave < k_hi) look(k_wave);
  int dup = 0;
  for (int o = tid; o < x.j; o += kFewThreads) dup |= a.seqs[o] == x.s;

  const uint64_t qrow0 = ((uint64_t)x.l * a.n + x.j) * a.T * g.Hq + x.h * G;
  for (int i = tid; i < R16 * kOct; i += kFewThreads) {
    const int row = i / kOct, o = i % kOct, t = row / G;
    Octet<QSRC> v;
    v.zero();
    if (row < R) v.load(a.q, nullptr, qrow0 + (uint64_t)t * g.Hq + (row - t * G), o, D);
    bf16x8 tt[NQ];
    v.terms(tt);
#pragma unroll
    for (int y = 0; y < NQ; ++y)
      __builtin_memcpy(&rows[y][row * D * 2 + ((o ^ swz<D>(row & 15)) * 16)], &tt[y], 16);
  }
  if (tid < R) {
    const floatx2 st = join_splits(a.stats + ((int64_t)u * R + tid) * a.splits, a.splits);
    row_stat[tid] = floatx2{st[0], st[1] == 0.f ? 0.f : 1.f / st[1]};   // (0: as in observe_sum_kernel)
  }
  if (__syncthreads_or(dup)) return;                   // an earlier listing counts
  const float c = g.scale * kLog2e;
  if (k_wave >= k_hi) return;
  fetch();
  look(k_wave + kStep);
  for (int k0 = k_wave; k0 < k_hi; k0 += kStep) {
    bf16x8 ka[2][1][KS];
#pragma unroll
    for (int y = 0; y < 2; ++y) keys[y].operand(ka[y]);
    float* const at = to;
    const float old = was;
    if (k0 + kStep < k_hi) {
      fetch();
      look(k0 + 2 * kStep);
    }
    floatx4 acc[2] = {{0.f, 0.f, 0.f, 0.f}, {0.f, 0.f, 0.f, 0.f}};
    // rows from the first that sees key k0, in tiles of 16
    const int r_lo = max(0, k0 - first) * G & ~15;
    for (int r0 = r_lo; r0 < R16; r0 += 16) {
      bf16x8 qb[NQ][KS];
#pragma unroll
      for (int y = 0; y < NQ; ++y)
#pragma unroll
        for (int z = 0; z < KS; ++z)
          __builtin_memcpy(&qb[y][z], &rows[y][(r0 + li) * D * 2 + (((gq * KS + z) ^ swz<D>(li)) * 16)], 16);
      const int r = r0 + li;
      const floatx2 stat = row_stat[min(r, R - 1)];
      floatx4 sv[2];
#pragma unroll
      for (int y = 0; y < 2; ++y) sv[y] = dot_tile<1, NQ, KS>(ka[y], qb);
      // the last key that the row sees (weights past it are dropped, not multiplied by 0:
      // against the maximum of a row that sees no key they may be infinite)
      const int sees = r < R ? first + r / G - k0 : -1;
#pragma unroll
      for (int y = 0; y < 2; ++y)
#pragma unroll
        for (int e = 0; e < 4; ++e) {
          const float p = __builtin_amdgcn_exp2f(fmaf(sv[y][e], c, -stat[0]));
          acc[y][e] += y * 16 + 4 * gq + e > sees ? 0.f : p * stat[1];
        }
    }
    const float v = deal_sums(acc, li);
    const int pos = k0 + mine;
    if (!(li & 1) && pos < k_hi && at) *at = pos >= x.len - a.n_new ? v : old + v;
  }
}

// The parts' sums, in order, to the accumulators: one workgroup per (unit, 256 keys).
__global__ __launch_bounds__(256) void observe_add_kernel(ObserveArgs a, int blocks) {
  const Geom& g = a.g;
  const uint32_t u = blockIdx.x / (uint32_t)blocks;
  const int pos = (int)(blockIdx.x % (uint32_t)blocks) * 256 + threadIdx.x;
  Unit x;
  if (!unit_of(a, u, &x)) return;
  int dup = 0;
  for (int o = threadIdx.x; o < x.j; o += 256) dup |= a.seqs[o] == x.s;
  if (__syncthreads_or(dup) || pos >= x.len) return;     // an earlier listing counts
  float v = 0.f;
  for (int i = 0; i < a.parts; ++i) v += a.sums[((int64_t)u * a.parts + i) * a.ld + pos];
  const int b = pos / g.bs, page = a.bt[(int64_t)x.s * g.max_blocks + b];
  if (page < 0 || page >= g.num_pages) return;
  float* to = a.w[x.l] + ((int64_t)page * g.Hkv + x.h) * g.bs + (pos - b * g.bs);
  *to = pos >= x.len - a.n_new ? v : *to + v;
}

// a grid of one dimension, of 256 threads a block: HIP counts its threads in 32 bits
bool grid_ok(int64_t blocks) { return blocks > 0 && blocks < ((int64_t)1 << 24); }

// 16-row tiles of a wave's rows, and of its keys (four of them, with 168 registers
// and three waves per SIMD, took 17 % longer: 2 prompts of 2048 queries).
constexpr int kHeld = 2;
constexpr int kHeldWg = kObsWaves * 16 * kHeld;         // of a workgroup

// Launches with fewer workgroups than this split: the row statistics their keys (512
// a split at least), the column sums their rows (256 a part at least).
constexpr int kObsWgs = 512;
// Few rows a unit: as long as it pays to read the keys once for 32 rows.  45 sequences of
// 2.6-3.8K tokens, 32/8 heads, whole calls: codes, 28 rows 148 -> 68 us, 128 rows 172 ->
// 148 (their statistics over 160 tokens, where the four waves have little to share, 61
// against 68); fp32 queries 279 -> 97, 64 rows 280 -> 154; bf16 rows, 32 rows 169 -> 129,
// but 64 rows' statistics 171 against 184.
bool few_rows(const Geom& g, int64_t R, int max_len, bool codes) {
  if (!codes) return g.dtype == KARA_BF16 && R <= kFewRows;
  return R <= (g.dtype == KARA_BF16 && max_len > 1024 ? 4 * kFewRows : 2 * kFewRows);
}
constexpr int kFewWgs = 2048;
static_assert(kFewWgs * kFewRows <= kObsWgs * kHeldWg, "their records fit");

struct Plan {
  int row_blocks, splits, split_keys, key_blocks, parts, part_rows, few_keys;
  int64_t units, ld;
  bool few;
  size_t stats_bytes, bytes;
};

Plan plan_of(const Geom& g, int n, int n_layers, int T, int max_len, bool codes) {
  Plan x{};
  x.units = (int64_t)n_layers * n * g.Hkv;
  const int64_t R = (int64_t)g.G * T;
  x.few = few_rows(g, R, max_len, codes);
  const int row_wg = x.few ? kFewRows : kHeldWg;
  x.row_blocks = (int)((R + row_wg - 1) / row_wg);
  x.splits = 1;
  while (x.splits < kMaxSplits && x.units * x.row_blocks * x.splits < (x.few ? kFewWgs : kObsWgs) && max_len > x.splits * 2 * 512)
    x.splits *= 2;
  x.split_keys = ((max_len + x.splits - 1) / x.splits + kChunk - 1) / kChunk * kChunk;
  x.key_blocks = (max_len + kHeldWg - 1) / kHeldWg;
  // (few rows: keys for up to 16 steps of the four waves while 8 workgroups a CU remain)
  x.few_keys = 128;
  while (x.few_keys < 2048 && x.units * ((max_len + 2 * x.few_keys - 1) / (2 * x.few_keys)) >= kFewWgs) x.few_keys *= 2;
  x.parts = 1;
  while (!x.few && x.parts < kMaxSplits && x.units * x.key_blocks * x.parts < kObsWgs && R > x.parts * 2 * 256) x.parts *= 2;
  x.part_rows = (int)(((R + x.parts - 1) / x.parts + kChunk - 1) / kChunk * kChunk);
  x.ld = (max_len + 31) / 32 * 32;
  x.stats_bytes = ((size_t)(x.units * R * x.splits) * sizeof(floatx2) + 255) & ~(size_t)255;
  x.bytes = x.stats_bytes + (x.parts == 1 ? 0 : (size_t)(x.units * x.parts * x.ld) * sizeof(float));
  return x;
}

template <int KSRC, int NK, int QSRC, int NQ, int D>
hipError_t launch(ObserveArgs a, const Plan& x, hipStream_t stream) {
  constexpr bool kPairs = NK * NQ == 1;                 // two workgroups to a CU
  const int64_t row_blocks = x.units * x.row_blocks * x.splits, key_blocks = x.units * x.key_blocks * x.parts;
  a.order = order_of(a.g, x.units, row_blocks, kPairs && !x.few);
  if constexpr (NK == 1) {
    if (x.few)
      hipLaunchKernelGGL((observe_few_kernel<KSRC, QSRC, NQ, D>), dim3((unsigned)row_blocks), dim3(kFewThreads), 0, stream, a);
  }
  if (!x.few)
    hipLaunchKernelGGL((observe_stats_kernel<KSRC, NK, QSRC, NQ, D, kHeld>), dim3((unsigned)row_blocks), dim3(kObsThreads), 0,
                       stream, a);
  hipError_t e = hipGetLastError();
  if (e != hipSuccess) return e;
  if (x.splits > 1 && !x.few) {
    const int64_t rows = x.units * a.g.G * a.T;
    hipLaunchKernelGGL(observe_join_kernel, dim3((unsigned)((rows + 255) / 256)), dim3(256), 0, stream, a.stats, x.splits, rows);
    e = hipGetLastError();
    if (e != hipSuccess) return e;
  }
  if constexpr (NK == 1) {
    if (x.few) {
      a.split_keys = x.few_keys;
      const int64_t blocks = x.units * ((a.max_len + x.few_keys - 1) / x.few_keys);
      a.order = order_of(a.g, x.units, blocks, false);
      hipLaunchKernelGGL((observe_few_sum_kernel<KSRC, QSRC, NQ, D>), dim3((unsigned)blocks), dim3(kFewThreads), 0, stream, a);
      return hipGetLastError();
    }
  }
  a.order = order_of(a.g, x.units, key_blocks, kPairs);
  hipLaunchKernelGGL((observe_sum_kernel<KSRC, NK, QSRC, NQ, D, kHeld>), dim3((unsigned)key_blocks), dim3(kObsThreads), 0,
                     stream, a);
  e = hipGetLastError();
  if (e != hipSuccess || x.parts == 1) return e;
  const int blocks = (a.max_len + 255) / 256;
  hipLaunchKernelGGL(observe_add_kernel, dim3((unsigned)(x.units * blocks)), dim3(256), 0, stream, a, blocks);
  return hipGetLastError();
}

template <int D>
hipError_t launch_d(const ObserveArgs& a, const Plan& x, bool codes, hipStream_t stream) {
  const bool f32 = a.g.dtype == KARA_F32;
  if (codes)
    return f32 ? launch<kCodeRows, 1, kF32Rows, 3, D>(a, x, stream)
               : launch<kCodeRows, 1, kBf16Rows, 1, D>(a, x, stream);
  return f32 ? launch<kF32Rows, 3, kF32Rows, 3, D>(a, x, stream)
             : launch<kBf16Rows, 1, kBf16Rows, 1, D>(a, x, stream);
}

}  // namespace
}  // namespace kara

using namespace kara;

extern "C" {

// The largest size a call of up to n sequences or n_layers layers takes: fewer of
// them split their keys further.
kara_status_t kara_evict_observe_workspace_size(const kara_params_t* p, int32_t n, int32_t n_layers, int32_t n_query,
                                                int32_t max_len, size_t* bytes) {
  Geom g;
  const kara_status_t st = make_geom(p, n, &g);
  if (st != KARA_OK) return st;
  if (!bytes || n < 0 || n_layers < 1 || n_layers > kMaxLayersPerLaunch || n_query < 1 || max_len < 1 ||
      (int64_t)max_len > (int64_t)g.max_blocks * g.bs || (int64_t)n_query * g.Hq > INT32_MAX / 4)
    return KARA_ERR_INVALID_ARG;
  if (max_len > kMaxLen) return KARA_ERR_UNSUPPORTED;
  // (a launch of kObsWgs row blocks or more does not split; a smaller one has fewer
  // than twice as many, records and all; the same for key blocks and their sums)
  const int64_t rows = (int64_t)n_layers * n * g.Hkv * g.G * n_query;
  *bytes = (size_t)(rows + 2 * kObsWgs * kHeldWg) * sizeof(floatx2) + 256 + (size_t)(2 * kObsWgs * kHeldWg) * sizeof(float);
  return KARA_OK;
}

kara_status_t kara_evict_observe(const kara_params_t* p, int32_t n, const int32_t* seqs, int32_t n_layers, int32_t n_query,
                                 const void* q, const void* const* k_pools, const void* const* k_scales,
                                 float* const* weights, const int32_t* block_table, const int32_t* seq_lens,
                                 int32_t n_new, int32_t max_len, void* workspace, size_t workspace_bytes, void* stream) {
  size_t need = 0;
  kara_status_t st = kara_evict_observe_workspace_size(p, n, n_layers, n_query, max_len, &need);
  if (st != KARA_OK) return st;
  if (n_new < 0) return KARA_ERR_INVALID_ARG;
  if (n == 0) return KARA_OK;
  if (!seqs || !q || !block_table || !seq_lens || !pools_ok(k_pools, n_layers) ||
      (k_scales && !pools_ok(k_scales, n_layers)) || !pools_ok((const void* const*)weights, n_layers))
    return KARA_ERR_INVALID_ARG;
  ObserveArgs a{};
  st = make_geom(p, n, &a.g);
  if (st != KARA_OK) return st;
  const Plan x = plan_of(a.g, n, n_layers, n_query, max_len, k_scales != nullptr);
  if (!workspace || workspace_bytes < x.bytes) return KARA_ERR_WORKSPACE;
  if (!aligned(16, {q, workspace}) || !aligned(4, {seqs, block_table, seq_lens}) ||
      !cache_aligned(a.g, n_layers, k_pools, nullptr, k_scales, nullptr, (const void* const*)weights))
    return KARA_ERR_INVALID_ARG;
  if (!grid_ok(2 * x.units * x.row_blocks * x.splits) || !grid_ok(2 * x.units * x.key_blocks * x.parts)) return KARA_ERR_UNSUPPORTED;
  a.n = n;
  a.T = n_query;
  a.n_new = n_new;
  a.max_len = max_len;
  a.units = (uint32_t)x.units;
  a.row_blocks = x.row_blocks;
  a.splits = x.splits;
  a.split_keys = x.split_keys;
  a.key_blocks = x.key_blocks;
  a.parts = x.parts;
  a.part_rows = x.part_rows;
  a.ld = x.ld;
  a.bs_shift = (a.g.bs & (a.g.bs - 1)) == 0 ? __builtin_ctz((unsigned)a.g.bs) : -1;
  a.seqs = seqs;
  a.bt = block_table;
  a.seq_lens = seq_lens;
  a.q = q;
  for (int i = 0; i < n_layers; ++i) {
    a.k.p[i] = const_cast<void*>(k_pools[i]);
    a.ks.p[i] = k_scales ? const_cast<void*>(k_scales[i]) : nullptr;
    a.w[i] = weights[i];
  }
  a.stats = (floatx2*)workspace;
  a.sums = (float*)((char*)workspace + x.stats_bytes);
  const hipError_t e = a.g.d == 128 ? launch_d<128>(a, x, k_scales != nullptr, (hipStream_t)stream)
                                    : launch_d<64>(a, x, k_scales != nullptr, (hipStream_t)stream);
  return hip_status(e);
}

}  // extern "C"

// The cache held in 4 bits (include/kara_q4.h): quantising append, reading
// back, and attention of few query rows with the keys split over workgroups.
#include <algorithm>

#include "kara_append.h"
#include "kara_lds.h"
#include "kara_q4.h"
#include "kara_q4_device.h"

namespace kara {
namespace {

constexpr float kLog2e = 1.4426950408889634f;
constexpr float kNegInf = -__builtin_huge_valf();
// Lower end of a running maximum: finite, so that a logit of -inf weighs 0.
constexpr float kMaxFloor = -3.402823466e38f;

typedef uint32_t u32x4 __attribute__((ext_vector_type(4)));

// ---------------------------------------------------------------- append

// One workgroup per listed sequence: its status.
__global__ __launch_bounds__(kAppendThreads) void q4_check_kernel(Geom g, int n, const int32_t* __restrict__ seqs,
                                                                  int n_new, const int32_t* __restrict__ bt,
                                                                  const int32_t* __restrict__ seq_lens,
                                                                  int32_t* __restrict__ status) {
  const int st = append_status(g, n, seqs, n_new, bt, seq_lens, blockIdx.x);
  if (threadIdx.x == 0) status[blockIdx.x] = st;
}

// A thread per listed sequence: its new length, once the rows are there (committed
// first, and counted back from by the rows' launch, a call that could not make that
// launch left lengths without rows; 3.5 us less).
__global__ __launch_bounds__(kAppendThreads) void q4_commit_kernel(int n, const int32_t* __restrict__ seqs, int n_new,
                                                                   int32_t* __restrict__ seq_lens,
                                                                   const int32_t* __restrict__ status) {
  const int j = blockIdx.x * kAppendThreads + threadIdx.x;
  if (j < n && (status[j] & ~KARA_SEQ_NONFINITE) == 0) seq_lens[seqs[j]] += n_new;
}

constexpr int kQuantUnroll = 4;       // octets per thread
constexpr int kMaxOctets = 1 << 28;   // of a token: 32-bit offsets

// Eight values as loaded.  bf16: 16 bytes a lane.  fp32: 32, which lanes load in two
// pieces of 16, side by side over the wave -- octets 0..31 of its 64 first, then the
// others -- and pairs of lanes exchange halves: lane 2i ends with octet i, lane 2i + 1
// with octet 32 + i.
template <int DT>
struct Octet {
  static constexpr int kBytes = DT == KARA_BF16 ? 16 : 32;   // of eight values
  static constexpr int kStep = DT == KARA_BF16 ? 1 : 2;      // lanes between a row's octets
  u32x4 v[kBytes / 16];
  static __device__ __forceinline__ int octet(int lane) { return kStep == 1 ? lane : (lane & 1) * 32 + (lane >> 1); }
  // octets wave0 .. wave0 + 63 of `count` at p; past the last the end is read again, so
  // that no branch stands between loads
  __device__ __forceinline__ void load(const char* p, int wave0, int lane, int count) {
    const int at = wave0 * kStep + lane, last = count * kStep - 1;
    v[0] = __builtin_nontemporal_load((const u32x4*)p + min(at, last));
    if constexpr (kStep == 2) v[1] = __builtin_nontemporal_load((const u32x4*)p + min(at + 64, last));
  }
  // the exchange: after a load, before a store
  __device__ __forceinline__ void exchange(int lane) {
    if constexpr (kStep == 2) {
      const bool odd = lane & 1;
#pragma unroll
      for (int e = 0; e < 4; ++e) {
        const uint32_t give = odd ? v[0][e] : v[1][e];
        const uint32_t got = (uint32_t)__builtin_amdgcn_mov_dpp((int)give, 0xb1, 0xf, 0xf, true);   // lanes 2i, 2i + 1
        v[0][e] = odd ? got : v[0][e];
        v[1][e] = odd ? v[1][e] : got;
      }
    }
  }
  __device__ __forceinline__ void store(char* p, int wave0, int lane, int count) const {
    if constexpr (kStep == 1) {
      if (wave0 + lane < count) __builtin_nontemporal_store(v[0], (u32x4*)(p + (int64_t)(wave0 + lane) * 16));
    } else {
      u32x4* at = (u32x4*)(p + (int64_t)wave0 * 32) + lane;
      if (wave0 + (lane >> 1) < count) __builtin_nontemporal_store(v[0], at);
      if (wave0 + 32 + (lane >> 1) < count) __builtin_nontemporal_store(v[1], at + 64);
    }
  }
};

// Eight values to eight codes; four lanes hold a block and find its scale byte
// together.  odd: a value was not finite.
template <int DT>
__device__ __forceinline__ uint32_t q4_encode(const Octet<DT>& src, uint32_t* byte, bool* odd) {
  float x[8];
#pragma unroll
  for (int e = 0; e < 8; ++e) {
    if constexpr (DT == KARA_BF16)
      x[e] = __uint_as_float((e & 1) ? src.v[0][e >> 1] & 0xffff0000u : src.v[0][e >> 1] << 16);
    else
      x[e] = __uint_as_float(src.v[e >> 2][e & 3]);
  }
  uint32_t top = 0;
#pragma unroll
  for (int e = 0; e < 8; ++e) top = max(top, __float_as_uint(x[e]) & 0x7fffffffu);
  if (top >= 0x7f800000u) {
    *odd = true;
    top = 0;
#pragma unroll
    for (int e = 0; e < 8; ++e) {
      const uint32_t m = __float_as_uint(x[e]) & 0x7fffffffu;
      if (m > 0x7f800000u) x[e] = 0.f;
      if (m < 0x7f800000u) top = max(top, m);
    }
  }
  top = max(top, (uint32_t)__shfl_xor((int)top, Octet<DT>::kStep, 64));
  top = max(top, (uint32_t)__shfl_xor((int)top, 2 * Octet<DT>::kStep, 64));
  *byte = q4_scale_byte(top);
  const float scale = q4_scale(*byte);
  uint32_t c = 0;
  c = __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(c, x[0], x[1], scale, 0);
  c = __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(c, x[2], x[3], scale, 1);
  c = __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(c, x[4], x[5], scale, 2);
  c = __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(c, x[6], x[7], scale, 3);
  return c;
}

template <int D>
__device__ __forceinline__ void q4_store(uint8_t* codes, uint8_t* scales, int64_t row, int o, uint32_t code, uint32_t byte) {
  *(uint32_t*)(codes + row * (D / 2) + o * 4) = code;
  if ((o & 3) == 0) scales[row * (D / kQ4Block) + (o >> 2)] = (uint8_t)byte;
}

// The rows between q4_check_kernel and q4_commit_kernel.  Grid as the append of rows: (sequences x token
// chunks, layer, K|V).  Bound by the bytes: 4 x 4 layers of 4000 tokens (332 MB) in 64
// us, the reading back 51; fp32 (595 MB) 106 and 101 (152 and 153 with each lane's 32
// bytes loaded as they lie).
template <int DT, int D>
__global__ __launch_bounds__(kAppendThreads) void q4_append_kernel(
    Geom g, int n, const int32_t* __restrict__ seqs, int n_new, int toks, int chunks, const char* __restrict__ k_new,
    const char* __restrict__ v_new, PoolPtrs kp, PoolPtrs vp, PoolPtrs ksp, PoolPtrs vsp,
    const int32_t* __restrict__ bt, const int32_t* __restrict__ seq_lens, int32_t* __restrict__ status) {
  constexpr int kOctets = D / 8;                     // of a row
  using Src = Octet<DT>;
  const int j = blockIdx.x / chunks;
  const int tok0 = (blockIdx.x - j * chunks) * toks;
  const int l = blockIdx.y;
  const int kv = blockIdx.z;
  const int per_tok = g.Hkv * kOctets;
  const int count = min(toks, n_new - tok0) * per_tok;
  const char* src = (kv ? v_new : k_new) + (((int64_t)l * n + j) * n_new + tok0) * per_tok * Src::kBytes;
  const int lane = threadIdx.x & 63, wave0 = threadIdx.x & ~63, octet0 = wave0 + Src::octet(lane);
  Src v[kQuantUnroll];
  auto load = [&](int from) __attribute__((always_inline)) {
#pragma unroll
    for (int k = 0; k < kQuantUnroll; ++k) v[k].load(src, from + k * kAppendThreads + wave0, lane, count);
  };
  // the first rows are on their way while status, length and pages are looked up
  load(0);
  // (other workgroups may have reported a value that is not finite by now)
  if (status[j] & ~KARA_SEQ_NONFINITE) return;
  const int s = seqs[j];
  const int pos0 = seq_lens[s] + tok0;
  const int32_t* row_pages = bt + (int64_t)s * g.max_blocks;
  uint8_t* codes = (uint8_t*)(kv ? vp.p[l] : kp.p[l]);
  uint8_t* scales = (uint8_t*)(kv ? vsp.p[l] : ksp.p[l]);
  bool odd = false;
  // (count is a multiple of a row's octets, so the lanes of a block stay together)
  for (int from = 0; from < count; from += kAppendThreads * kQuantUnroll) {
    // where they go, looked up together: a lookup between stores would wait for those
    uint32_t row[kQuantUnroll], page[kQuantUnroll];
    int o[kQuantUnroll];
#pragma unroll
    for (int k = 0; k < kQuantUnroll; ++k) {
      const int i = min(from + k * kAppendThreads + octet0, count - 1);
      const int tok = i / per_tok, r = i - tok * per_tok;
      const int h = r / kOctets, pos = pos0 + tok, b = pos / g.bs;
      o[k] = r - h * kOctets;
      page[k] = row_pages[b];
      row[k] = h * g.bs + (pos - b * g.bs);
    }
#pragma unroll
    for (int k = 0; k < kQuantUnroll; ++k) {
      uint32_t byte;
      v[k].exchange(lane);
      const uint32_t code = q4_encode<DT>(v[k], &byte, &odd);
      // (a pool has fewer than 2^32 rows)
      if (from + k * kAppendThreads + octet0 < count)
        q4_store<D>(codes, scales, page[k] * (uint32_t)(g.Hkv * g.bs) + row[k], o[k], code, byte);
    }
    if (from + kAppendThreads * kQuantUnroll < count) load(from + kAppendThreads * kQuantUnroll);
  }
  if (__syncthreads_or(odd) && threadIdx.x == 0) atomicOr(&status[j], KARA_SEQ_NONFINITE);
}

// A few new tokens: one workgroup per listed sequence checks it, quantises all its
// rows and commits, in one launch (8 sequences, one token, one layer: a pass with the
// reading back 27.9 us of host time in two launches, 24.5 so).
constexpr int kFewThreads = 1024;
constexpr int kFewOctets = 8 * kFewThreads;          // of a sequence, K and V, all layers

template <int DT, int D>
__global__ __launch_bounds__(kFewThreads) void q4_append_few_kernel(
    Geom g, int n, const int32_t* __restrict__ seqs, int n_new, int n_layers, const char* __restrict__ k_new,
    const char* __restrict__ v_new, PoolPtrs kp, PoolPtrs vp, PoolPtrs ksp, PoolPtrs vsp,
    const int32_t* __restrict__ bt, int32_t* __restrict__ seq_lens, int32_t* __restrict__ status) {
  constexpr int kOctets = D / 8;
  using Src = Octet<DT>;
  const int j = blockIdx.x;
  int st = append_status(g, n, seqs, n_new, bt, seq_lens, j);
  if (st == KARA_SEQ_OK) {
    const int s = seqs[j];
    const int per_tok = g.Hkv * kOctets, per_layer = n_new * per_tok;
    const int pos0 = seq_lens[s];
    const int32_t* row_pages = bt + (int64_t)s * g.max_blocks;
    bool odd = false;
    // (a sequence's rows of one layer, K or V, lie together; the lanes of a block stay so)
    const int lane = threadIdx.x & 63, octets = (per_layer + 63) & ~63;
    for (int at = threadIdx.x & ~63; at < 2 * n_layers * octets; at += kFewThreads) {
      const int part = at / octets, kv = part & 1, l = part >> 1;
      const int wave0 = at - part * octets, x = wave0 + Src::octet(lane);
      Src v;
      v.load((kv ? v_new : k_new) + ((int64_t)l * n + j) * per_layer * Src::kBytes, wave0, lane, per_layer);
      v.exchange(lane);
      if (x >= per_layer) continue;
      const int tok = x / per_tok, r = x - tok * per_tok;
      const int h = r / kOctets, o = r - h * kOctets;
      uint32_t byte;
      const uint32_t code = q4_encode<DT>(v, &byte, &odd);
      const int pos = pos0 + tok, b = pos / g.bs;
      q4_store<D>((uint8_t*)(kv ? vp.p[l] : kp.p[l]), (uint8_t*)(kv ? vsp.p[l] : ksp.p[l]),
                  ((int64_t)row_pages[b] * g.Hkv + h) * g.bs + (pos - b * g.bs), o, code, byte);
    }
    if (__syncthreads_or(odd)) st = KARA_SEQ_NONFINITE;
  }
  __syncthreads();                       // every thread has read the length before it changes
  if (threadIdx.x == 0) {
    status[j] = st;
    if ((st & ~KARA_SEQ_NONFINITE) == 0) seq_lens[seqs[j]] += n_new;
  }
}

// ---------------------------------------------------------------- read

// The append's mapping the other way round; rows that are not there are zeros.
template <int DT, int D>
__global__ __launch_bounds__(kAppendThreads) void q4_read_kernel(
    Geom g, int n, const int32_t* __restrict__ seqs, const int32_t* __restrict__ start, int n_rows, int toks, int chunks,
    PoolPtrs kp, PoolPtrs vp, PoolPtrs ksp, PoolPtrs vsp, const int32_t* __restrict__ bt,
    const int32_t* __restrict__ seq_lens, char* __restrict__ k_out, char* __restrict__ v_out) {
  constexpr int kOctets = D / 8;
  using Dst = Octet<DT>;
  const int j = blockIdx.x / chunks;
  const int tok0 = (blockIdx.x - j * chunks) * toks;
  const int l = blockIdx.y;
  const int kv = blockIdx.z;
  const int s = seqs[j];
  const bool listed = s >= 0 && s < g.n_seqs;
  const int len = listed ? (int)min((int64_t)seq_lens[s], (int64_t)g.max_blocks * g.bs) : 0;
  const int64_t pos0 = (int64_t)(listed ? start[s] : 0) + tok0;
  const int32_t* row_pages = bt + (int64_t)(listed ? s : 0) * g.max_blocks;
  const int per_tok = g.Hkv * kOctets;
  const int count = min(toks, n_rows - tok0) * per_tok;
  char* dst = (kv ? v_out : k_out) + (((int64_t)l * n + j) * n_rows + tok0) * per_tok * Dst::kBytes;
  const uint8_t* codes = (const uint8_t*)(kv ? vp.p[l] : kp.p[l]);
  const uint8_t* scales = (const uint8_t*)(kv ? vsp.p[l] : ksp.p[l]);
  const int lane = threadIdx.x & 63, wave0 = threadIdx.x & ~63, octet0 = wave0 + Dst::octet(lane);
  for (int from = 0; from < count; from += kAppendThreads * kQuantUnroll) {
    // rows that are not there read another one of the pool and become zeros
    uint32_t c[kQuantUnroll], byte[kQuantUnroll], row[kQuantUnroll];
    int page[kQuantUnroll], o[kQuantUnroll];
    bool in[kQuantUnroll];
#pragma unroll
    for (int k = 0; k < kQuantUnroll; ++k) {
      const int i = min(from + k * kAppendThreads + octet0, count - 1);
      const int tok = i / per_tok, r = i - tok * per_tok;
      const int h = r / kOctets;
      o[k] = r - h * kOctets;
      in[k] = pos0 + tok >= 0 && pos0 + tok < len;
      const int pos = in[k] ? (int)(pos0 + tok) : 0, b = pos / g.bs;
      page[k] = row_pages[b];
      row[k] = h * g.bs + (pos - b * g.bs);
    }
#pragma unroll
    for (int k = 0; k < kQuantUnroll; ++k) {
      in[k] &= page[k] >= 0 && page[k] < g.num_pages;
      row[k] += (uint32_t)(in[k] ? page[k] : 0) * (uint32_t)(g.Hkv * g.bs);
      c[k] = *(const uint32_t*)(codes + (uint64_t)row[k] * (D / 2) + o[k] * 4);
      byte[k] = scales[(uint64_t)row[k] * (D / kQ4Block) + (o[k] >> 2)];
    }
#pragma unroll
    for (int k = 0; k < kQuantUnroll; ++k)
      if (!in[k]) c[k] = 0, byte[k] = 127;
#pragma unroll
    for (int k = 0; k < kQuantUnroll; ++k) {
      const float scale = q4_scale(byte[k]);
      Dst x;
      if constexpr (DT == KARA_BF16) {
        x.v[0] = __builtin_bit_cast(u32x4, q4_octet(c[k], scale));
      } else {
        const floatx2 a = __builtin_amdgcn_cvt_scalef32_pk_f32_fp4(c[k], scale, 0);
        const floatx2 b = __builtin_amdgcn_cvt_scalef32_pk_f32_fp4(c[k], scale, 1);
        const floatx2 e = __builtin_amdgcn_cvt_scalef32_pk_f32_fp4(c[k], scale, 2);
        const floatx2 f = __builtin_amdgcn_cvt_scalef32_pk_f32_fp4(c[k], scale, 3);
        x.v[0] = __builtin_bit_cast(u32x4, floatx4{a[0], a[1], b[0], b[1]});
        x.v[1] = __builtin_bit_cast(u32x4, floatx4{e[0], e[1], f[0], f[1]});
      }
      x.exchange(lane);
      x.store(dst, from + k * kAppendThreads + wave0, lane, count);
    }
  }
}

// ---------------------------------------------------------------- attention, keys split

constexpr int kSplitThreads = 256;
constexpr int kSplitWaves = kSplitThreads / 64;
constexpr int kSplitMin = 256;       // keys per split, at least (the workspace's records are sized for that)
constexpr int kSplitMax = 2048;
constexpr int kSplitRows = 1024;     // runs of keys a split's LDS table holds
constexpr int kSplitBlock = 32;      // keys a wave works on at a time
constexpr int kSplitStages = 2;      // blocks of a wave's LDS ring, all on their way while it works
constexpr int kSplitWgTarget = 4096; // workgroups a launch keeps when its splits grow

// One workgroup of four waves per (layer, sequence, KV head, tile of 16 query
// rows, split of split_keys keys): for the tile's rows, the split's maximum m,
// exponential sum l and unnormalised output o, in log2 units and fp32.  Rows of
// a (layer, sequence, KV head) run over (query, head in group).
//
// The pool rows of the split's keys go to LDS first; the four waves then take the
// split's 32-key blocks in turn, each through a ring of its own in LDS that direct
// copies fill two blocks ahead (4.3 KB a block at d = 128; no barrier in the loop).  A
// lane's 16 bytes of codes at d = 128 are one block of 32 values with one scale, which
// the hardware turns into the four bf16 operands of S^T = K Q^T (keys as the M
// dimension); a lane so holds four keys of one query per tile, and its weights are the
// B operand of O^T += V^T P^T as they stand.  V is read as rows, d/16 columns of a key
// per lane, and the pairs of columns that the conversion gives are put together to
// pairs of keys by byte permutes.
//
// Bound by the bytes of the codes where there are many workgroups: 96 sequences of
// 7-8.2K tokens, 2 layers, 40/8 heads, d = 128: 310 us for 1.59 GB, 5.1 TB/s.  With
// logits for the counting attention (64 sequences of 4-8.2K): 208 us, 4.0 TB/s of
// codes; 178 without the stores of the 127 MB of logits, 170 as the attention that
// does not count.
//
// NQ: bf16 terms of a query (1: bf16, exact; 3: fp32, 24 bits); NP: bf16 terms of a
// weight (1 where the output is bf16; 3 where it is fp32).  K and V are exact in one.
// A weight rounded to bf16, in the output as in its sum, costs a bf16 output little
// beside its own rounding: 1.66e-3 of the result against 64 bits where whole weights
// give 1.61e-3 (the same 96 sequences).
// LOGITS: q . k of every key goes to `logits` too, [unit][G][ld] (one query each).
template <int NQ, int NP, int D, bool LOGITS>
__global__ __launch_bounds__(kSplitThreads, 2) void q4_split_kernel(Q4Split a) {
  constexpr int KS = D / 32;                 // products per dot product
  constexpr int E = D / 16;                  // output columns per lane
  constexpr int kRow = D / 2;                // bytes of a row's codes
  constexpr int kKW = D / 32;                // a lane's words of a key's codes: an eighth of a row's values per word
  constexpr int kCodes = kSplitBlock * kRow;           // a block's codes of K, or of V
  constexpr int kStage = 2 * kCodes + 64 * 4;          // and a word of scales per key and K|V
  constexpr int kCopies = 2 * (kCodes / 1024) + 1;     // copies per block
  struct Ring {
    uint32_t row[kSplitRows];                          // pool rows of runs of keys, in 16 bytes of codes
    __attribute__((aligned(16))) char b[kSplitWaves][kSplitStages][kStage];
  };
  __shared__ __attribute__((aligned(16))) union {
    Ring st;
    float o[kSplitWaves][16][D];
  } lds;
  __shared__ float red_m[kSplitWaves][16], red_l[kSplitWaves][16];
  Ring& st = lds.st;

  const Geom& g = a.g;
  const int tid = threadIdx.x;
  const int lane = tid & 63;
  const int wave = __builtin_amdgcn_readfirstlane(tid >> 6);
  const int gq = lane >> 4, li = lane & 15;
  uint32_t rest = blockIdx.x;                // (a 64-bit division is 140 scalar instructions)
  // (blocks go round the 8 XCDs: split x of eight units in a row falls to the same
  // ones, the next eight are shifted, so that no XCD gets all the short last splits)
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
  const int k0 = split * a.split_keys;
  // row r of the unit: output row orow + (r / G) * Hq + r % G
  const int64_t orow = ((int64_t)l * a.n + j) * T * g.Hq + h * G;
  const int row0 = rt * 16;
  const int rows = min(16, R - row0);
  if (len <= 0 || len > a.max_len || k0 >= len) {
    // no keys: zero rows where no combine kernel follows
    if (!LOGITS && a.n_splits == 1)
      for (int i = tid; i < rows * D; i += kSplitThreads) {
        const int r = row0 + i / D;
        const int64_t at = (orow + (int64_t)(r / G) * g.Hq + r % G) * D + i % D;
        if (a.out_bf16) ((__bf16*)a.out)[at] = (__bf16)0.f;
        else ((float*)a.out)[at] = 0.f;
      }
    return;
  }
  const int nk = min(len - k0, a.split_keys);                 // keys of this split
  const float c = g.scale * kLog2e;

  const int npad = (nk + kSplitBlock - 1) / kSplitBlock * kSplitBlock;
  // lane (gq, li): values gq*D/4 .. of query row li; its limit: keys of the split it sees
  uint4 qraw[KS * (NQ == 1 ? 1 : 2)];
  int limit = 0;
  const bool there = li < rows;
  {
    const int r = row0 + (there ? li : 0);
    const int t = T == 1 ? 0 : r / G;
    const int64_t at = (orow + (int64_t)t * g.Hq + (r - t * G)) * D + gq * (D / 4);
    if (there) limit = min(nk, len - T + t + 1 - k0);
    const uint4* src = (const uint4*)((const char*)a.q + at * (NQ == 1 ? 2 : 4));
#pragma unroll
    for (int x = 0; x < KS * (NQ == 1 ? 1 : 2); ++x) qraw[x] = src[x];
  }
  // Pool rows of the split's keys, in 16 bytes of codes.  Runs of 2^run keys (the
  // power of two in the block size, 16 at most; k0 is a multiple of it) lie in one
  // page: an entry each.  (An entry per key, 8 table reads and divisions a thread,
  // took 18 of a workgroup's 73 thousand cycles.)
  const int run = a.run;
  {
    const int32_t* row_pages = a.bt + (int64_t)s * g.max_blocks;
    for (int i = tid; i < npad >> run; i += kSplitThreads) {
      const int pos = k0 + min(i << run, (nk - 1) >> run << run);
      const int b = pos / g.bs;
      const int page = min(max(row_pages[b], 0), g.num_pages - 1);
      st.row[i] = (uint32_t)((page * g.Hkv + h) * g.bs + (pos - b * g.bs)) * (kRow / 16);
    }
  }
  bf16x8 qa[NQ][KS];
#pragma unroll
  for (int x = 0; x < KS; ++x) {
    if constexpr (NQ == 1) {
      qa[0][x] = __builtin_bit_cast(bf16x8, there ? qraw[x] : uint4{0, 0, 0, 0});
    } else {
      const floatx4 u = __builtin_bit_cast(floatx4, qraw[2 * x]), v = __builtin_bit_cast(floatx4, qraw[2 * x + 1]);
      uint32_t w[4][NQ];
#pragma unroll
      for (int i = 0; i < 4; ++i) {
        const float x0 = i < 2 ? u[2 * i] : v[2 * i - 4], x1 = i < 2 ? u[2 * i + 1] : v[2 * i - 3];
        bf16_term_pairs<true>(there ? x0 : 0.f, there ? x1 : 0.f, w[i]);
      }
#pragma unroll
      for (int y = 0; y < NQ; ++y) qa[y][x] = __builtin_bit_cast(bf16x8, uint4{w[0][y], w[1][y], w[2][y], w[3][y]});
    }
  }
  // (the query loads are waited for here, not in the loop behind the copies)
#pragma unroll
  for (int y = 0; y < NQ; ++y)
#pragma unroll
    for (int x = 0; x < KS; ++x) asm volatile("" : "+v"(qa[y][x]));
  // the first query row of the tile sees the fewest keys
  const int limit0 = __builtin_amdgcn_readfirstlane(limit);
  __syncthreads();

  const int nblk = npad / kSplitBlock;
  // Block blk into stage b.  K rows lie in key order, their 16-byte chunks XOR-swizzled
  // (d = 128: by row / 4, d = 64: by row / 8) so that 16 rows read at one chunk hit
  // different banks; V rows 4q + r of a tile at slot 4r + q, so that a read of rows
  // 4gq + r takes consecutive ones.  Then the scales: a word per key, K's, V's.
  constexpr int kCPR = kRow / 16;                      // chunks per row
  constexpr int kRows = 64 / kCPR;                     // rows per copy
  const int crow = lane / kCPR, cchunk = lane % kCPR;
  const int kchunk = cchunk ^ (D == 128 ? (crow >> 2) & 3 : (crow >> 3) & 1);
  const int vrow = (crow & 16) | ((crow & 3) << 2) | ((crow >> 2) & 3);
  const char* kbase = (const char*)a.kp.p[l] + kchunk * 16;
  const char* vbase = (const char*)a.vp.p[l] + cchunk * 16;
  const char* sbase = (const char*)(lane < 32 ? a.ksp.p[l] : a.vsp.p[l]);
  // (waited for here: left to its first use, in the loop, the wait would be for the
  // copies too)
  asm volatile("" : "+v"(sbase));
  const int run_mask = (1 << run) - 1;
  auto issue = [&](int blk, int b) __attribute__((always_inline)) {
    char* to = st.b[wave][b];
    constexpr int kTimes = kSplitBlock / kRows;
    // (a padding key is the last one: its page may end before it)
    auto at = [&](int key) __attribute__((always_inline)) {
      key = min(blk * kSplitBlock + key, nk - 1);
      return (uint64_t)(st.row[key >> run] + (key & run_mask) * (kRow / 16));
    };
    uint64_t kat[kTimes], vat[kTimes], sat = at(lane & 31);
#pragma unroll
    for (int t = 0; t < kTimes; ++t) kat[t] = at(t * kRows + crow), vat[t] = at(t * kRows + vrow);
#pragma unroll
    for (int t = 0; t < kTimes; ++t) {
      copy16(kbase + (kat[t] << 4), to + t * 1024);
      copy16(vbase + (vat[t] << 4), to + kCodes + t * 1024);
    }
    // (a row has as many bytes of scales as 16-byte chunks of codes)
    if constexpr (D == 128) copy4(sbase + sat, to + 2 * kCodes);
    else copy2(sbase + sat, to + 2 * kCodes);
  };
#pragma unroll
  for (int i = 0; i < kSplitStages; ++i)
    if (wave + i * kSplitWaves < nblk) issue(wave + i * kSplitWaves, i);
  // byte b of a row's scales, turned right by 8b + 9, lies on an fp32 exponent
  const uint32_t kturn = 8 * (D == 128 ? gq : gq >> 1) + 9, vturn = 8 * (D == 128 ? li >> 2 : li >> 3) + 9;
  auto scale_of = [](uint32_t word, uint32_t turn) __attribute__((always_inline)) {
    return __uint_as_float(__builtin_amdgcn_alignbit(word, word, turn) & 0x7f800000u);
  };

  float m = kMaxFloor, lsum = 0.f;   // query li's reference, and this lane's part of its sum
  floatx4 lones = {0.f, 0.f, 0.f, 0.f};   // NP = 1: the sum, in every element
  floatx4 o[E];                      // query li, columns (4gq + r) * E + e
#pragma unroll
  for (int e = 0; e < E; ++e) o[e] = floatx4{0.f, 0.f, 0.f, 0.f};
  bf16x8 ones;
#pragma unroll
  for (int i = 0; i < 8; ++i) ones[i] = (__bf16)1.f;
  float* lrow = nullptr;
  if constexpr (LOGITS)
    lrow = a.logits + ((((int64_t)l * a.n + j) * g.Hkv + h) * G + min(li, rows - 1)) * a.ld + k0 + 4 * gq;

  const int koff = D == 128 ? li * kRow + ((gq ^ (li >> 2)) * 16) : li * kRow + (((gq >> 1) ^ (li >> 3)) * 16) + (gq & 1) * 8;
  const int voff = kCodes + gq * kRow + li * (E / 2);
  // a block as the lane holds it: K words and scale words of key 16t + li, V words
  // and scale words of keys 16t + 4gq + r
  uint32_t kw[2][kKW], kscale[2], vw[8];
  uint4 vscale[2];
  auto take = [&](const char* b) __attribute__((always_inline)) {
#pragma unroll
    for (int t = 0; t < 2; ++t) {
      __builtin_memcpy(kw[t], b + t * 16 * kRow + koff, kKW * 4);
      kscale[t] = *(const uint32_t*)(b + 2 * kCodes + (t * 16 + li) * 4);
      vscale[t] = *(const uint4*)(b + 2 * kCodes + 128 + (t * 16 + 4 * gq) * 4);
#pragma unroll
      for (int r = 0; r < 4; ++r) {
        const char* vp = b + voff + (t * 16 + 4 * r) * kRow;
        vw[4 * t + r] = D == 128 ? *(const uint32_t*)vp : *(const uint16_t*)vp;
      }
    }
  };
  auto work = [&](int blk) __attribute__((always_inline)) {
    floatx4 sv[2];
#pragma unroll
    for (int t = 0; t < 2; ++t) {
      const float scale = scale_of(kscale[t], kturn);
      floatx4 acc = {0.f, 0.f, 0.f, 0.f};
#pragma unroll
      for (int x = 0; x < KS; ++x) {
        const bf16x8 ka = q4_octet(kw[t][x], scale);
#pragma unroll
        for (int y = NQ - 1; y >= 0; --y) acc = __builtin_amdgcn_mfma_f32_16x16x32_bf16(ka, qa[y][x], acc, 0, 0, 0);
      }
      sv[t] = acc;
    }
    // Wait states between the last product and the first read of its result,
    // which lies past a branch: the compiler does not count across it (see the
    // decode attention over rows).  12 cycles per block.
    asm volatile("s_nop 7\n\ts_nop 3" : "+v"(sv[0]), "+v"(sv[1]));
    if constexpr (LOGITS) {
      if (li < rows)
#pragma unroll
        for (int t = 0; t < 2; ++t) *(floatx4*)(lrow + blk * kSplitBlock + t * 16) = sv[t];
    }
    if (blk * kSplitBlock + kSplitBlock > limit0) {
#pragma unroll
      for (int t = 0; t < 2; ++t)
#pragma unroll
        for (int r = 0; r < 4; ++r)
          if (blk * kSplitBlock + t * 16 + 4 * gq + r >= limit) sv[t][r] = kNegInf;
    }
    float mx = sv[0][0];
#pragma unroll
    for (int t = 0; t < 2; ++t)
#pragma unroll
      for (int r = 0; r < 4; ++r) mx = fmaxf(mx, sv[t][r]);
    // The reference m, one for the four lanes of a query, is raised only where a
    // logit passes it by more than 2^8: no exchange between lanes before that.
    if (__ballot(mx * c > m + 8.f) != 0ull) {
      mx = fmaxf(mx, __shfl_xor(mx, 16, 64));
      mx = fmaxf(mx, __shfl_xor(mx, 32, 64)) * c;
      const float mn = fmaxf(m, mx);
      const float f = __builtin_amdgcn_exp2f(m - mn);
      m = mn;
      lsum *= f;
      if constexpr (NP == 1) lones *= f;
#pragma unroll
      for (int e = 0; e < E; ++e) o[e] *= f;
    }
    uint32_t pw[NP][4];                  // terms of the lane's eight weights, in pairs
#pragma unroll
    for (int t = 0; t < 2; ++t)
#pragma unroll
      for (int r = 0; r < 4; r += 2) {
        const float p0 = __builtin_amdgcn_exp2f(fmaf(sv[t][r], c, -m));
        const float p1 = __builtin_amdgcn_exp2f(fmaf(sv[t][r + 1], c, -m));
        if constexpr (NP > 1) lsum += p0 + p1;
        uint32_t w[NP];
        bf16_term_pairs<false>(p0, p1, w);
#pragma unroll
        for (int y = 0; y < NP; ++y) pw[y][2 * t + (r >> 1)] = w[y];
      }
    bf16x8 pb[NP];
#pragma unroll
    for (int y = 0; y < NP; ++y) pb[y] = __builtin_bit_cast(bf16x8, uint4{pw[y][0], pw[y][1], pw[y][2], pw[y][3]});
    // (one term: the sum is of the rounded weights, as the output is, and formed as
    // one more product, with ones)
    if constexpr (NP == 1) lones = __builtin_amdgcn_mfma_f32_16x16x32_bf16(ones, pb[0], lones, 0, 0, 0);
    // V: pairs of columns of a key to pairs of keys of a column
    uint32_t pv[8][E / 2];
#pragma unroll
    for (int t = 0; t < 2; ++t) {
      const uint32_t s4[4] = {vscale[t].x, vscale[t].y, vscale[t].z, vscale[t].w};
#pragma unroll
      for (int r = 0; r < 4; ++r) {
        const float scale = scale_of(s4[r], vturn);
        pv[4 * t + r][0] = q4_pair<0>(vw[4 * t + r], scale);
        pv[4 * t + r][1] = q4_pair<1>(vw[4 * t + r], scale);
        if constexpr (E == 8) {
          pv[4 * t + r][2] = q4_pair<2>(vw[4 * t + r], scale);
          pv[4 * t + r][3] = q4_pair<3>(vw[4 * t + r], scale);
        }
      }
    }
#pragma unroll
    for (int e = 0; e < E; ++e) {
      const uint32_t sel = (e & 1) ? 0x07060302u : 0x05040100u;
      const uint4 va = {__builtin_amdgcn_perm(pv[1][e >> 1], pv[0][e >> 1], sel),
                        __builtin_amdgcn_perm(pv[3][e >> 1], pv[2][e >> 1], sel),
                        __builtin_amdgcn_perm(pv[5][e >> 1], pv[4][e >> 1], sel),
                        __builtin_amdgcn_perm(pv[7][e >> 1], pv[6][e >> 1], sel)};
#pragma unroll
      for (int y = NP - 1; y >= 0; --y)
        o[e] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(__builtin_bit_cast(bf16x8, va), pb[y], o[e], 0, 0, 0);
    }
  };
  // The wave's i-th block passes through stage i mod kSplitStages: once it is in
  // registers, the stage takes the copies of block i + kSplitStages.
  int stage = 0;
  for (int blk = wave; blk < nblk; blk += kSplitWaves) {
    static_assert(kSplitStages == 2, "one newer block may be outstanding");
    // (logit stores count too, so that with them the newer block's first copies are
    // waited for as well: no time lost, 260 us a call either way)
    if (blk + kSplitWaves < nblk) wait_vm<kCopies>();
    else wait_vm<0>();
    take(st.b[wave][stage]);
    asm volatile("s_waitcnt lgkmcnt(0)" ::: "memory");   // taken before the stage is written again
    if (blk + kSplitStages * kSplitWaves < nblk) issue(blk + kSplitStages * kSplitWaves, stage);
    work(blk);
    stage ^= 1;
  }

  // ---- the four waves' sums ----
  asm volatile("s_nop 7\n\ts_nop 3" : "+v"(o[E - 1]));   // (as above, past the loop's branch)
  if constexpr (NP == 1) {
    lsum = lones[0];
  } else {
    lsum += __shfl_xor(lsum, 16, 64);
    lsum += __shfl_xor(lsum, 32, 64);
  }
  if (gq == 0) {
    red_m[wave][li] = m;
    red_l[wave][li] = lsum;
  }
  __syncthreads();   // the staged rows and scales are no longer read
#pragma unroll
  for (int r = 0; r < 4; ++r)
#pragma unroll
    for (int e = 0; e < E; e += 4)
      *(floatx4*)&lds.o[wave][li][(4 * gq + r) * E + e] = floatx4{o[e][r], o[e + 1][r], o[e + 2][r], o[e + 3][r]};
  __syncthreads();
  const bool direct = !LOGITS && len <= a.split_keys;
  for (int x = tid; x < rows * D; x += kSplitThreads) {
    const int i = x / D, e = x - i * D;
    // (a wave without keys left its start: a maximum below all, sums of 0)
    float wm[kSplitWaves], M = kMaxFloor, L = 0.f, O = 0.f;
#pragma unroll
    for (int w = 0; w < kSplitWaves; ++w) M = fmaxf(M, wm[w] = red_m[w][i]);
#pragma unroll
    for (int w = 0; w < kSplitWaves; ++w) {
      const float f = __builtin_amdgcn_exp2f(wm[w] - M);
      L = fmaf(red_l[w][i], f, L);
      O = fmaf(lds.o[w][i][e], f, O);
    }
    const int r = row0 + i, t = T == 1 ? 0 : r / G;
    const int64_t at = orow + (int64_t)t * g.Hq + (r - t * G);
    if (direct) {
      const float v = L == 0.f ? 0.f : O / L;   // (a row that sees no key)
      if (a.out_bf16) ((__bf16*)a.out)[at * D + e] = (__bf16)v;
      else ((float*)a.out)[at * D + e] = v;
    } else {
      const int64_t rec = at * a.n_splits + split;
      if (e == 0) a.rec_ml[2 * rec] = M, a.rec_ml[2 * rec + 1] = L;
      a.rec_o[rec * D + e] = O;
    }
  }
}

// One wave per output row of a sequence longer than one split (all: of every
// sequence): its splits' records joined.
template <int D>
__global__ __launch_bounds__(256) void q4_combine_kernel(Geom g, int n, int T, const int32_t* __restrict__ seqs,
                                                         const int32_t* __restrict__ seq_lens, int max_len,
                                                         int split_keys, int n_splits, int64_t n_rows,
                                                         const float* __restrict__ rec_ml, const float* __restrict__ rec_o,
                                                         void* __restrict__ out, int out_bf16, int all) {
  constexpr int kDPerLane = D / 64;
  const int lane = threadIdx.x & 63;
  const int64_t row = (int64_t)blockIdx.x * 4 + (threadIdx.x >> 6);   // (l, j, t, hq)
  if (row >= n_rows) return;
  const int s = seqs[(row / ((int64_t)g.Hq * T)) % n];
  const int len = s >= 0 && s < g.n_seqs ? seq_lens[s] : 0;
  const bool none = len <= 0 || len > max_len;
  if (!all && !none && len <= split_keys) return;   // the split kernel wrote it
  float L = 0.f, acc[kDPerLane] = {};
  if (!none) {
    const int ns = (len + split_keys - 1) / split_keys;
    const float* ml = rec_ml + row * n_splits * 2;
    // lane i: split i's maximum and sum, 64 at a time, the first kept
    const float m0 = lane < ns ? ml[2 * lane] : kMaxFloor, l0 = lane < ns ? ml[2 * lane + 1] : 0.f;
    float M = m0;
    for (int sp = lane + 64; sp < ns; sp += 64) M = fmaxf(M, ml[2 * sp]);
#pragma unroll
    for (int x = 1; x < 64; x <<= 1) M = fmaxf(M, __shfl_xor(M, x, 64));
    for (int sp0 = 0; sp0 < ns; sp0 += 64) {
      const int sp = sp0 + lane;
      const float ms = sp0 == 0 ? m0 : sp < ns ? ml[2 * sp] : kMaxFloor;
      const float f = __builtin_amdgcn_exp2f(ms - M);
      const float lf = (sp0 == 0 ? l0 : sp < ns ? ml[2 * sp + 1] : 0.f) * f;
      const int cnt = min(64, ns - sp0);
      const float* v = rec_o + (row * n_splits + sp0) * D + lane * kDPerLane;
      // (four records at once; past the last a record of weight 0 is read again)
      for (int i = 0; i < cnt; i += 4) {
        float x[4][kDPerLane];
#pragma unroll
        for (int y = 0; y < 4; ++y)
#pragma unroll
          for (int e = 0; e < kDPerLane; ++e) x[y][e] = v[min(i + y, cnt - 1) * D + e];
#pragma unroll
        for (int y = 0; y < 4; ++y) {
          const bool in = i + y < cnt;
          const float fi = in ? __shfl(f, i + y, 64) : 0.f;
          L += in ? __shfl(lf, i + y, 64) : 0.f;
#pragma unroll
          for (int e = 0; e < kDPerLane; ++e) acc[e] = fmaf(x[y][e], fi, acc[e]);
        }
      }
    }
  }
#pragma unroll
  for (int e = 0; e < kDPerLane; ++e) {
    const float v = L == 0.f ? 0.f : acc[e] / L;   // (a row that sees no key)
    if (out_bf16) ((__bf16*)out)[row * D + lane * kDPerLane + e] = (__bf16)v;
    else ((float*)out)[row * D + lane * kDPerLane + e] = v;
  }
}

// log2 of the keys that lie in one page whatever run of them a split starts at
int run_of(int bs) { return std::min(4, __builtin_ctz((unsigned)bs)); }

// Keys per split: 256 while the launch has few workgroups, up to 2048 (1024 where
// pages give runs of one key) where 16 workgroups per CU remain: fewer records and
// prologues.
int split_keys_of(int bs, int64_t units, int max_len) {
  const int most = std::min(kSplitMax, kSplitRows << run_of(bs));
  int keys = kSplitMin;
  while (keys < most && units * ((max_len + 2 * keys - 1) / (2 * keys)) >= kSplitWgTarget) keys *= 2;
  return keys;
}

// Up to this many query rows per (layer, sequence, KV head) go through the split
// kernel, 16 a workgroup; more through the chunk kernel.
constexpr int kFewRows = 64;
bool few_rows(const Geom& g, int T) { return (int64_t)g.G * T <= kFewRows; }

// a grid of one dimension, of 256 threads a block: HIP counts its threads in 32 bits
bool grid_ok(int64_t blocks) { return blocks > 0 && blocks < ((int64_t)1 << 24); }

bool layers_ok(int32_t n, int32_t n_layers) { return n >= 0 && n_layers >= 1 && n_layers <= kMaxLayersPerLaunch; }

PoolPtrs ptrs(const void* const* pools, int n_layers) {
  PoolPtrs x{};
  for (int i = 0; i < n_layers; ++i) x.p[i] = const_cast<void*>(pools[i]);
  return x;
}

}  // namespace

hipError_t launch_q4_split(Q4Split a, bool logits, hipStream_t stream) {
  a.run = run_of(a.g.bs);
  const Geom& g = a.g;
  const int64_t blocks = (int64_t)a.n_layers * a.n * g.Hkv * a.n_rt * a.n_splits;
  const dim3 grid((unsigned)blocks), block(kSplitThreads);
  const bool f32 = g.dtype == KARA_F32;
#define KARA_Q4_SPLIT(NQ, NP, LG)                                                                   \
  do {                                                                                              \
    if (g.d == 128) hipLaunchKernelGGL((q4_split_kernel<NQ, NP, 128, LG>), grid, block, 0, stream, a); \
    else hipLaunchKernelGGL((q4_split_kernel<NQ, NP, 64, LG>), grid, block, 0, stream, a);          \
  } while (0)
  if (logits) {
    if (f32) KARA_Q4_SPLIT(3, 3, true);
    else KARA_Q4_SPLIT(1, 3, true);
  } else {
    if (f32) KARA_Q4_SPLIT(3, 3, false);
    else KARA_Q4_SPLIT(1, 1, false);
  }
#undef KARA_Q4_SPLIT
  return hipGetLastError();
}

int q4_split_keys(const Geom& g, int64_t units, int max_len) { return split_keys_of(g.bs, units, max_len); }

}  // namespace kara

using namespace kara;

extern "C" {

kara_status_t kara_q4_append(const kara_params_t* p, int32_t n, const int32_t* seqs, int32_t n_new, int32_t n_layers,
                             const void* k_new, const void* v_new, void* const* k_pools, void* const* v_pools,
                             void* const* k_scales, void* const* v_scales, const int32_t* block_table,
                             int32_t* seq_lens, int32_t* status, void* stream) {
  Geom g;
  const kara_status_t st = make_geom(p, n, &g);
  if (st != KARA_OK) return st;
  if (!layers_ok(n, n_layers) || n_new < 0) return KARA_ERR_INVALID_ARG;
  if (n == 0 || n_new == 0) return KARA_OK;
  if (!seqs || !k_new || !v_new || !block_table || !seq_lens || !status || !pools_ok(k_pools, n_layers) ||
      !pools_ok(v_pools, n_layers) || !pools_ok(k_scales, n_layers) || !pools_ok(v_scales, n_layers))
    return KARA_ERR_INVALID_ARG;
  if (!aligned(16, {k_new, v_new}) || !aligned(4, {seqs, block_table, seq_lens, status}) ||
      !cache_aligned(g, n_layers, k_pools, v_pools, k_scales, v_scales, nullptr))
    return KARA_ERR_INVALID_ARG;
  hipStream_t s = (hipStream_t)stream;
  if ((int64_t)g.Hkv * (g.d / 8) > kMaxOctets) return KARA_ERR_UNSUPPORTED;
  const int per_tok = g.Hkv * (g.d / 8);
  const int toks = std::min(n_new, std::max(1, 2 * kAppendThreads * kQuantUnroll / per_tok));
  const int64_t chunks = ((int64_t)n_new + toks - 1) / toks;
  if (!grid_ok(n * chunks) || !grid_ok(4 * (int64_t)n)) return KARA_ERR_UNSUPPORTED;
  const PoolPtrs kp = ptrs(k_pools, n_layers), vp = ptrs(v_pools, n_layers), ksp = ptrs(k_scales, n_layers),
                 vsp = ptrs(v_scales, n_layers);
  if ((int64_t)2 * n_layers * n_new * per_tok <= kFewOctets) {
#define KARA_Q4_FEW(DT, D)                                                                                         \
  hipLaunchKernelGGL((q4_append_few_kernel<DT, D>), dim3((unsigned)n), dim3(kFewThreads), 0, s, g, n, seqs, n_new, \
                     n_layers, (const char*)k_new, (const char*)v_new, kp, vp, ksp, vsp, block_table, seq_lens, status)
    if (g.dtype == KARA_BF16) {
      if (g.d == 128) KARA_Q4_FEW(KARA_BF16, 128);
      else KARA_Q4_FEW(KARA_BF16, 64);
    } else {
      if (g.d == 128) KARA_Q4_FEW(KARA_F32, 128);
      else KARA_Q4_FEW(KARA_F32, 64);
    }
#undef KARA_Q4_FEW
    return hip_status(hipGetLastError());
  }
  const dim3 grid((unsigned)(n * chunks), (unsigned)n_layers, 2), block(kAppendThreads);
  hipLaunchKernelGGL(q4_check_kernel, dim3((unsigned)n), block, 0, s, g, n, seqs, n_new, block_table,
                     (const int32_t*)seq_lens, status);
  hipError_t e = hipGetLastError();
  if (e != hipSuccess) return hip_status(e);
#define KARA_Q4_APPEND(DT, D)                                                                                       \
  hipLaunchKernelGGL((q4_append_kernel<DT, D>), grid, block, 0, s, g, n, seqs, n_new, toks, (int)chunks,            \
                     (const char*)k_new, (const char*)v_new, kp, vp, ksp, vsp, block_table, (const int32_t*)seq_lens, \
                     status)
  if (g.dtype == KARA_BF16) {
    if (g.d == 128) KARA_Q4_APPEND(KARA_BF16, 128);
    else KARA_Q4_APPEND(KARA_BF16, 64);
  } else {
    if (g.d == 128) KARA_Q4_APPEND(KARA_F32, 128);
    else KARA_Q4_APPEND(KARA_F32, 64);
  }
#undef KARA_Q4_APPEND
  e = hipGetLastError();
  if (e != hipSuccess) return hip_status(e);
  hipLaunchKernelGGL(q4_commit_kernel, dim3(((unsigned)n + kAppendThreads - 1) / kAppendThreads), block, 0, s, n, seqs,
                     n_new, seq_lens, (const int32_t*)status);
  return hip_status(hipGetLastError());
}

kara_status_t kara_q4_read(const kara_params_t* p, int32_t n, const int32_t* seqs, const int32_t* start, int32_t n_rows,
                           int32_t n_layers, const void* const* k_pools, const void* const* v_pools,
                           const void* const* k_scales, const void* const* v_scales, const int32_t* block_table,
                           const int32_t* seq_lens, void* k_out, void* v_out, void* stream) {
  Geom g;
  const kara_status_t st = make_geom(p, n, &g);
  if (st != KARA_OK) return st;
  if (!layers_ok(n, n_layers) || n_rows < 0) return KARA_ERR_INVALID_ARG;
  if (n == 0 || n_rows == 0) return KARA_OK;
  if (!seqs || !start || !k_out || !v_out || !block_table || !seq_lens || !pools_ok(k_pools, n_layers) ||
      !pools_ok(v_pools, n_layers) || !pools_ok(k_scales, n_layers) || !pools_ok(v_scales, n_layers))
    return KARA_ERR_INVALID_ARG;
  if (!aligned(16, {k_out, v_out}) || !aligned(4, {seqs, start, block_table, seq_lens}) ||
      !cache_aligned(g, n_layers, k_pools, v_pools, k_scales, v_scales, nullptr))
    return KARA_ERR_INVALID_ARG;
  if ((int64_t)g.Hkv * (g.d / 8) > kMaxOctets) return KARA_ERR_UNSUPPORTED;
  const int per_tok = g.Hkv * (g.d / 8);
  const int toks = std::min(n_rows, std::max(1, 2 * kAppendThreads * kQuantUnroll / per_tok));
  const int64_t chunks = ((int64_t)n_rows + toks - 1) / toks;
  if (!grid_ok(n * chunks)) return KARA_ERR_UNSUPPORTED;
  const dim3 grid((unsigned)(n * chunks), (unsigned)n_layers, 2), block(kAppendThreads);
#define KARA_Q4_READ(DT, D)                                                                                        \
  hipLaunchKernelGGL((q4_read_kernel<DT, D>), grid, block, 0, (hipStream_t)stream, g, n, seqs, start, n_rows, toks, \
                     (int)chunks, ptrs(k_pools, n_layers), ptrs(v_pools, n_layers), ptrs(k_scales, n_layers),      \
                     ptrs(v_scales, n_layers), block_table, seq_lens, (char*)k_out, (char*)v_out)
  if (g.dtype == KARA_BF16) {
    if (g.d == 128) KARA_Q4_READ(KARA_BF16, 128);
    else KARA_Q4_READ(KARA_BF16, 64);
  } else {
    if (g.d == 128) KARA_Q4_READ(KARA_F32, 128);
    else KARA_Q4_READ(KARA_F32, 64);
  }
#undef KARA_Q4_READ
  return hip_status(hipGetLastError());
}

kara_status_t kara_q4_attention_workspace_size(const kara_params_t* p, int32_t n, int32_t n_layers, int32_t n_query,
                                               int32_t max_len, size_t* bytes) {
  Geom g;
  const kara_status_t st = make_geom(p, n, &g);
  if (st != KARA_OK) return st;
  if (!bytes || !layers_ok(n, n_layers) || n_query < 1 || max_len < 1 || (int64_t)max_len > (int64_t)g.max_blocks * g.bs ||
      (int64_t)n_query * g.Hq > INT32_MAX / 4)
    return KARA_ERR_INVALID_ARG;
  if (max_len > kMaxLen) return KARA_ERR_UNSUPPORTED;
  const size_t rec = (g.d + 2) * sizeof(float);
  const int64_t rows = (int64_t)n_layers * n * n_query * g.Hq;
  if (few_rows(g, n_query)) {
    const int64_t n_splits = (max_len + kSplitMin - 1) / kSplitMin;
    *bytes = n_splits == 1 ? 0 : (size_t)(rows * n_splits) * rec;
  } else {
    // (a launch that splits its keys has so many workgroups at most, records and all)
    const Q4ChunkPlan x = q4_chunk_plan(g, n, n_layers, n_query, max_len);
    *bytes = (size_t)kQ4ChunkWgs * x.qt * 128 * rec;
  }
  return KARA_OK;
}

kara_status_t kara_q4_attention(const kara_params_t* p, int32_t n, const int32_t* seqs, int32_t n_layers,
                                int32_t n_query, const void* q, const void* const* k_pools, const void* const* v_pools,
                                const void* const* k_scales, const void* const* v_scales, const int32_t* block_table,
                                const int32_t* seq_lens, int32_t max_len, void* out, void* workspace,
                                size_t workspace_bytes, void* stream) {
  size_t need = 0;
  kara_status_t st = kara_q4_attention_workspace_size(p, n, n_layers, n_query, max_len, &need);
  if (st != KARA_OK) return st;
  if (n == 0) return KARA_OK;
  if (!seqs || !q || !block_table || !seq_lens || !out || !pools_ok(k_pools, n_layers) || !pools_ok(v_pools, n_layers) ||
      !pools_ok(k_scales, n_layers) || !pools_ok(v_scales, n_layers))
    return KARA_ERR_INVALID_ARG;
  if (need && (!workspace || workspace_bytes < need)) return KARA_ERR_WORKSPACE;
  Q4Split a{};
  st = make_geom(p, n, &a.g);
  if (st != KARA_OK) return st;
  const Geom& g = a.g;
  if (!aligned(16, {q, out, need ? workspace : nullptr}) || !aligned(4, {seqs, block_table, seq_lens}) ||
      !cache_aligned(g, n_layers, k_pools, v_pools, k_scales, v_scales, nullptr))
    return KARA_ERR_INVALID_ARG;
  a.n = n;
  a.n_layers = n_layers;
  a.T = n_query;
  const bool few = few_rows(g, n_query);
  const int64_t rows = (int64_t)n_layers * n * n_query * g.Hq;
  Q4ChunkPlan plan{};
  if (few) {
    a.n_rt = (int)(((int64_t)g.G * n_query + 15) / 16);
    const int64_t units = (int64_t)n_layers * n * g.Hkv * a.n_rt;
    a.split_keys = split_keys_of(g.bs, units, max_len);
    a.n_splits = (max_len + a.split_keys - 1) / a.split_keys;
    if (!grid_ok(units * a.n_splits)) return KARA_ERR_UNSUPPORTED;
  } else {
    plan = q4_chunk_plan(g, n, n_layers, n_query, max_len);
    a.n_rt = plan.n_rb;
    a.split_keys = plan.split_keys;
    a.n_splits = plan.splits;
    if (!grid_ok(2 * plan.blocks)) return KARA_ERR_UNSUPPORTED;
  }
  if (!grid_ok((rows + 3) / 4)) return KARA_ERR_UNSUPPORTED;
  a.max_len = max_len;
  a.seqs = seqs;
  a.bt = block_table;
  a.seq_lens = seq_lens;
  a.q = q;
  a.kp = ptrs(k_pools, n_layers);
  a.vp = ptrs(v_pools, n_layers);
  a.ksp = ptrs(k_scales, n_layers);
  a.vsp = ptrs(v_scales, n_layers);
  a.rec_o = (float*)workspace;
  a.rec_ml = a.rec_o + rows * a.n_splits * g.d;
  a.out = out;
  a.out_bf16 = g.dtype == KARA_BF16;
  const hipError_t e = few ? launch_q4_split(a, false, (hipStream_t)stream) : launch_q4_chunk(a, plan, (hipStream_t)stream);
  if (e != hipSuccess || a.n_splits == 1) return hip_status(e);
  const dim3 grid((unsigned)((rows + 3) / 4));
  if (g.d == 128)
    hipLaunchKernelGGL((q4_combine_kernel<128>), grid, dim3(256), 0, (hipStream_t)stream, g, n, n_query, seqs, seq_lens,
                       max_len, a.split_keys, a.n_splits, rows, (const float*)a.rec_ml, (const float*)a.rec_o, out,
                       (int)a.out_bf16, (int)!few);
  else
    hipLaunchKernelGGL((q4_combine_kernel<64>), grid, dim3(256), 0, (hipStream_t)stream, g, n, n_query, seqs, seq_lens,
                       max_len, a.split_keys, a.n_splits, rows, (const float*)a.rec_ml, (const float*)a.rec_o, out,
                       (int)a.out_bf16, (int)!few);
  return hip_status(hipGetLastError());
}

}  // extern "C"

// Eviction by accumulated attention weight (include/kara_evict.h): decoding
// attention that counts each key's weight, selection by those counts, and the
// cut of the cache in place.
#include <algorithm>

#include "kara_evict.h"
#include "kara_harness.h"
#include "kara_internal.h"
#include "kara_page_check.h"

namespace kara {
namespace {

typedef uint32_t u32x4 __attribute__((ext_vector_type(4)));
typedef float floatx4 __attribute__((ext_vector_type(4)));

constexpr float kLog2e = 1.4426950408889634f;
constexpr float kMaxFloor = -3.402823466e38f;
constexpr int kMaxGroup = KARA_HARNESS_MAX_GROUP;

// a grid of one dimension, of 256 threads a block: HIP counts its threads in 32 bits
bool grid_ok(int64_t blocks) { return blocks > 0 && blocks < ((int64_t)1 << 24); }
size_t align256(size_t v) { return (v + 255) & ~(size_t)255; }

struct WeightPtrs {
  float* p[kMaxLayersPerLaunch];
};

// ---------------------------------------------------------------- attention that counts

constexpr int kFinThreads = 256;
constexpr int kFinKeys = 4 * kFinThreads;   // keys per step

// Second half of a counting decoding step: the splits' records joined to the
// output (a record: maximum and sum, ml_step apart, and o, o_step apart), and every
// key's weight -- exp2(logit - M) / L over the group's query heads -- added to its
// accumulator.  One workgroup per (layer, sequence, KV head, `steps` runs of 1024
// keys); a sequence's workgroups share out its query heads' outputs.  64 sequences of
// 4-8.2K tokens, 2 layers, 40/8 heads: 49 us for 165 MB, 3.4 TB/s (accumulators come
// in pieces of a page's 16 tokens).
template <int D>
__global__ __launch_bounds__(kFinThreads) void evict_finish_kernel(
    Geom g, int n, const int32_t* __restrict__ seqs, const int32_t* __restrict__ bt, const int32_t* __restrict__ seq_lens,
    int n_new, int max_len, int split_keys, int n_splits, int chunks, int steps, const float* __restrict__ rec_ml, int ml_step,
    const float* __restrict__ rec_o, int o_step, const float* __restrict__ logits, int64_t ld, WeightPtrs wp, float* __restrict__ out) {
  __shared__ float red_m[kMaxGroup], red_i[kMaxGroup];
  const int tid = threadIdx.x, lane = tid & 63, wave = tid >> 6;
  uint32_t rest = blockIdx.x;
  const int chunk = rest % (uint32_t)chunks;
  rest /= (uint32_t)chunks;
  const int h = rest % (uint32_t)g.Hkv;
  rest /= (uint32_t)g.Hkv;
  const int j = rest % (uint32_t)n;
  const int l = rest / (uint32_t)n;
  const int s = seqs[j], G = g.G;
  const int64_t orow = ((int64_t)l * n + j) * g.Hq + h * G;
  const int len = s >= 0 && s < g.n_seqs ? seq_lens[s] : 0;
  if (len <= 0 || len > max_len) {
    if (chunk == 0)
      for (int i = tid; i < G * D; i += kFinThreads) out[orow * D + i] = 0.f;
    return;
  }
  const int k0 = chunk * steps * kFinKeys;
  if (k0 >= len) return;
  const int ns = (len + split_keys - 1) / split_keys;
  const int nc = (len + steps * kFinKeys - 1) / (steps * kFinKeys);      // this sequence's workgroups
  int dup = 0;
  for (int o = tid; o < j; o += kFinThreads) dup |= seqs[o] == s;
  for (int i = wave; i < G; i += kFinThreads / 64) {
    const float* w = rec_ml + (orow + i) * n_splits * ml_step;
    float M = kMaxFloor, L = 0.f;
    for (int sp = lane; sp < ns; sp += 64) M = fmaxf(M, w[(int64_t)sp * ml_step]);
#pragma unroll
    for (int x = 1; x < 64; x <<= 1) M = fmaxf(M, __shfl_xor(M, x, 64));
    for (int sp = lane; sp < ns; sp += 64) 
      L += w[(int64_t)sp * ml_step + 1] * __builtin_amdgcn_exp2f(w[(int64_t)sp * ml_step] - M);
#pragma unroll
    for (int x = 1; x < 64; x <<= 1) L += __shfl_xor(L, x, 64);
    if (lane == 0) red_m[i] = M, red_i[i] = L == 0.f ? 0.f : 1.f / L;     // (0: every logit is -inf)
  }
  dup = __syncthreads_or(dup);
  for (int i = chunk; i < G; i += nc) {
    const float* w = rec_ml + (orow + i) * n_splits * ml_step;
    const float* o = rec_o + (orow + i) * n_splits * o_step;
    for (int e = tid; e < D; e += kFinThreads) {
      float acc = 0.f;
#pragma unroll 8
      for (int sp = 0; sp < ns; ++sp)
        acc += o[(int64_t)sp * o_step + e] * __builtin_amdgcn_exp2f(w[(int64_t)sp * ml_step] - red_m[i]);
      out[(orow + i) * D + e] = acc * red_i[i];
    }
  }
  if (dup) return;        // an earlier listing counts
  const float c = g.scale * kLog2e;
  const int32_t* row_pages = bt + (int64_t)s * g.max_blocks;
  for (int k = k0 + 4 * tid; k < min(len, k0 + steps * kFinKeys); k += kFinKeys) {
    // four keys; in one page and on 16 bytes where pages allow it
    const bool quad = (g.bs & 3) == 0;
    floatx4* to = nullptr;
    floatx4 was = {0.f, 0.f, 0.f, 0.f};
    if (quad) {
      const int b = k / g.bs;
      const int page = row_pages[b];
      if (page < 0 || page >= g.num_pages) continue;
      to = (floatx4*)(wp.p[l] + ((int64_t)page * g.Hkv + h) * g.bs + (k - b * g.bs));
      was = *to;
    }
    float add[4] = {0.f, 0.f, 0.f, 0.f};
    for (int i0 = 0; i0 < G; i0 += 4) {
      floatx4 x[4];
#pragma unroll
      for (int y = 0; y < 4; ++y) x[y] = *(const floatx4*)(logits + (orow + min(i0 + y, G - 1)) * ld + k);
#pragma unroll
      for (int y = 0; y < 4; ++y) {
        if (i0 + y >= G) break;
#pragma unroll
        for (int e = 0; e < 4; ++e)
          add[e] = fmaf(__builtin_amdgcn_exp2f(fmaf(x[y][e], c, -red_m[i0 + y])), red_i[i0 + y], add[e]);
      }
    }
    if (quad) {
      floatx4 now;
#pragma unroll
      for (int e = 0; e < 4; ++e) now[e] = k + e >= len ? was[e] : k + e >= len - n_new ? add[e] : was[e] + add[e];
      *to = now;
      continue;
    }
#pragma unroll
    for (int e = 0; e < 4; ++e) {
      const int pos = k + e;
      if (pos >= len) break;
      const int b = pos / g.bs;
      const int page = row_pages[b];
      if (page < 0 || page >= g.num_pages) continue;
      float* one = wp.p[l] + ((int64_t)page * g.Hkv + h) * g.bs + (pos - b * g.bs);
      *one = pos >= len - n_new ? add[e] : *one + add[e];
    }
  }
}

// ---------------------------------------------------------------- the cut

struct EvictArgs {
  Geom g;
  int n, n_layers, keep, n_sink, n_recent, max_len;
  int commit;
  const int32_t *seqs, *bt, *seq_lens;
  int32_t *kept, *status;
  int32_t *freed, *n_freed;   // commit: pages released (each listing's blocks past the cut)
  int32_t* old_len;           // [n] lengths before the cut, 0 where there is none
  PoolPtrs k, v, ks, vs;      // rows or codes; scales (null: rows)
  WeightPtrs w;
  int row_bytes;              // of k and v
  int scale_bytes;            // of ks and vs; 0: none
  int cols;                   // pieces that the move cuts a row into
};

// What the last launch writes where the call commits: no earlier one can change a
// table or a length, so a call that fails between them leaves sequences as they were.
struct EvictCommit {
  int32_t *bt, *seq_lens;
};

// Pages of a listed sequence as they were before the cut: while rows move, one
// workgroup takes those past it out of the table, and the others read them in `freed`.
struct Pages {
  const int32_t *row, *tail;
  int first_tail;
  __device__ __forceinline__ Pages(const EvictArgs& a, int j, int s)
      : row(a.bt + (int64_t)s * a.g.max_blocks),
        tail(a.freed + (int64_t)j * a.g.max_blocks),
        first_tail(a.commit ? (a.keep + a.g.bs - 1) / a.g.bs : a.g.max_blocks) {}
  __device__ __forceinline__ int operator[](int b) const { return *(b < first_tail ? row + b : tail + (b - first_tail)); }
};

// One workgroup per listed sequence: its status, its length in old_len (0: left
// alone) and, where the call commits, its pages past the cut in `freed`.
__global__ __launch_bounds__(kValidateThreads) void evict_validate_kernel(EvictArgs a) {
  __shared__ uint32_t lds[kValidateLds];
  const Geom& g = a.g;
  const int j = blockIdx.x, tid = threadIdx.x;
  const int s = a.seqs[j];
  int st = KARA_SEQ_BAD_INDEX, len = 0;
  if (s >= 0 && s < g.n_seqs) {
    int dup = 0;
    for (int o = tid; o < a.n; o += kValidateThreads) dup |= o != j && a.seqs[o] == s;
    st = __syncthreads_or(dup) ? KARA_SEQ_DUP_TRIGGER : 0;
    len = a.seq_lens[s];
    if (len < 0 || len > a.max_len || (int64_t)len > (int64_t)g.max_blocks * g.bs)
      st |= KARA_SEQ_BAD_WINDOW;
    else
      st |= pages_status(a.bt + (int64_t)s * g.max_blocks, 0, (len + g.bs - 1) / g.bs, g.num_pages, lds);
  }
  if (st != 0) len = 0;
  if (tid == 0) {
    a.status[j] = st;
    a.old_len[j] = len;
  }
  if (!a.commit) return;
  const int old_b = (len + g.bs - 1) / g.bs, new_b = (min(len, a.keep) + g.bs - 1) / g.bs;
  const int32_t* row = a.bt + (int64_t)(st == 0 ? s : 0) * g.max_blocks;
  int32_t* fr = a.freed + (int64_t)j * g.max_blocks;
  for (int c = tid; c < g.max_blocks; c += kValidateThreads) fr[c] = c < old_b - new_b ? row[new_b + c] : -1;
  if (tid == 0) a.n_freed[j] = 0;        // (until the pages are released)
}

constexpr int kPickThreads = 512;
constexpr int kPickWaves = kPickThreads / 64;
constexpr int kPickLds = 16384;      // keys held in LDS; a longer row is read again in each pass
constexpr int kPickBits = 11;        // of a digit
constexpr int kPickBins = 1 << kPickBits;

// Order-preserving: a larger weight has the larger key, -0 ranks as 0, NaN below all.
__device__ __forceinline__ uint32_t weight_key(float f) {
  uint32_t u = __float_as_uint(f);
  if ((u & 0x7fffffffu) > 0x7f800000u) return 0;
  if ((u & 0x7fffffffu) == 0) u = 0;
  return (u & 0x80000000u) ? ~u : (u | 0x80000000u);
}

// One workgroup per (layer, sequence, KV head): the positions that stay.  A
// radix selection over the accumulators between the first n_sink and the last
// n_recent positions finds the key of the last one taken and how many equal
// ones are; then every wave writes its part of the sequence in order.  Digits of 11
// bits are taken from the keys' offset above the smallest, from its highest bit on:
// accumulated weights share their exponents, and digits cut from the keys
// themselves would meet in a handful of bins.
__global__ __launch_bounds__(kPickThreads) void evict_pick_kernel(EvictArgs a) {
  extern __shared__ __attribute__((aligned(16))) uint32_t keys[];
  __shared__ __attribute__((aligned(16))) uint32_t hist[kPickBins];
  __shared__ uint32_t found[3];                        // digit, items wanted in its bin, items in it
  __shared__ uint32_t wave_a[kPickWaves], wave_b[kPickWaves];
  const Geom& g = a.g;
  const int tid = threadIdx.x, lane = tid & 63, wave = tid >> 6;
  uint32_t rest = blockIdx.x;
  const int h = rest % (uint32_t)g.Hkv;
  rest /= (uint32_t)g.Hkv;
  const int j = rest % (uint32_t)a.n, l = rest / (uint32_t)a.n;
  int32_t* kept = a.kept + (int64_t)blockIdx.x * a.keep;
  const int len = a.old_len[j];
  if (len <= a.keep) {
    for (int i = tid; i < a.keep; i += kPickThreads) kept[i] = i < len ? i : -1;
    return;
  }
  const Pages pages(a, j, a.seqs[j]);
  const float* w = a.w.p[l];
  const int lo = a.n_sink, hi = len - a.n_recent;      // candidates
  const uint32_t want = (uint32_t)(a.keep - a.n_sink - a.n_recent);
  auto fetch = [&](int pos) __attribute__((always_inline)) {
    const int b = pos / g.bs;
    return weight_key(w[((int64_t)pages[b] * g.Hkv + h) * g.bs + (pos - b * g.bs)]);
  };
  const bool in_lds = len <= kPickLds;
  uint32_t kmin = ~0u, kmax = 0;
  if (in_lds && (g.bs & 3) == 0) {
    // four keys lie in one page, on 16 bytes
    for (int i = 4 * tid; i < len; i += 4 * kPickThreads) {
      const int b = i / g.bs;
      const floatx4 f = *(const floatx4*)(w + ((int64_t)pages[b] * g.Hkv + h) * g.bs + (i - b * g.bs));
      u32x4 k;
#pragma unroll
      for (int e = 0; e < 4; ++e) {
        k[e] = weight_key(f[e]);
        if (i + e >= lo && i + e < hi) kmin = min(kmin, k[e]), kmax = max(kmax, k[e]);
      }
      *(u32x4*)(keys + i) = k;           // (up to three past the length)
    }
  } else {
    for (int i = tid; i < len; i += kPickThreads) {
      const uint32_t k = fetch(i);
      if (i >= lo && i < hi) kmin = min(kmin, k), kmax = max(kmax, k);
      if (in_lds) keys[i] = k;
    }
  }
#pragma unroll
  for (int x = 1; x < 64; x <<= 1) {
    kmin = min(kmin, (uint32_t)__shfl_xor((int)kmin, x, 64));
    kmax = max(kmax, (uint32_t)__shfl_xor((int)kmax, x, 64));
  }
  if (lane == 0) wave_a[wave] = kmin, wave_b[wave] = kmax;
  *(u32x4*)&hist[4 * tid] = u32x4{0, 0, 0, 0};
  static_assert(kPickBins == 4 * kPickThreads, "four bins a thread");
  __syncthreads();
#pragma unroll
  for (int x = 0; x < kPickWaves; ++x) kmin = min(kmin, wave_a[x]), kmax = max(kmax, wave_b[x]);
  // the key's offset above the smallest of the candidates
  auto key = [&](int pos) __attribute__((always_inline)) { return (in_lds ? keys[pos] : fetch(pos)) - kmin; };

  // the last one taken is `prefix` above kmin (with the digits below `shift` open
  // where its bin is taken whole), `need` of the equal ones
  uint32_t prefix = 0, need = want;
  int shift = kmax > kmin ? 32 - __builtin_clz(kmax - kmin) : 0;
  bool first = true;
  while (shift > 0 && need > 0) {
    const int above_shift = shift;
    shift = max(0, shift - kPickBits);
    const uint32_t mask = (1u << (above_shift - shift)) - 1u;
    for (int i = lo + tid; i < hi; i += kPickThreads) {
      const uint32_t k = key(i);
      if (first || ((k ^ prefix) >> above_shift) == 0) atomicAdd(&hist[(k >> shift) & mask], 1u);
    }
    __syncthreads();
    // bins from the largest: thread i holds kPickBins - 1 - 4i and the three below
    const u32x4 c4 = *(const u32x4*)&hist[kPickBins - 4 - 4 * tid];
    const uint32_t c[4] = {c4[3], c4[2], c4[1], c4[0]};
    const uint32_t tot = c[0] + c[1] + c[2] + c[3];
    uint32_t above = tot;
#pragma unroll
    for (int x = 1; x < 64; x <<= 1) {
      const uint32_t up = (uint32_t)__shfl_up((int)above, x, 64);
      if (lane >= x) above += up;
    }
    if (lane == 63) wave_a[wave] = above;
    above -= tot;
    __syncthreads();
    for (int x = 0; x < wave; ++x) above += wave_a[x];
    *(u32x4*)&hist[kPickBins - 4 - 4 * tid] = u32x4{0, 0, 0, 0};
#pragma unroll
    for (int e = 0; e < 4; ++e) {
      if (above < need && need <= above + c[e]) found[0] = kPickBins - 1 - 4 * tid - e, found[1] = need - above, found[2] = c[e];
      above += c[e];
    }
    __syncthreads();
    prefix |= found[0] << shift;
    need = found[1];
    first = false;
    if (found[1] == found[2]) break;
    __syncthreads();                     // (found is read before the next pass writes it)
  }
  // taken: keys above the prefix, and of those equal to it (in the digits that were
  // looked at) the first `need`
  const uint32_t edge = prefix >> shift;
  const bool any = want > 0;
  const int per = ((len + kPickWaves * 64 - 1) / (kPickWaves * 64)) * 64;     // positions per wave
  const int w0 = min(wave * per, len), w1 = min(w0 + per, len);
  auto rank = [&](int pos) __attribute__((always_inline)) {                   // 2: stays, 1: stays if among the first
    if (pos >= w1) return 0;
    if (pos < lo || pos >= hi) return 2;
    if (!any) return 0;
    const uint32_t k = key(pos) >> shift;
    return k > edge ? 2 : k == edge ? 1 : 0;
  };
  uint32_t gt = 0, eq = 0;
  for (int i = w0; i < w1; i += 64) {
    const int r = rank(i + lane);
    gt += (uint32_t)__popcll(__ballot(r == 2));
    eq += (uint32_t)__popcll(__ballot(r == 1));
  }
  __syncthreads();                       // (wave_a is free)
  if (lane == 0) wave_a[wave] = gt, wave_b[wave] = eq;
  __syncthreads();
  uint32_t at = 0, eq_at = 0;          // taken, and equal ones, before this wave's part
  for (int x = 0; x < wave; ++x) {
    at += wave_a[x];
    eq_at += wave_b[x];
  }
  at += min(eq_at, need);
  const uint64_t below = ((uint64_t)1 << lane) - 1;
  for (int i = w0; i < w1; i += 64) {
    const int r = rank(i + lane);
    const uint64_t e = __ballot(r == 1);
    const bool stays = r == 2 || (r == 1 && eq_at + (uint32_t)__popcll(e & below) < need);
    const uint64_t b = __ballot(stays);
    if (stays) kept[at + (uint32_t)__popcll(b & below)] = i + lane;
    at += (uint32_t)__popcll(b);
    eq_at += (uint32_t)__popcll(e);
  }
}

constexpr int kMoveThreads = 1024;
constexpr int kMoveUnroll = 8;
constexpr int kMoveStage = 65536 / 4;     // rows held in LDS, at most

// One workgroup per (layer, sequence, KV head, part): a piece of the K rows or of the V
// rows, or the small arrays (scales, accumulators).  Row i takes row kept[i] >= i, so working up in
// tiles -- a tile's rows all loaded before any of it is stored -- never overwrites
// a row still to be read.  Wide rows are cut into pieces, a workgroup each.  Bound by
// the bytes: 64 sequences x 4 layers cut from 3.9-8.2K to 3.8K tokens (8.1 GB) in
// 1576 us, 5.1 TB/s.  1024 threads a workgroup: that cut was 2 % slower with 256; 8
// sequences of one layer, where a tile's latency is all that the launch spends, took
// 36 us with 256, 24 so.  The workgroup of a sequence's first small arrays commits.
template <bool STAGED>
__global__ __launch_bounds__(kMoveThreads) void evict_move_kernel(EvictArgs a, EvictCommit out) {
  extern __shared__ uint32_t stage[];
  const Geom& g = a.g;
  const int tid = threadIdx.x;
  const int parts = 2 * a.cols + 1, part = blockIdx.x % (uint32_t)parts;
  const uint32_t u = blockIdx.x / (uint32_t)parts;
  uint32_t rest = u;
  const int h = rest % (uint32_t)g.Hkv;
  rest /= (uint32_t)g.Hkv;
  const int j = rest % (uint32_t)a.n, l = rest / (uint32_t)a.n;
  const int len = a.old_len[j];
  if (len <= a.keep) return;
  const int32_t* kept = a.kept + (int64_t)u * a.keep;
  const Pages pages(a, j, a.seqs[j]);
  auto row = [&](int pos) __attribute__((always_inline)) {
    const int b = pos / g.bs;
    return ((uint32_t)pages[b] * g.Hkv + h) * g.bs + (pos - b * g.bs);    // (a pool has fewer than 2^32 rows)
  };
  // pool rows that row i comes from and goes to
  if constexpr (STAGED) {
    for (int i = tid; i < a.keep; i += kMoveThreads) {
      stage[i] = row(kept[i]);
      stage[a.keep + i] = row(i);
    }
    __syncthreads();
  }
  auto source = [&](int i) __attribute__((always_inline)) { return STAGED ? stage[i] : row(kept[i]); };
  auto target = [&](int i) __attribute__((always_inline)) { return STAGED ? stage[a.keep + i] : row(i); };
  if (part < 2 * a.cols) {
    const int piece = a.row_bytes / a.cols;
    char* base = (char*)(part & 1 ? a.v.p[l] : a.k.p[l]) + (part >> 1) * piece;
    const int cpr = piece >> 4, rpp = kMoveThreads / cpr, tile = rpp * kMoveUnroll;
    const int c = tid % cpr, r = tid / cpr;
    for (int x0 = 0; x0 < a.keep; x0 += tile) {
      u32x4 v[kMoveUnroll];
      uint32_t dst[kMoveUnroll];
      bool moves[kMoveUnroll];
#pragma unroll
      for (int k = 0; k < kMoveUnroll; ++k) {
        const int i = x0 + k * rpp + r;
        moves[k] = false;
        if (i < a.keep) {
          const uint32_t src = source(i);
          dst[k] = target(i);
          moves[k] = src != dst[k];
          if (moves[k]) v[k] = __builtin_nontemporal_load((const u32x4*)(base + (uint64_t)src * a.row_bytes + c * 16));
        }
      }
      // all of this tile's loads have landed before any thread stores
      asm volatile("s_waitcnt vmcnt(0)" ::: "memory");
      __syncthreads();
#pragma unroll
      for (int k = 0; k < kMoveUnroll; ++k)
        if (moves[k]) __builtin_nontemporal_store(v[k], (u32x4*)(base + (uint64_t)dst[k] * a.row_bytes + c * 16));
    }
    return;
  }
  constexpr int kRows = 4;               // of a thread and tile
  for (int x0 = 0; x0 < a.keep; x0 += kMoveThreads * kRows) {
    float w[kRows];
    uint32_t sk[kRows], sv[kRows];
    uint32_t to[kRows];
    bool moves[kRows];
#pragma unroll
    for (int k = 0; k < kRows; ++k) {
      const int i = x0 + k * kMoveThreads + tid;
      moves[k] = false;
      if (i >= a.keep) continue;
      const uint32_t from = source(i);
      to[k] = target(i);
      moves[k] = from != to[k];
      if (!moves[k]) continue;
      w[k] = a.w.p[l][from];
      if (a.scale_bytes == 4) {
        sk[k] = ((const uint32_t*)a.ks.p[l])[from];
        sv[k] = ((const uint32_t*)a.vs.p[l])[from];
      } else if (a.scale_bytes == 2) {
        sk[k] = ((const uint16_t*)a.ks.p[l])[from];
        sv[k] = ((const uint16_t*)a.vs.p[l])[from];
      }
    }
    asm volatile("s_waitcnt vmcnt(0)" ::: "memory");
    __syncthreads();
#pragma unroll
    for (int k = 0; k < kRows; ++k) {
      if (!moves[k]) continue;
      a.w.p[l][to[k]] = w[k];
      if (a.scale_bytes == 4) {
        ((uint32_t*)a.ks.p[l])[to[k]] = sk[k];
        ((uint32_t*)a.vs.p[l])[to[k]] = sv[k];
      } else if (a.scale_bytes == 2) {
        ((uint16_t*)a.ks.p[l])[to[k]] = (uint16_t)sk[k];
        ((uint16_t*)a.vs.p[l])[to[k]] = (uint16_t)sv[k];
      }
    }
  }
  if (a.commit && l == 0 && h == 0) {
    // blocks past the cut and the length: no workgroup of this launch reads them here
    const int s = a.seqs[j];
    const int old_b = (len + g.bs - 1) / g.bs, new_b = (a.keep + g.bs - 1) / g.bs;
    for (int b = new_b + tid; b < old_b; b += kMoveThreads) out.bt[(int64_t)s * g.max_blocks + b] = -1;
    if (tid == 0) {
      a.n_freed[j] = old_b - new_b;
      out.seq_lens[s] = a.keep;
    }
  }
}

bool layers_ok(int32_t n, int32_t n_layers) { return n >= 0 && n_layers >= 1 && n_layers <= kMaxLayersPerLaunch; }

PoolPtrs ptrs(const void* const* pools, int n_layers) {
  PoolPtrs x{};
  if (pools)
    for (int i = 0; i < n_layers; ++i) x.p[i] = const_cast<void*>(pools[i]);
  return x;
}

WeightPtrs weight_ptrs(float* const* w, int n_layers) {
  WeightPtrs x{};
  for (int i = 0; i < n_layers; ++i) x.p[i] = w[i];
  return x;
}

// both scale arrays or neither
bool scales_ok(const void* const* ks, const void* const* vs, int n_layers) {
  return (!ks && !vs) || (pools_ok(ks, n_layers) && pools_ok(vs, n_layers));
}

struct CountWs {
  size_t records, logits, total;
  int64_t ld;
};

CountWs count_ws(const Geom& g, int n, int n_layers, int max_len) {
  const int64_t rows = (int64_t)n_layers * n * g.Hq;
  const int64_t splits = (max_len + KARA_HARNESS_SPLIT_KEYS - 1) / KARA_HARNESS_SPLIT_KEYS;
  CountWs w{};
  w.ld = (max_len + 31) / 32 * 32;       // (the splits write whole blocks of up to 32 keys)
  w.logits = align256((size_t)(rows * splits * (g.d + 2)) * sizeof(float));
  w.total = align256(w.logits + (size_t)(rows * w.ld) * sizeof(float));
  return w;
}

}  // namespace
}  // namespace kara

using namespace kara;

extern "C" {

kara_status_t kara_evict_attention_workspace_size(const kara_params_t* p, int32_t n, int32_t n_layers, int32_t max_len,
                                                  size_t* bytes) {
  Geom g;
  const kara_status_t st = make_geom(p, n, &g);
  if (st != KARA_OK) return st;
  if (g.G > kMaxGroup) return KARA_ERR_UNSUPPORTED;
  if (!bytes || !layers_ok(n, n_layers) || max_len < 1 || (int64_t)max_len > (int64_t)g.max_blocks * g.bs)
    return KARA_ERR_INVALID_ARG;
  if (max_len > kMaxLen) return KARA_ERR_UNSUPPORTED;
  *bytes = count_ws(g, n, n_layers, max_len).total;
  return KARA_OK;
}

kara_status_t kara_evict_attention(const kara_params_t* p, int32_t n, const int32_t* seqs, int32_t n_layers,
                                   const void* q, const void* const* k_pools, const void* const* v_pools,
                                   const void* const* k_scales, const void* const* v_scales, float* const* weights,
                                   const int32_t* block_table, const int32_t* seq_lens, int32_t n_new, int32_t max_len,
                                   float* out, void* workspace, size_t workspace_bytes, void* stream) {
  size_t need = 0;
  kara_status_t st = kara_evict_attention_workspace_size(p, n, n_layers, max_len, &need);
  if (st != KARA_OK) return st;
  if (n_new < 0) return KARA_ERR_INVALID_ARG;
  if (n == 0) return KARA_OK;
  if (!seqs || !q || !block_table || !seq_lens || !out || !pools_ok(k_pools, n_layers) || !pools_ok(v_pools, n_layers) ||
      !scales_ok(k_scales, v_scales, n_layers) || !pools_ok((const void* const*)weights, n_layers))
    return KARA_ERR_INVALID_ARG;
  if (!workspace || workspace_bytes < need) return KARA_ERR_WORKSPACE;
  Geom g;
  st = make_geom(p, n, &g);
  if (st != KARA_OK) return st;
  if (!aligned(16, {q, out, workspace}) || !aligned(4, {seqs, block_table, seq_lens}) ||
      !cache_aligned(g, n_layers, k_pools, v_pools, k_scales, v_scales, (const void* const*)weights))
    return KARA_ERR_INVALID_ARG;
  const CountWs w = count_ws(g, n, n_layers, max_len);
  float* records = (float*)workspace;
  float* logits = (float*)((char*)workspace + w.logits);
  const int64_t units = (int64_t)n_layers * n * g.Hkv;
  // (more keys a workgroup where 8 per CU remain)
  int steps = 1;
  while (steps < 4 && units * ((max_len + 2 * steps * kFinKeys - 1) / (2 * steps * kFinKeys)) >= 2048) steps *= 2;
  const int chunks = (max_len + steps * kFinKeys - 1) / (steps * kFinKeys);
  if (!grid_ok(units * ((max_len + KARA_HARNESS_SPLIT_KEYS - 1) / KARA_HARNESS_SPLIT_KEYS))) return KARA_ERR_UNSUPPORTED;
  hipStream_t s = (hipStream_t)stream;
  const PoolPtrs kp = ptrs(k_pools, n_layers), vp = ptrs(v_pools, n_layers);
  int keys = 0;
  hipError_t e;
  if (k_scales) {
    Q4Split a{};
    a.g = g;
    a.n = n;
    a.n_layers = n_layers;
    a.T = 1;
    a.n_rt = 1;
    a.split_keys = keys = q4_split_keys(g, units, max_len);
    a.n_splits = (max_len + keys - 1) / keys;
    a.max_len = max_len;
    a.seqs = seqs;
    a.bt = block_table;
    a.seq_lens = seq_lens;
    a.q = q;
    a.kp = kp;
    a.vp = vp;
    a.ksp = ptrs(k_scales, n_layers);
    a.vsp = ptrs(v_scales, n_layers);
    a.rec_o = records;
    a.rec_ml = records + (int64_t)n_layers * n * g.Hq * a.n_splits * g.d;
    a.logits = logits;
    a.ld = w.ld;
    e = launch_q4_split(a, true, s);
  } else {
    e = launch_decode_logits(g, n, seqs, n_layers, q, kp, vp, block_table, seq_lens, max_len, records, logits, w.ld, &keys, s);
  }
  if (e != hipSuccess) return hip_status(e);
  const int n_splits = (max_len + keys - 1) / keys;
  // rows' records are m, l, o[d]; 4-bit ones hold o and m, l apart
  const float* rec_o = k_scales ? records : records + 2;
  const float* rec_ml = k_scales ? records + (int64_t)n_layers * n * g.Hq * n_splits * g.d : records;
  const int o_step = k_scales ? g.d : g.d + 2, ml_step = k_scales ? 2 : g.d + 2;
  const dim3 grid((unsigned)(units * chunks)), block(kFinThreads);
  if (g.d == 128)
    hipLaunchKernelGGL((evict_finish_kernel<128>), grid, block, 0, s, g, n, seqs, block_table, seq_lens, n_new, max_len, keys,
                       n_splits, chunks, steps, rec_ml, ml_step, rec_o, o_step, (const float*)logits, w.ld, weight_ptrs(weights, n_layers), out);
  else
    hipLaunchKernelGGL((evict_finish_kernel<64>), grid, block, 0, s, g, n, seqs, block_table, seq_lens, n_new, max_len, keys,
                       n_splits, chunks, steps, rec_ml, ml_step, rec_o, o_step, (const float*)logits, w.ld, weight_ptrs(weights, n_layers), out);
  return hip_status(hipGetLastError());
}

kara_status_t kara_evict_workspace_size(const kara_params_t* p, int32_t n, int32_t n_layers, int32_t keep, size_t* bytes) {
  Geom g;
  const kara_status_t st = make_geom(p, n, &g);
  if (st != KARA_OK) return st;
  if (!bytes || !layers_ok(n, n_layers) || keep < 1) return KARA_ERR_INVALID_ARG;
  if (keep > kMaxLen) return KARA_ERR_UNSUPPORTED;      // (positions step in 32 bits)
  *bytes = align256((size_t)n * sizeof(int32_t)) + (size_t)n_layers * n * g.Hkv * keep * sizeof(int32_t);
  return KARA_OK;
}

kara_status_t kara_evict_tokens(const kara_params_t* p, int32_t n, const int32_t* seqs, int32_t n_layers, int32_t keep,
                                int32_t n_sink, int32_t n_recent, void* const* k_pools, void* const* v_pools,
                                void* const* k_scales, void* const* v_scales, float* const* weights,
                                int32_t* block_table, int32_t* seq_lens, int32_t max_len, int32_t commit, int32_t* kept,
                                int32_t* freed, int32_t* n_freed, int32_t* status, void* workspace,
                                size_t workspace_bytes, void* stream) {
  size_t need = 0;
  kara_status_t st = kara_evict_workspace_size(p, n, n_layers, keep, &need);
  if (st != KARA_OK) return st;
  EvictArgs a{};
  st = make_geom(p, n, &a.g);
  if (st != KARA_OK) return st;
  const Geom& g = a.g;
  if (n_sink < 0 || n_recent < 0 || (int64_t)n_sink + n_recent > keep || max_len < 1 ||
      (int64_t)max_len > (int64_t)g.max_blocks * g.bs)
    return KARA_ERR_INVALID_ARG;
  if (max_len > kMaxLen) return KARA_ERR_UNSUPPORTED;
  if (n == 0) return KARA_OK;
  if (!seqs || !block_table || !seq_lens || !status || !pools_ok(k_pools, n_layers) || !pools_ok(v_pools, n_layers) ||
      !scales_ok(k_scales, v_scales, n_layers) || !pools_ok((const void* const*)weights, n_layers) ||
      (commit && (!freed || !n_freed)))
    return KARA_ERR_INVALID_ARG;
  if (kept) need = (size_t)n * sizeof(int32_t);     // (the lengths alone)
  if (!workspace || workspace_bytes < need) return KARA_ERR_WORKSPACE;
  if (!aligned(16, {workspace}) || !aligned(4, {seqs, block_table, seq_lens, kept, freed, n_freed, status}) ||
      !cache_aligned(g, n_layers, k_pools, v_pools, k_scales, v_scales, (const void* const*)weights))
    return KARA_ERR_INVALID_ARG;
  const int64_t units = (int64_t)n_layers * n * g.Hkv;
  if (!grid_ok(units * 4 * (2 * 4 + 1))) return KARA_ERR_UNSUPPORTED;
  a.n = n;
  a.n_layers = n_layers;
  a.keep = keep;
  a.n_sink = n_sink;
  a.n_recent = n_recent;
  a.max_len = max_len;
  a.seqs = seqs;
  a.bt = block_table;
  a.seq_lens = seq_lens;
  a.commit = commit != 0;
  a.old_len = (int32_t*)workspace;
  a.kept = kept ? kept : (int32_t*)((char*)workspace + align256((size_t)n * sizeof(int32_t)));
  a.freed = commit ? freed : nullptr;
  a.n_freed = commit ? n_freed : nullptr;
  a.status = status;
  a.k = ptrs(k_pools, n_layers);
  a.v = ptrs(v_pools, n_layers);
  a.ks = ptrs(k_scales, n_layers);
  a.vs = ptrs(v_scales, n_layers);
  a.w = weight_ptrs(weights, n_layers);
  a.row_bytes = k_scales ? g.d / 2 : g.d * g.esize;
  a.scale_bytes = k_scales ? g.d / 32 : 0;
  hipStream_t s = (hipStream_t)stream;
  hipLaunchKernelGGL(evict_validate_kernel, dim3((unsigned)n), dim3(kValidateThreads), 0, s, a);
  hipError_t e = hipGetLastError();
  if (e != hipSuccess) return hip_status(e);
  const size_t pick_lds = (size_t)std::min((max_len + 3) / 4 * 4, kPickLds) * sizeof(uint32_t);
  hipLaunchKernelGGL(evict_pick_kernel, dim3((unsigned)units), dim3(kPickThreads), pick_lds, s, a);
  e = hipGetLastError();
  if (e != hipSuccess) return hip_status(e);
  const int64_t staged = 2 * (int64_t)keep;
  // Rows in pieces of 128 bytes, of 64 while the launch leaves CUs without a workgroup:
  // half as many tiles one after the other (8 sequences of one layer 24 -> 18.5 us, two
  // 12.7 -> 7.4; the large cut above 1589 -> 1576).
  a.cols = std::max(1, a.row_bytes / 128);
  while (units * 2 * a.cols < 256 && a.row_bytes / a.cols > 64) a.cols *= 2;
  const dim3 grid((unsigned)(units * (2 * a.cols + 1))), block(kMoveThreads);
  const EvictCommit out{block_table, seq_lens};
  if (staged <= kMoveStage) hipLaunchKernelGGL((evict_move_kernel<true>), grid, block, (size_t)staged * 4, s, a, out);
  else hipLaunchKernelGGL((evict_move_kernel<false>), grid, block, 0, s, a, out);
  return hip_status(hipGetLastError());
}

}  // extern "C"

// Tokens appended to the paged cache with the position rotation on the way, into rows
// or into 8 bits, and the 8-bit cache's plain append and reading back
// (include/kara_rope.h, include/kara_q8.h).
#include <algorithm>
#include <cmath>
#include <type_traits>

#include "kara_append.h"
#include "kara_call.h"
#include "kara_q8_device.h"
#include "kara_rope.h"

namespace kara {
namespace {

typedef uint32_t u32x4 __attribute__((ext_vector_type(4)));
typedef uint32_t u32x2 __attribute__((ext_vector_type(2)));

constexpr int kStoreThreads = 256;
constexpr int kFewThreads = 1024;
constexpr int kTile = 32;             // tokens that share a table of angles
constexpr int kGroupHeads = 16;       // KV heads of a workgroup, at most
constexpr int kStoreWgs = 1024;       // workgroups of a launch, where heads can be dealt out
constexpr int kMaxOctets = 1 << 22;   // of a token's heads: 32 tokens' items stay in 32 bits

struct StoreHead {
  Dims g;
  int n, n_new, n_layers, counted;
  int units;                          // runs of tokens per (layer, sequence)
  int group;                          // KV heads of a workgroup
  int half;                           // pairs that turn; 0: none
  double step;                        // frequencies: exp2(-step i) revolutions / 2 pi
  const float* inv_freq;
  const int32_t *seqs, *bt;
  int32_t *seq_lens, *rope_pos, *status;
  const char *q, *k_new, *v_new;
  char* q_out;
};
template <int NL>
struct Store : StoreHead {
  Pools<NL> kp, vp, ksp, vsp;
};

// Eight values as they lie in memory
template <int DT>
struct Raw {
  u32x4 v[DT == KARA_BF16 ? 1 : 2];
  __device__ __forceinline__ void load(const char* p) {
#pragma unroll
    for (int i = 0; i < (DT == KARA_BF16 ? 1 : 2); ++i) v[i] = __builtin_nontemporal_load((const u32x4*)p + i);
  }
  template <bool STREAM>
  __device__ __forceinline__ void store(char* p) const {
#pragma unroll
    for (int i = 0; i < (DT == KARA_BF16 ? 1 : 2); ++i) {
      if constexpr (STREAM) __builtin_nontemporal_store(v[i], (u32x4*)p + i);
      else *((u32x4*)p + i) = v[i];
    }
  }
  __device__ __forceinline__ void values(float (&x)[8]) const {
#pragma unroll
    for (int e = 0; e < 8; ++e) {
      if constexpr (DT == KARA_BF16)
        x[e] = __uint_as_float((e & 1) ? v[0][e >> 1] & 0xffff0000u : v[0][e >> 1] << 16);
      else
        x[e] = __uint_as_float(v[e >> 2][e & 3]);
    }
  }
  __device__ __forceinline__ void set(const float (&x)[8]) {
    if constexpr (DT == KARA_BF16) {
#pragma unroll
      for (int i = 0; i < 4; ++i) {
        const bf16x2 t = {(__bf16)x[2 * i], (__bf16)x[2 * i + 1]};
        v[0][i] = __builtin_bit_cast(uint32_t, t);
      }
    } else {
#pragma unroll
      for (int e = 0; e < 8; ++e) v[e >> 2][e & 3] = __float_as_uint(x[e]);
    }
  }
};

// Rows are taken by pairs of octets: item i of a row is octets i and i + half/8 where
// they turn together, else the next two of those that stay.
struct Pair {
  int a, b;
  bool turns;
};
__device__ __forceinline__ Pair pair_of(int i, int half) {
  const int ho = half >> 3;
  if (i < ho) return {i, i + ho, true};
  return {2 * i, 2 * i + 1, false};
}

template <int D>
struct Angles {
  // (rows padded by 16 bytes: the lanes of two tokens read different banks)
  float cos[kTile][D / 2 + 4], sin[kTile][D / 2 + 4];
  double rev[D / 2];      // revolutions a position
};

constexpr float kPi = 3.14159265358979f;

// cos and sin of `count` tokens from rotary position pos on, by all threads.  In half turns an
// angle is a + b, a its rounding to fp32 and b, of 2^-25 at most, what that left: sin(a + b) =
// sin a + pi b cos a and cos(a + b) = cos a - pi b sin a, to b^2.
template <int D, int THREADS>
__device__ __forceinline__ void fill_angles(Angles<D>& t, const StoreHead& a, int64_t pos, int count) {
  for (int x = threadIdx.x; x < count * a.half; x += THREADS) {
    const int tok = x / a.half, i = x - tok * a.half;
    const double rev = (double)(pos + tok) * t.rev[i], half_turns = 2.0 * (rev - rint(rev));
    const float a_part = (float)half_turns, rest = (float)(half_turns - (double)a_part) * kPi;
    float sn, cs;
    sincospif(a_part, &sn, &cs);
    t.cos[tok][i] = fmaf(-rest, sn, cs);
    t.sin[tok][i] = fmaf(rest, cs, sn);
  }
}

template <int D, int THREADS>
__device__ __forceinline__ void fill_frequencies(Angles<D>& t, const StoreHead& a) {
  constexpr double kPerTurn = 0.15915494309189533576888376337251;   // 1 / 2 pi
  for (int i = threadIdx.x; i < a.half; i += THREADS)
    t.rev[i] = (a.inv_freq ? (double)a.inv_freq[i] : exp2(-a.step * i)) * kPerTurn;
}

template <int D>
__device__ __forceinline__ void turn(const Angles<D>& t, int tok, int octet, float (&x)[8], float (&y)[8]) {
#pragma unroll
  for (int e = 0; e < 8; e += 4) {
    const floatx4 c = *(const floatx4*)&t.cos[tok][octet * 8 + e], s = *(const floatx4*)&t.sin[tok][octet * 8 + e];
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      const float u = x[e + i], v = y[e + i];
      x[e + i] = u * c[i] - v * s[i];
      y[e + i] = v * c[i] + u * s[i];
    }
  }
}

__device__ __forceinline__ uint32_t wave_max(uint32_t x) {
#pragma unroll
  for (int i = 1; i < 64; i <<= 1) x = max(x, (uint32_t)__shfl_xor((int)x, i, 64));
  return x;
}

// Magnitude of eight values as fp32 bits, those that are not finite left out; a NaN becomes 0.
__device__ __forceinline__ uint32_t finite_top(float (&x)[8], bool* odd) {
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
  return top;
}

// A token's angles are formed once, in LDS, for all its heads, queries, and layers of a
// launch of few tokens: pos * f in revolutions in fp64, sine and cosine of its fraction in
// fp32, with what the fraction's rounding to fp32 leaves.
//
// Bound by the bytes where tokens are many: 4 x 4000 tokens x 4 layers, 32/8 heads, d = 128:
// into rows 314 us for 1.57 GB, into codes 291 for 1.44, both 5.0 TB/s, a large copy's rate, and
// what the counters of memory traffic hold; codes read back too 344.  Pages of more tokens than a
// wave's lanes hold read K and V twice, with a table of angles for every 32 tokens in both sweeps:
// 14 x 1476 tokens x 4 layers, pages of 256, read back 623 us (1.34 GB fetched for 1.02), pages
// of 16 432.
//
// One run of tokens of sequence s = seqs[j] in layers [l0, l1), `heads` KV heads from h0 on and
// their query heads, by all threads.  8 bits: the tokens that fall into one page, as its
// scale is formed of all of them; a wave takes a (layer, K|V, head) at a time, HELD items of
// a lane.  Rows: 32 tokens.  (More than one layer: of 64 HELD items of a head at most.)
// Returns whether a value to be quantised was not finite.
template <int DT, int D, bool Q8, int THREADS, int HELD, int NL>
__device__ __forceinline__ bool store_unit(const Store<NL>& a, Angles<D>& t, uint32_t (&tops)[2 * kGroupHeads],
                                           uint32_t (&bytes)[2 * kGroupHeads], int j, int l0, int l1, int unit, int h0,
                                           int heads, int s, int pos0, int64_t rot0) {
  constexpr int kItems = D / 16;                 // of a row
  constexpr int kRow = D * (DT == KARA_BF16 ? 2 : 4), kOct = kRow / (D / 8);
  constexpr int kWaves = THREADS / 64;
  constexpr int kTokens = 64 * HELD / kItems;    // whose items a wave's lanes hold
  const Dims& g = a.g;
  const int tid = threadIdx.x, lane = tid & 63;
  const int wave = __builtin_amdgcn_readfirstlane(tid >> 6);
  const int layers = l1 - l0;
  int tok0 = unit * kTile, tok1 = min(tok0 + kTile, a.n_new), block = 0;
  if constexpr (Q8) {
    block = pos0 / g.bs + unit;
    const int64_t first = (int64_t)block * g.bs - pos0;         // the page's first token
    tok0 = (int)min(max(first, (int64_t)0), (int64_t)a.n_new);
    tok1 = (int)min(first + g.bs, (int64_t)a.n_new);
  }
  if (tok0 >= tok1) return false;
  const int32_t* row_pages = a.bt + (int64_t)s * g.max_blocks;
  auto src0 = [&](int l) __attribute__((always_inline)) { return ((int64_t)l * a.n + j) * a.n_new; };   // row of token 0
  const char* src_of[2] = {a.k_new, a.v_new};
  bool odd = false;

  // an item's octets as fp32, turned where they turn
  auto item = [&](int l, int kv, int tile0, int head, int x, float (&u)[8], float (&v)[8], int& tok, Pair& p)
                  __attribute__((always_inline)) {
    tok = x / kItems;
    p = pair_of(x - tok * kItems, kv ? 0 : a.half);
    const char* row = src_of[kv] + ((src0(l) + tile0 + tok) * g.Hkv + head) * kRow;
    Raw<DT> ra, rb;
    ra.load(row + p.a * kOct);
    rb.load(row + p.b * kOct);
    ra.values(u);
    rb.values(v);
    if (p.turns) turn(t, tok, p.a, u, v);
  };

  // rows turned one by one, `total` items of them: four on their way at a time, where there
  // are so many (THREADS == kStoreThreads).  stream: they are not read again soon.
  struct Item {
    const char* from;
    char* to;
    Pair p;
    int tok;
  };
  auto rows_by_item = [&](auto stream, int total, auto where) __attribute__((always_inline)) {
    constexpr int kAtOnce = THREADS == kStoreThreads ? 4 : 1;
    for (int x0 = tid; x0 < total; x0 += kAtOnce * THREADS) {
      Item it[kAtOnce];
      Raw<DT> ra[kAtOnce], rb[kAtOnce];
#pragma unroll
      for (int k = 0; k < kAtOnce; ++k) {
        it[k] = where(min(x0 + k * THREADS, total - 1));
        ra[k].load(it[k].from + it[k].p.a * kOct);
        rb[k].load(it[k].from + it[k].p.b * kOct);
      }
#pragma unroll
      for (int k = 0; k < kAtOnce; ++k) {
        if (x0 + k * THREADS >= total) break;
        if (it[k].p.turns) {
          float u[8], v[8];
          ra[k].values(u);
          rb[k].values(v);
          turn(t, it[k].tok, it[k].p.a, u, v);
          ra[k].set(u);
          rb[k].set(v);
        }
        ra[k].template store<decltype(stream)::value && kAtOnce != 1>(it[k].to + it[k].p.a * kOct);
        rb[k].template store<decltype(stream)::value && kAtOnce != 1>(it[k].to + it[k].p.b * kOct);
      }
    }
  };

  const bool whole = tok1 - tok0 <= kTokens;     // one tile
  if (Q8 && !whole) {
    // the page's largest magnitudes first
    for (int i = tid; i < 2 * kGroupHeads; i += THREADS) tops[i] = 0;
    for (int tile0 = tok0; tile0 < tok1; tile0 += kTokens) {
      const int count = min(kTokens, tok1 - tile0);
      __syncthreads();
      fill_angles<D, THREADS>(t, a, rot0 + tile0, count);
      __syncthreads();
      for (int job = wave; job < 2 * heads; job += kWaves) {
        const int kv = job >= heads, head = h0 + (kv ? job - heads : job);
        uint32_t top = 0;
        for (int x = lane; x < count * kItems; x += 64) {
          float u[8], v[8];
          int tok;
          Pair p;
          item(l0, kv, tile0, head, x, u, v, tok, p);
          top = max(top, max(finite_top(u, &odd), finite_top(v, &odd)));
        }
        top = wave_max(top);
        if (lane == 0) tops[job] = max(tops[job], top);
      }
    }
  }
  constexpr int kStep = Q8 ? kTokens : kTile;
  for (int tile0 = tok0; tile0 < tok1; tile0 += kStep) {
    const int count = min(kStep, tok1 - tile0);
    __syncthreads();
    fill_angles<D, THREADS>(t, a, rot0 + tile0, count);
    __syncthreads();
    if constexpr (Q8) {
      const int page = row_pages[block];
      const int slot0 = pos0 + tok0 - block * g.bs;             // of the page's first new token
      for (int x0 = wave; x0 < layers * 2 * heads; x0 += kWaves) {
        const int l = l0 + x0 / (2 * heads), job = x0 - (l - l0) * 2 * heads;
        const int kv = job >= heads, head = h0 + (kv ? job - heads : job);
        float u[HELD][8], v[HELD][8];
        int tok[HELD];
        Pair p[HELD];
        uint32_t top = 0;
#pragma unroll
        for (int k = 0; k < HELD; ++k) {
          const int x = lane + 64 * k;
          if (x >= count * kItems) continue;
          item(l, kv, tile0, head, x, u[k], v[k], tok[k], p[k]);
          top = max(top, max(finite_top(u[k], &odd), finite_top(v[k], &odd)));
        }
        const int64_t unit_at = (int64_t)page * g.Hkv + head;
        uint8_t* codes = (uint8_t*)(kv ? a.vp.p[l] : a.kp.p[l]) + unit_at * g.bs * D;
        uint8_t* scales = (uint8_t*)(kv ? a.vsp.p[l] : a.ksp.p[l]) + unit_at;
        uint32_t byte;
        if (tile0 == tok0) {
          byte = q8_scale_byte(whole ? wave_max(top) : tops[job]);
          if (slot0 > 0) {
            // older tokens of the page: the larger scale, theirs rounded to it where it grows
            const uint32_t was = min(max((uint32_t)*scales, kQ8Lowest), kQ8Highest);
            if (byte > was) {
              const float ratio = q8_scale(127 + was - byte > 254 ? 0 : 127 + was - byte);
              for (int i = lane; i < slot0 * (D / 4); i += 64)
                ((uint32_t*)codes)[i] = q8_rescale(((const uint32_t*)codes)[i], ratio);
            }
            byte = max(byte, was);
          }
          if (lane == 0) {
            *scales = (uint8_t)byte;
            if (!whole) bytes[job] = byte;                      // for the page's further tiles
          }
        } else {
          byte = bytes[job];
        }
        const float per_unit = q8_per_unit(byte);
#pragma unroll
        for (int k = 0; k < HELD; ++k) {
          if (lane + 64 * k >= count * kItems) continue;
          uint8_t* row = codes + (int64_t)(slot0 + tile0 - tok0 + tok[k]) * D;
          *(u32x2*)(row + p[k].a * 8) = u32x2{q8_codes(u[k][0], u[k][1], u[k][2], u[k][3], per_unit),
                                              q8_codes(u[k][4], u[k][5], u[k][6], u[k][7], per_unit)};
          *(u32x2*)(row + p[k].b * 8) = u32x2{q8_codes(v[k][0], v[k][1], v[k][2], v[k][3], per_unit),
                                              q8_codes(v[k][4], v[k][5], v[k][6], v[k][7], per_unit)};
        }
      }
    } else {
      // rows of the tile, (K|V, token, head) in order
      const int layer_rows = 2 * count * heads;
      rows_by_item(std::false_type{}, layers * layer_rows * kItems, [&](int x) __attribute__((always_inline)) {
        const int lrow = x / kItems;
        const int l = l0 + lrow / layer_rows, row = lrow - (l - l0) * layer_rows;
        const int kv = row >= count * heads, r = kv ? row - count * heads : row;
        const int tok = r / heads, head = h0 + r - tok * heads;
        const int pos = pos0 + tile0 + tok, b = pos / g.bs;
        return Item{src_of[kv] + ((src0(l) + tile0 + tok) * g.Hkv + head) * kRow,
                    (char*)(kv ? a.vp.p[l] : a.kp.p[l]) + (((int64_t)row_pages[b] * g.Hkv + head) * g.bs + (pos - b * g.bs)) * kRow,
                    pair_of(x - lrow * kItems, kv ? 0 : a.half), tok};
      });
    }
    if (a.q) {
      const int qh = heads * g.G;
      rows_by_item(std::true_type{}, layers * count * qh * kItems, [&](int x) __attribute__((always_inline)) {
        const int lrow = x / kItems;
        const int l = l0 + lrow / (count * qh), row = lrow - (l - l0) * count * qh;
        const int tok = row / qh, head = h0 * g.G + row - tok * qh;
        const int64_t at = ((src0(l) + tile0 + tok) * g.Hq + head) * kRow;
        return Item{a.q + at, a.q_out + at, pair_of(x - lrow * kItems, a.half), tok};
      });
    }
  }
  return odd;
}

__device__ __forceinline__ void start_of(const StoreHead& a, int s, int* pos0, int64_t* rot0) {
  const int back = a.counted ? a.n_new : 0;
  *pos0 = a.seq_lens[s] - back;
  *rot0 = a.rope_pos ? (int64_t)a.rope_pos[s] - back : *pos0;
}

__global__ __launch_bounds__(kAppendThreads) void store_check_kernel(StoreHead a) {
  const int st = append_status(a.g, a.n, a.seqs, a.n_new, a.bt, a.seq_lens, blockIdx.x, a.counted != 0);
  if (threadIdx.x == 0) a.status[blockIdx.x] = st;
}

// (after the rows, so that a call that could not make their launch counts nothing)
__global__ __launch_bounds__(kAppendThreads) void store_commit_kernel(StoreHead a) {
  const int j = blockIdx.x * kAppendThreads + threadIdx.x;
  if (j < a.n && (a.status[j] & ~KARA_SEQ_NONFINITE) == 0) {
    a.seq_lens[a.seqs[j]] += a.n_new;
    if (a.rope_pos) a.rope_pos[a.seqs[j]] += a.n_new;
  }
}

// Grid (sequence x unit, layer, group of heads), between the check and the commit.
template <int DT, int D, bool Q8, int NL>
__global__ __launch_bounds__(kStoreThreads) void store_kernel(Store<NL> a) {
  __shared__ __attribute__((aligned(16))) Angles<D> t;
  __shared__ uint32_t tops[2 * kGroupHeads], bytes[2 * kGroupHeads];
  const int j = blockIdx.x / a.units, unit = blockIdx.x - j * a.units;
  // (other workgroups may have reported a value that is not finite by now)
  if (a.status[j] & ~KARA_SEQ_NONFINITE) return;
  fill_frequencies<D, kStoreThreads>(t, a);
  const int s = a.seqs[j];
  int pos0;
  int64_t rot0;
  start_of(a, s, &pos0, &rot0);
  __syncthreads();
  const int l = blockIdx.y, h0 = blockIdx.z * a.group;
  const bool odd = store_unit<DT, D, Q8, kStoreThreads, kTile * (D / 16) / 64>(
      a, t, tops, bytes, j, l, l + 1, unit, h0, min(a.group, a.g.Hkv - h0), s, pos0, rot0);
  if (Q8 && __syncthreads_or(odd) && threadIdx.x == 0) atomicOr(&a.status[j], KARA_SEQ_NONFINITE);
}

// A few new tokens: one workgroup per listed sequence checks it, appends all its rows and
// commits, in one launch (8 sequences, one token, one layer: 6.6 us; 64 into codes 10.7).  (The
// tokens' items of a head are one a lane at most, so that no page has further tiles, and `tops`
// and `bytes` are not used.)
template <int DT, int D, bool Q8, int NL>
__global__ __launch_bounds__(kFewThreads) void store_few_kernel(Store<NL> a) {
  __shared__ __attribute__((aligned(16))) Angles<D> t;
  __shared__ uint32_t tops[2 * kGroupHeads], bytes[2 * kGroupHeads];
  const int j = blockIdx.x;
  fill_frequencies<D, kFewThreads>(t, a);
  int st = append_status(a.g, a.n, a.seqs, a.n_new, a.bt, a.seq_lens, j, a.counted != 0);
  __syncthreads();
  if (st == KARA_SEQ_OK) {
    const int s = a.seqs[j];
    int pos0;
    int64_t rot0;
    start_of(a, s, &pos0, &rot0);
    bool odd = false;
    for (int unit = 0; unit < a.units; ++unit)
      odd |= store_unit<DT, D, Q8, kFewThreads, 1>(a, t, tops, bytes, j, 0, a.n_layers, unit, 0, a.g.Hkv, s, pos0, rot0);
    if (Q8 && __syncthreads_or(odd)) st = KARA_SEQ_NONFINITE;
  }
  __syncthreads();                       // every thread has read the length before it changes
  if (threadIdx.x == 0) {
    a.status[j] = st;
    if ((st & ~KARA_SEQ_NONFINITE) == 0 && !a.counted) {
      a.seq_lens[a.seqs[j]] += a.n_new;
      if (a.rope_pos) a.rope_pos[a.seqs[j]] += a.n_new;
    }
  }
}

// ---------------------------------------------------------------- read

// The pages' rows back, an octet a lane (4 x 4000 tokens x 4 layers: 393 MB in 60-83 us, by
// what the caches still hold).
constexpr int kReadUnroll = 4;

template <int DT, int D, int NL>
__global__ __launch_bounds__(kStoreThreads) void q8_read_kernel(
    Dims g, int n, const int32_t* __restrict__ seqs, const int32_t* __restrict__ start, int n_rows, int toks, int chunks,
    Pools<NL> kp, Pools<NL> vp, Pools<NL> ksp, Pools<NL> vsp, const int32_t* __restrict__ bt,
    const int32_t* __restrict__ seq_lens, char* __restrict__ k_out, char* __restrict__ v_out) {
  constexpr int kOctets = D / 8, kOct = DT == KARA_BF16 ? 16 : 32;
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
  char* dst = (kv ? v_out : k_out) + (((int64_t)l * n + j) * n_rows + tok0) * per_tok * kOct;
  const uint8_t* codes = (const uint8_t*)(kv ? vp.p[l] : kp.p[l]);
  const uint8_t* scales = (const uint8_t*)(kv ? vsp.p[l] : ksp.p[l]);
  for (int from = threadIdx.x; from < count; from += kStoreThreads * kReadUnroll) {
    u32x2 c[kReadUnroll];
    uint32_t byte[kReadUnroll], unit[kReadUnroll];
    int page[kReadUnroll], slot[kReadUnroll], o[kReadUnroll];
    bool in[kReadUnroll];
#pragma unroll
    for (int k = 0; k < kReadUnroll; ++k) {
      const int i = min(from + k * kStoreThreads, count - 1);
      const int tok = i / per_tok, r = i - tok * per_tok;
      const int h = r / kOctets;
      o[k] = r - h * kOctets;
      in[k] = pos0 + tok >= 0 && pos0 + tok < len;
      const int pos = in[k] ? (int)(pos0 + tok) : 0, b = pos / g.bs;
      page[k] = row_pages[b];
      slot[k] = pos - b * g.bs;
      unit[k] = h;
    }
#pragma unroll
    for (int k = 0; k < kReadUnroll; ++k) {
      in[k] &= page[k] >= 0 && page[k] < g.num_pages;
      // (a pool has fewer than 2^32 rows)
      unit[k] += (uint32_t)(in[k] ? page[k] : 0) * (uint32_t)g.Hkv;
      c[k] = *(const u32x2*)(codes + ((uint64_t)unit[k] * g.bs + slot[k]) * D + o[k] * 8);
      byte[k] = scales[unit[k]];
    }
#pragma unroll
    for (int k = 0; k < kReadUnroll; ++k) {
      if (from + k * kStoreThreads >= count) break;
      if (!in[k]) c[k] = u32x2{0, 0}, byte[k] = 127;
      const float scale = q8_scale(byte[k]);
      u32x4* to = (u32x4*)(dst + (int64_t)(from + k * kStoreThreads) * kOct);
      if constexpr (DT == KARA_BF16) {
        __builtin_nontemporal_store(__builtin_bit_cast(u32x4, q8_octet(c[k][0], c[k][1], scale)), to);
      } else {
#pragma unroll
        for (int i = 0; i < 2; ++i) {
          const floatx2 x = __builtin_amdgcn_cvt_scalef32_pk_f32_fp8(c[k][i], scale, false);
          const floatx2 y = __builtin_amdgcn_cvt_scalef32_pk_f32_fp8(c[k][i], scale, true);
          __builtin_nontemporal_store(__builtin_bit_cast(u32x4, floatx4{x[0], x[1], y[0], y[1]}), to + i);
        }
      }
    }
  }
}

// a grid of one dimension, of up to 1024 threads a block: HIP counts its threads in 32 bits
bool grid_ok(int64_t blocks) { return blocks > 0 && blocks < ((int64_t)1 << 22); }

bool layers_ok(int32_t n, int32_t n_layers) { return n >= 0 && n_layers >= 1 && n_layers <= kMaxLayersPerLaunch; }

template <int DT, int D, bool Q8, int NL>
kara_status_t launch_store(const Store<NL>& a, hipStream_t s) {
  // a few items in all: one workgroup a sequence
  const int64_t items = (int64_t)a.n_layers * a.n_new * (2 * a.g.Hkv + (a.q ? a.g.Hq : 0)) * (D / 16);
  if (a.n_new * (D / 16) <= 64 && items <= 8 * kFewThreads) {
    hipLaunchKernelGGL((store_few_kernel<DT, D, Q8, NL>), dim3((unsigned)a.n), dim3(kFewThreads), 0, s, a);
    return hip_status(hipGetLastError());
  }
  hipLaunchKernelGGL(store_check_kernel, dim3((unsigned)a.n), dim3(kAppendThreads), 0, s, (const StoreHead&)a);
  hipError_t e = hipGetLastError();
  if (e != hipSuccess) return hip_status(e);
  const unsigned groups = (unsigned)((a.g.Hkv + a.group - 1) / a.group);
  hipLaunchKernelGGL((store_kernel<DT, D, Q8, NL>), dim3((unsigned)(a.n * a.units), (unsigned)a.n_layers, groups),
                     dim3(kStoreThreads), 0, s, a);
  e = hipGetLastError();
  if (e != hipSuccess || a.counted) return hip_status(e);
  hipLaunchKernelGGL(store_commit_kernel, dim3((unsigned)((a.n + kAppendThreads - 1) / kAppendThreads)),
                     dim3(kAppendThreads), 0, s, (const StoreHead&)a);
  return hip_status(hipGetLastError());
}

// The call both appends come to; rope: null for none.
kara_status_t store(const kara_params_t* p, const kara_rope_t* rope, int32_t n, const int32_t* seqs, int32_t n_new,
                    int32_t n_layers, const void* q, const void* k_new, const void* v_new, void* q_out,
                    void* const* k_pools, void* const* v_pools, void* const* k_scales, void* const* v_scales,
                    const int32_t* block_table, int32_t* seq_lens, int32_t* rope_pos, int32_t counted, int32_t* status,
                    void* stream) {
  Geom g;
  const kara_status_t st = make_geom(p, n, &g);
  if (st != KARA_OK) return st;
  StoreHead a{};
  a.g = dims_of(g);
  if (!layers_ok(n, n_layers) || n_new < 0 || counted < 0 || counted > 1) return KARA_ERR_INVALID_ARG;
  if (rope) {
    const int dim = rope->dim == 0 ? g.d : rope->dim;
    if (dim < 0 || dim % 16 != 0 || dim > g.d) return KARA_ERR_INVALID_ARG;
    if (!rope->inv_freq && !(rope->theta > 0.f && std::isfinite(rope->theta))) return KARA_ERR_INVALID_ARG;
    if (!aligned(4, {rope->inv_freq})) return KARA_ERR_INVALID_ARG;
    a.half = dim / 2;
    a.step = rope->inv_freq ? 0.0 : std::log2((double)rope->theta) * 2.0 / dim;
    a.inv_freq = rope->inv_freq;
  }
  if ((k_scales == nullptr) != (v_scales == nullptr) || (q == nullptr) != (q_out == nullptr)) return KARA_ERR_INVALID_ARG;
  if (n == 0 || n_new == 0) return KARA_OK;
  const bool q8 = k_scales != nullptr;
  if (!seqs || !k_new || !v_new || !block_table || !seq_lens || !status || !pools_ok(k_pools, n_layers) ||
      !pools_ok(v_pools, n_layers) || (q8 && (!pools_ok(k_scales, n_layers) || !pools_ok(v_scales, n_layers))))
    return KARA_ERR_INVALID_ARG;
  if (!aligned(16, {q, k_new, v_new, q_out}) || !aligned(4, {seqs, block_table, seq_lens, rope_pos, status}) ||
      !pools_aligned(16, k_pools, n_layers) || !pools_aligned(16, v_pools, n_layers))
    return KARA_ERR_INVALID_ARG;
  if ((int64_t)g.Hq * (g.d / 8) > kMaxOctets) return KARA_ERR_UNSUPPORTED;
  // (8 bits: a run of n_new tokens enters one page more where it starts late in one)
  const int64_t units = q8 ? ((int64_t)n_new + g.bs - 2) / g.bs + 1 : ((int64_t)n_new + kTile - 1) / kTile;
  // (a page of many tokens is one workgroup's for a head: fewer heads each where there are
  // few of them)
  a.group = std::min(g.Hkv, kGroupHeads);
  while (a.group > 1 && n * units * n_layers * ((g.Hkv + a.group - 1) / a.group) < kStoreWgs) a.group = (a.group + 1) / 2;
  if (!grid_ok(n * units) || (g.Hkv + a.group - 1) / a.group > 65535) return KARA_ERR_UNSUPPORTED;
  a.units = (int)units;
  a.n = n;
  a.n_new = n_new;
  a.n_layers = n_layers;
  a.counted = counted;
  a.seqs = seqs;
  a.bt = block_table;
  a.seq_lens = seq_lens;
  a.rope_pos = rope_pos;
  a.status = status;
  a.q = (const char*)q;
  a.k_new = (const char*)k_new;
  a.v_new = (const char*)v_new;
  a.q_out = (char*)q_out;
  hipStream_t s = (hipStream_t)stream;
  auto launch = [&](auto call) {
    set_pools(&call.kp, k_pools, n_layers);
    set_pools(&call.vp, v_pools, n_layers);
    set_pools(&call.ksp, k_scales, n_layers);
    set_pools(&call.vsp, v_scales, n_layers);
#define KARA_STORE(DT, D) return q8 ? launch_store<DT, D, true>(call, s) : launch_store<DT, D, false>(call, s)
    if (g.dtype == KARA_BF16) {
      if (g.d == 128) KARA_STORE(KARA_BF16, 128);
      KARA_STORE(KARA_BF16, 64);
    }
    if (g.d == 128) KARA_STORE(KARA_F32, 128);
    KARA_STORE(KARA_F32, 64);
#undef KARA_STORE
  };
  if (n_layers <= kFewLayers) return launch(Store<kFewLayers>{a, {}, {}, {}, {}});
  return launch(Store<kMaxLayersPerLaunch>{a, {}, {}, {}, {}});
}

}  // namespace
}  // namespace kara

using namespace kara;

extern "C" {

kara_status_t kara_rope_append(const kara_params_t* p, const kara_rope_t* rope, int32_t n, const int32_t* seqs,
                               int32_t n_new, int32_t n_layers, const void* q, const void* k_new, const void* v_new,
                               void* q_out, void* const* k_pools, void* const* v_pools, void* const* k_scales,
                               void* const* v_scales, const int32_t* block_table, int32_t* seq_lens,
                               int32_t* rope_pos, int32_t counted, int32_t* status, void* stream) {
  if (!rope) return KARA_ERR_INVALID_ARG;
  return store(p, rope, n, seqs, n_new, n_layers, q, k_new, v_new, q_out, k_pools, v_pools, k_scales, v_scales,
               block_table, seq_lens, rope_pos, counted, status, stream);
}

kara_status_t kara_q8_append(const kara_params_t* p, int32_t n, const int32_t* seqs, int32_t n_new, int32_t n_layers,
                             const void* k_new, const void* v_new, void* const* k_pools, void* const* v_pools,
                             void* const* k_scales, void* const* v_scales, const int32_t* block_table,
                             int32_t* seq_lens, int32_t* status, void* stream) {
  if (n > 0 && n_new > 0 && (!k_scales || !v_scales)) return KARA_ERR_INVALID_ARG;
  return store(p, nullptr, n, seqs, n_new, n_layers, nullptr, k_new, v_new, nullptr, k_pools, v_pools, k_scales, v_scales,
               block_table, seq_lens, nullptr, 0, status, stream);
}

kara_status_t kara_q8_read(const kara_params_t* p, int32_t n, const int32_t* seqs, const int32_t* start, int32_t n_rows,
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
      !pools_aligned(16, k_pools, n_layers) || !pools_aligned(16, v_pools, n_layers))
    return KARA_ERR_INVALID_ARG;
  if ((int64_t)g.Hkv * (g.d / 8) > kMaxOctets) return KARA_ERR_UNSUPPORTED;
  const int per_tok = g.Hkv * (g.d / 8);
  const int toks = std::min(n_rows, std::max(1, 2 * kStoreThreads * kReadUnroll / per_tok));
  const int64_t chunks = ((int64_t)n_rows + toks - 1) / toks;
  if (!grid_ok(n * chunks)) return KARA_ERR_UNSUPPORTED;
  const dim3 grid((unsigned)(n * chunks), (unsigned)n_layers, 2), block(kStoreThreads);
  auto launch = [&](auto kp) {
    auto vp = kp, ksp = kp, vsp = kp;
    set_pools(&kp, k_pools, n_layers);
    set_pools(&vp, v_pools, n_layers);
    set_pools(&ksp, k_scales, n_layers);
    set_pools(&vsp, v_scales, n_layers);
    constexpr int NL = sizeof(kp) / sizeof(void*);
#define KARA_Q8_READ(DT, D)                                                                                             \
  hipLaunchKernelGGL((q8_read_kernel<DT, D, NL>), grid, block, 0, (hipStream_t)stream, dims_of(g), n, seqs, start, n_rows, \
                     toks, (int)chunks, kp, vp, ksp, vsp, block_table, seq_lens, (char*)k_out, (char*)v_out)
    if (g.dtype == KARA_BF16) {
      if (g.d == 128) KARA_Q8_READ(KARA_BF16, 128);
      else KARA_Q8_READ(KARA_BF16, 64);
    } else {
      if (g.d == 128) KARA_Q8_READ(KARA_F32, 128);
      else KARA_Q8_READ(KARA_F32, 64);
    }
#undef KARA_Q8_READ
  };
  if (n_layers <= kFewLayers) launch(Pools<kFewLayers>{});
  else launch(Pools<kMaxLayersPerLaunch>{});
  return hip_status(hipGetLastError());
}

}  // extern "C"

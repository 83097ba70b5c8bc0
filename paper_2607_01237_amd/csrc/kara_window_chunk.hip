// Attention within a sliding window and the first tokens (include/kara_window.h) of many
// query rows, a prompt's chunk over what is cached, over 8-bit codes or bf16 rows.  Bound
// by the matrix products.
//
// One workgroup of 8 waves owns 128 QT query rows of one (layer, sequence, KV head),
// rows ordered (query, head in group), and walks the keys of their span 64 at a time.  A
// chunk passes through LDS once for all rows, with one barrier: rows copied straight to a
// ring of four stages, three chunks ahead; codes fetched into registers two chunks ahead,
// converted in hardware to bf16 -- exactly -- and written to the other of two stages while
// the products of the present one run.  From there S^T = K Q^T, weights as they stand the B
// operand of O^T += V^T P^T with V through the transposed LDS read, the row sums one more
// product with ones.  A chunk of 256 rows of 128 takes 4550 cycles of a CU, 2.0 us on a full card:
// its products 2180 (counted), its LDS reads 2050 (every wave reads all of K and V, 256 KB at 128
// bytes a cycle) and its vector instructions some 2100 (331 of a SIMD counted, 64 of them
// exponentials, of 16 cycles, the others of 4), which two waves a SIMD overlap in part.
//
// NT: bf16 terms of a query and of a weight (1: bf16 calls; 3: fp32 ones over codes).  bf16
// calls so round a weight, in the output as in its sum, to bf16: 2.3e-3 of the result against
// 64 bits where whole weights would give 1.7e-3, the output's own rounding; a second term
// makes V's products twice as many, and calls a quarter to a third longer (us with one and
// with two: 4 x 1024 queries in a window of 1024 96, 119; over 8.7K tokens 538, 716, codes 541,
// 702; 4 x 512 over 2.5-8.7K, codes 243, 304).
//
// 4 sequences x 1024 queries over 8.7K tokens, 32/8 heads, d = 128: rows 534 us, codes 539
// (1.03, 1.02 PFLOP/s); in a window of 1024 over 2.5-8.7K 98 us (704 TFLOP/s: 18 chunks a row
// block, beside which its start, queries and results count); 16 x 1024 380 us.  4 x 512 over
// 2.5-8.7K, codes: 243 us.
#include <algorithm>
#include <type_traits>

#include "kara_lds.h"
#include "kara_q8_device.h"
#include "kara_window_call.h"

namespace kara {
namespace {

constexpr int kCUs = 256;
constexpr int kChKeys = 64;
constexpr int kLeastChunks = 8;         // of a split
constexpr float kLog2e = 1.4426950408889634f;
constexpr float kNegInf = -__builtin_huge_valf();
constexpr float kMaxFloor = -3.402823466e38f;
constexpr float kHeadroom = 8.f;

constexpr int kRuns = 1024;             // runs of keys in the LDS table at a time

template <bool Q8, int D, int W>
struct ChCfg {
  static constexpr int kThreads = W * 64;
  static constexpr int kRow = D * 2;                 // bytes of a row in LDS
  static constexpr int kChunks = kRow / 16;
  static constexpr int kKS = D / 32;                 // products per dot product
  static constexpr int kDT = D / 16;                 // 16-row tiles of O^T
  static constexpr int kTile = kChKeys * kRow;       // a chunk of K, or of V
  static constexpr int kSrc = Q8 ? D : 2 * D;        // bytes of a row in the pool
  static constexpr int kPieces = kSrc / 16;          // 16-byte pieces of it, a thread each
  static constexpr int kStagers = kChKeys * kPieces; // pieces of K's chunk, and of V's
  static constexpr int kKeys = kStagers > kThreads ? kStagers / kThreads : 1;   // keys of a thread
  static constexpr int kKeyStep = kThreads / kPieces;
  // Rows: a ring of four stages, copied three chunks ahead.  Codes: two, written from registers.
  static constexpr int kStages = Q8 ? 2 : 4;
  static constexpr int kCopies = 2 * kKeys;          // of a thread and chunk
  // XOR swizzles of a row's 16-byte chunks
  static __device__ __forceinline__ int swz_k(int row) {
    if constexpr (D == 128) return ((row & 3) << 2) | ((row >> 2) & 3);
    return ((row & 3) << 1) | ((row >> 2) & 1);
  }
  static __device__ __forceinline__ int swz_v(int row) { return (2 * (D == 128 ? row : row >> 1)) & (kChunks - 1); }
};

// Values of keys that no row sees: read in their place.
__device__ const uint4 kZeroRow[16] = {};

typedef short v4i16 __attribute__((ext_vector_type(4)));
__device__ inline v4i16 read_tr(const char* p) {
  return __builtin_amdgcn_ds_read_tr16_b64_v4i16(
      (__attribute__((address_space(3))) v4i16*)(__attribute__((address_space(3))) char*)p);
}

// Where a call has fewer than two workgroups to a CU, long sequences' keys are split, so
// that it does not end with them: a row block of a sequence of c chunks (its last block's)
// becomes ceil(c / P) workgroups, P the chunks of all blocks over the CUs, 512 keys at
// least.  The others write their rows; these write records, which a second launch joins (a
// join of 64 rows a workgroup, 12.8 us for half of 4 x 512 queries' blocks).  9 x 118 queries x
// 2 layers over 23-5990 tokens 223 -> 167 us, 4 x 512 over 2.5-8.7K 273 -> 243, where all
// blocks in two halves took 309.
struct ChunkSplit {
  int most;              // sequences whose keys may be split: the first `most` threads' (0: none)
  float *o, *ml;         // records [..][rows_wg][D]; [..][rows_wg]: m, l
  int2* of_seq;          // [n]: splits, and the first record
};

template <bool Q8, int NT, int D, int QT>
__global__ __launch_bounds__(512, 2) void window_chunk_kernel(WindowCall a, ChunkSplit x) {
  constexpr int W = 8;
  using C = ChCfg<Q8, D, W>;
  constexpr int kRowsWg = W * 16 * QT;
  constexpr int KS = C::kKS, DT = C::kDT, KP = C::kKeys;
  __shared__ __attribute__((aligned(16))) char smem[C::kStages][2 * C::kTile];
  __shared__ uint32_t run_row[kRuns], run_scale[Q8 ? kRuns : 1];   // pool rows of runs of keys; K's scale byte, V's above it
  const Dims& g = a.g;
  const int tid = threadIdx.x, lane = tid & 63;
  const int wave = __builtin_amdgcn_readfirstlane(tid >> 6);
  const int gq = lane >> 4, li = lane & 15;

  // Sequences in the order of their workgroups' chunks, the longest first: this workgroup's
  // is the one whose range of blocks it lies in.
  const uint32_t units = (uint32_t)(a.n_layers * g.Hkv);         // of a sequence
  const uint32_t blocks = units * (uint32_t)a.n_rt;
  int j, s, len, splits = 1, piece_chunks = 0, first_record = 0;
  uint32_t rest = blockIdx.x;
  if (a.n <= C::kThreads) {
    struct Seq {
      int len, splits, chunks;       // chunks of one workgroup, at most
    };
    Seq* seqs = (Seq*)smem[0];
    int* found = (int*)(seqs + a.n);
    int s0 = 0;
    Seq mine{0, 1, 1};
    if (tid < a.n) {
      s0 = a.seqs[tid];
      mine.len = s0 >= 0 && s0 < g.n_seqs ? a.seq_lens[s0] : 0;
      const bool live = mine.len > 0 && mine.len <= a.max_len;
      const int R0 = g.G * a.T;
      mine.chunks = live ? (span_of(mine.len, a.T, g.G, (a.n_rt - 1) * kRowsWg, R0, a.window, a.sink).n + kChKeys - 1) / kChKeys : 1;
      seqs[tid] = mine;
    }
    if (tid == 0) found[0] = -1, found[1] = 1 << 30;
    __syncthreads();
    if (x.most > 0) {
      uint64_t all = 0;
      for (int o = 0; o < a.n; ++o) all += (uint32_t)seqs[o].chunks;
      const uint64_t per = (all * blocks + kCUs - 1) / kCUs;
      int share = (int)(per < (uint64_t)kLeastChunks ? (uint64_t)kLeastChunks : per > (1u << 29) ? (uint64_t)(1u << 29) : per);
      // Up to 3/8 more chunks each where all of them then run at once (a workgroup too many
      // would double the time of equal ones): a candidate a thread.  (1 x 300 queries over 8K
      // tokens, 40 blocks: 6 splits 64 us, 7, one round and a part, 100.)
      const int candidate = share + tid * max(1, share >> 10);
      uint32_t wgs = 0;
      if (candidate <= share + share / 8 * 3)
        for (int o = 0; o < a.n; ++o) wgs += blocks * (uint32_t)((seqs[o].chunks + candidate - 1) / candidate);
      if (wgs != 0 && wgs <= kCUs) atomicMin(&found[1], candidate);
      __syncthreads();
      if (found[1] < (1 << 30)) share = found[1];
      mine.splits = (mine.chunks + share - 1) / share;
      mine.chunks = (mine.chunks + mine.splits - 1) / mine.splits;
      __syncthreads();
      if (tid < a.n) seqs[tid] = mine;
      __syncthreads();
    }
    if (tid < a.n) {
      uint32_t at = 0, record = 0;
      for (int o = 0; o < a.n; ++o) {
        const Seq other = seqs[o];
        if (other.chunks > mine.chunks || (other.chunks == mine.chunks && o < tid)) at += blocks * (uint32_t)other.splits;
        if (o < tid && other.splits > 1) record += blocks * (uint32_t)other.splits;
      }
      if (rest >= at && rest - at < blocks * (uint32_t)mine.splits) {
        found[0] = tid, found[1] = s0, found[2] = mine.len, found[3] = mine.splits, found[4] = mine.chunks;
        found[5] = (int)record, found[6] = (int)(rest - at);
      }
    }
    __syncthreads();
    j = __builtin_amdgcn_readfirstlane(found[0]);
    s = __builtin_amdgcn_readfirstlane(found[1]);
    len = __builtin_amdgcn_readfirstlane(found[2]);
    splits = __builtin_amdgcn_readfirstlane(found[3]);
    piece_chunks = __builtin_amdgcn_readfirstlane(found[4]);
    first_record = __builtin_amdgcn_readfirstlane(found[5]);
    rest = __builtin_amdgcn_readfirstlane(found[6]);
    __syncthreads();
    if (j < 0) return;                   // (the launch has room for the most splits)
    if (x.most > 0 && rest == 0 && tid == 0) x.of_seq[j] = int2{splits, first_record};
  } else {
    j = rest / blocks;
    rest -= (uint32_t)j * blocks;
    s = a.seqs[j];
    len = s >= 0 && s < g.n_seqs ? a.seq_lens[s] : 0;
  }
  // All row blocks and splits of a (layer, KV head) on one XCD, whose L2 then holds its keys
  // once, where the units divide among the 8.
  uint32_t u;
  const uint32_t per = (uint32_t)a.n_rt * (uint32_t)splits;
  if (units % 8 == 0) {
    u = rest / (8 * per) * 8 + rest % 8;
    rest = rest / 8 % per;
  } else {
    u = rest / per;
    rest = rest % per;
  }
  const int split = rest % (uint32_t)splits;
  const int rb = a.n_rt - 1 - (int)(rest / (uint32_t)splits);     // the blocks that see most keys first
  const int h = u % (uint32_t)g.Hkv, l = u / (uint32_t)g.Hkv;
  const int G = g.G, T = a.T, R = G * T;
  const int row0 = rb * kRowsWg;
  const int64_t orow = ((int64_t)l * a.n + j) * T * g.Hq + h * G;
  const bool none = len <= 0 || len > a.max_len;
  const Span sp = span_of(none ? 0 : len, T, G, row0, min(row0 + kRowsWg, R), a.window, a.sink);
  const int first = len - T;                               // position of query 0
  const int k_lo = split * piece_chunks * kChKeys;
  // (the last split takes what is left: a block may see a few keys more than the sequence's last)
  const int k_hi = none ? 0 : split + 1 < splits ? min(sp.n, k_lo + piece_chunks * kChKeys) : sp.n;
  const int n_chunks = k_hi > k_lo ? (k_hi - k_lo + kChKeys - 1) / kChKeys : 0;

  // ---- this wave's queries as B operands (lane: query li of each tile) ----
  const int wrow0 = row0 + wave * 16 * QT;
  bf16x8 qop[QT][NT][KS];
  int qhi[QT];                           // the last key it sees
#pragma unroll
  for (int qt = 0; qt < QT; ++qt) {
    const int r = min(wrow0 + qt * 16 + li, R - 1);
    const int t = r / G;
    qhi[qt] = first + t - sp.gap;
    const int64_t at = (orow + (int64_t)t * g.Hq + (r - t * G)) * D;
#pragma unroll
    for (int x = 0; x < KS; ++x) {
      if constexpr (NT == 1) {
        qop[qt][0][x] = *(const bf16x8*)((const __bf16*)a.q + at + (gq * KS + x) * 8);
      } else {
        const floatx4* src = (const floatx4*)((const float*)a.q + at + (gq * KS + x) * 8);
        const floatx4 p = src[0], q = src[1];
        uint32_t w[4][NT];
#pragma unroll
        for (int i = 0; i < 4; ++i)
          bf16_term_pairs<true>(i < 2 ? p[2 * i] : q[2 * i - 4], i < 2 ? p[2 * i + 1] : q[2 * i - 3], w[i]);
#pragma unroll
        for (int y = 0; y < NT; ++y) qop[qt][y][x] = __builtin_bit_cast(bf16x8, uint4{w[0][y], w[1][y], w[2][y], w[3][y]});
      }
    }
  }
  // last keys that the wave's first and last row see
  const int wave_hi0 = first + min(wrow0, R - 1) / G - sp.gap;
  const int wave_hi1 = first + min(wrow0 + 16 * QT - 1, R - 1) / G - sp.gap;

  floatx4 o[QT][DT], lsum[QT];
  float m[QT];
#pragma unroll
  for (int qt = 0; qt < QT; ++qt) {
    m[qt] = kMaxFloor;
    lsum[qt] = floatx4{0.f, 0.f, 0.f, 0.f};
#pragma unroll
    for (int dt = 0; dt < DT; ++dt) o[qt][dt] = floatx4{0.f, 0.f, 0.f, 0.f};
  }
  bf16x8 ones;
#pragma unroll
  for (int i = 0; i < 8; ++i) ones[i] = (__bf16)1.f;
  const float c = g.scale * kLog2e;

  // ---- staging: thread (key, piece) of K and of V, KP keys ----
  const bool stager = tid < C::kStagers;
  const int skey = tid / C::kPieces, spiece = tid % C::kPieces;
  const int32_t* row_pages = a.bt + (int64_t)(none ? 0 : s) * g.max_blocks;
  // (keys that some row sees, sinks not counted: from any_lo on)
  const int any_lo = sp.i0 - a.window + 1 - sp.gap;
  const int run = a.run, run_mask = (1 << run) - 1;
  // Runs of 2^run keys lie in one page: an entry each, kRuns of them at a time.  (Keys that no
  // row sees may be on no page: any row of the pool stands for them.)
  int seg_end = k_lo;                    // keys before it are in the table, or were
  auto load_segment = [&]() __attribute__((always_inline)) {
    const int from = seg_end;
    const int runs = min(kRuns, (k_hi - from + run_mask) >> run);
    for (int i = tid; i < runs; i += C::kThreads) {
      const int pos = sp.position(from + (i << run)), b = pos / g.bs;
      const uint32_t unit = (uint32_t)min(max(row_pages[b], 0), g.num_pages - 1) * (uint32_t)g.Hkv + (uint32_t)h;
      run_row[i] = unit * (uint32_t)g.bs + (uint32_t)(pos - b * g.bs);     // (a pool has fewer than 2^32 rows)
      if constexpr (Q8)
        run_scale[i] = (uint32_t)((const uint8_t*)a.ksp.p[l])[unit] | (uint32_t)((const uint8_t*)a.vsp.p[l])[unit] << 16;
    }
    seg_end = from + (kRuns << run);
  };
  // before chunk ch is addressed, by all threads
  auto reach = [&](int ch) __attribute__((always_inline)) {
    if (k_lo + ch * kChKeys >= seg_end) {
      // (rare: every earlier copy lands first, as the table's loads are waited for with
      // the compiler's own count)
      wait_vm<0>();
      lds_barrier();
      load_segment();
      lds_barrier();
    }
  };
  // entry of key v, which the table holds
  auto entry_of = [&](int v) __attribute__((always_inline)) { return (v - (seg_end - (kRuns << run))) >> run; };
  auto seen = [&](int v) __attribute__((always_inline)) { return v < k_hi && (v >= any_lo || v < a.sink); };

  // rows: pieces from the pool to LDS, those of one row by adjacent lanes
  int kpiece[KP], vpiece[KP];
#pragma unroll
  for (int i = 0; i < KP; ++i) {
    const int key = skey + i * C::kKeyStep;
    kpiece[i] = (spiece ^ C::swz_k(key & 15)) * 16;
    vpiece[i] = (spiece ^ C::swz_v(key)) * 16;
  }
  const char* const kpool = (const char*)a.kp.p[l];
  const char* const vpool = (const char*)a.vp.p[l];
  auto issue = [&](int ch) __attribute__((always_inline)) {
    char* st = smem[ch % C::kStages];
#pragma unroll
    for (int i = 0; i < KP; ++i) {
      const int v = k_lo + ch * kChKeys + skey + i * C::kKeyStep, there = min(v, k_hi - 1);
      const uint64_t row = (uint64_t)(run_row[entry_of(there)] + (uint32_t)(there & run_mask)) * C::kSrc;
      copy16(kpool + row + kpiece[i], st + (i * W + wave) * 1024);
      // what no row sees may be anything: its weights are 0, its values must be finite
      copy16(seen(v) ? vpool + row + vpiece[i] : (const char*)kZeroRow + vpiece[i], st + C::kTile + (i * W + wave) * 1024);
    }
  };

  // codes: through registers
  uint4 kw[KP], vw[KP];
  uint32_t scales[KP];
  auto fetch = [&](int ch) __attribute__((always_inline)) {
#pragma unroll
    for (int i = 0; i < KP; ++i) {
      const int v = k_lo + ch * kChKeys + skey + i * C::kKeyStep, there = min(v, k_hi - 1);
      const int e = entry_of(there);
      const uint64_t row = (uint64_t)(run_row[e] + (uint32_t)(there & run_mask)) * C::kSrc + spiece * 16;
      kw[i] = *(const uint4*)(kpool + row);
      vw[i] = *(const uint4*)(vpool + row);
      scales[i] = run_scale[Q8 ? e : 0];
    }
  };
  auto stage = [&](int ch) __attribute__((always_inline)) {
#pragma unroll
    for (int i = 0; i < KP; ++i) {
      const int key = skey + i * C::kKeyStep;
      char* const kto = &smem[ch % C::kStages][key * C::kRow];
      char* const vto = kto + C::kTile;
      const int kz = C::swz_k(key & 15), vz = C::swz_v(key);
      const bool live = seen(k_lo + ch * kChKeys + key);
      // (a piece is two octets; odd keys write the second first, so that two keys' lanes
      // write different chunks at a time)
      const int turn = key & 1;
      const uint4 vv = live ? vw[i] : uint4{0, 0, 0, 0};
      const float kscale = q8_scale(scales[i] & 255), vscale = live ? q8_scale(scales[i] >> 16) : 0.f;
      const uint32_t k0 = turn ? kw[i].z : kw[i].x, k1 = turn ? kw[i].w : kw[i].y;
      const uint32_t k2 = turn ? kw[i].x : kw[i].z, k3 = turn ? kw[i].y : kw[i].w;
      const uint32_t v0 = turn ? vv.z : vv.x, v1 = turn ? vv.w : vv.y, v2 = turn ? vv.x : vv.z, v3 = turn ? vv.y : vv.w;
      *(bf16x8*)(kto + (((2 * spiece + turn) ^ kz) * 16)) = q8_octet(k0, k1, kscale);
      *(bf16x8*)(kto + (((2 * spiece + 1 - turn) ^ kz) * 16)) = q8_octet(k2, k3, kscale);
      *(bf16x8*)(vto + (((2 * spiece + turn) ^ vz) * 16)) = q8_octet(v0, v1, vscale);
      *(bf16x8*)(vto + (((2 * spiece + 1 - turn) ^ vz) * 16)) = q8_octet(v2, v3, vscale);
    }
  };

  // A lane's reads of a row's chunks: their offsets differ in the chunk's bits alone, so one
  // is kept and the others are formed where they are used (registers are what the loop is
  // short of).
  static_assert((KS & (KS - 1)) == 0, "XOR of the chunk");
  const int koff = li * C::kRow + (((gq * KS) ^ C::swz_k(li)) * 16);
  const int vrow = 4 * gq + (li >> 2);
  const int voff = C::kTile + vrow * C::kRow + ((((li & 3) >> 1) ^ C::swz_v(vrow)) * 16) + (li & 1) * 8;

  // whether key v is seen by the query whose last key is hi; the window's part alone
  auto within = [&](int v, int hi) __attribute__((always_inline)) { return (uint32_t)(hi - v) < (uint32_t)a.window; };
  auto sees = [&](int v, int hi) __attribute__((always_inline)) { return within(v, hi) || (v <= hi && v < a.sink); };
  floatx4 sv[QT][4];
  auto phase_a = [&](const char* st, int k0, auto masked) __attribute__((always_inline)) {
    int at = koff;
    asm volatile("" : "+v"(at));
#pragma unroll
    for (int kt = 0; kt < 4; ++kt) {
#pragma unroll
      for (int x = 0; x < KS; ++x) {
        const bf16x8 ka = *(const bf16x8*)(st + (at ^ (x * 16)) + kt * 16 * C::kRow);
#pragma unroll
        for (int y = NT - 1; y >= 0; --y)
#pragma unroll
          for (int qt = 0; qt < QT; ++qt)
            sv[qt][kt] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(
                ka, qop[qt][y][x], x == 0 && y == NT - 1 ? floatx4{0.f, 0.f, 0.f, 0.f} : sv[qt][kt], 0, 0, 0);
      }
    }
    // (no key past k_hi is seen: where a split ends inside a chunk, the span does)
    if constexpr (decltype(masked)::value) {
      auto mask = [&](auto with_sinks) __attribute__((always_inline)) {
#pragma unroll
        for (int kt = 0; kt < 4; ++kt) {
          const int v = k0 + kt * 16 + 4 * gq;
#pragma unroll
          for (int qt = 0; qt < QT; ++qt)
#pragma unroll
            for (int r = 0; r < 4; ++r) {
              const bool seen = decltype(with_sinks)::value ? sees(v + r, qhi[qt]) : within(v + r, qhi[qt]);
              if (!seen) sv[qt][kt][r] = kNegInf;
            }
        }
      };
      if (k0 < a.sink) mask(std::true_type{});
      else mask(std::false_type{});
    }
  };
  auto v_operand = [&](const char* st, int at, int jj, int dt) __attribute__((always_inline)) {
    const v4i16 lo = read_tr(st + (at ^ (dt * 32)) + (32 * jj) * C::kRow);
    const v4i16 hi = read_tr(st + (at ^ (dt * 32)) + (32 * jj + 16) * C::kRow);
    bf16x8 va;
    __builtin_memcpy(&va, &lo, 8);
    __builtin_memcpy((char*)&va + 8, &hi, 8);
    return va;
  };
  // Whether a value of the chunk is infinite or NaN.
  auto odd_values = [&](const char* st) __attribute__((always_inline)) {
    uint32_t hit = 0;
    const int at = voff;
#pragma unroll
    for (int jj = 0; jj < 2; ++jj)
#pragma unroll
      for (int dt = 0; dt < DT; ++dt) {
        const uint4 w = __builtin_bit_cast(uint4, v_operand(st, at, jj, dt));
        hit |= ((w.x & 0x7fff7fffu) + 0x00800080u) | ((w.y & 0x7fff7fffu) + 0x00800080u) |
               ((w.z & 0x7fff7fffu) + 0x00800080u) | ((w.w & 0x7fff7fffu) + 0x00800080u);
      }
    return __ballot((hit & 0x80008000u) != 0) != 0ull;
  };
  auto phase_b = [&](const char* st, int k0, auto careful) __attribute__((always_inline)) {
    bf16x8 pb[QT][NT][2];
#pragma unroll
    for (int qt = 0; qt < QT; ++qt) {
      float cmax = kNegInf;
#pragma unroll
      for (int kt = 0; kt < 4; ++kt)
#pragma unroll
        for (int r = 0; r < 4; ++r) cmax = fmaxf(cmax, sv[qt][kt][r]);
      // the reference, one for a query's four lanes, is raised only past a headroom
      if (__ballot(cmax * c > m[qt] + kHeadroom) != 0ull) {
        cmax = fmaxf(cmax, __shfl_xor(cmax, 16, 64));
        cmax = fmaxf(cmax, __shfl_xor(cmax, 32, 64)) * c;
        const float mn = fmaxf(m[qt], cmax);
        const float f = __builtin_amdgcn_exp2f(m[qt] - mn);
        m[qt] = mn;
        lsum[qt] *= f;
#pragma unroll
        for (int dt = 0; dt < DT; ++dt) o[qt][dt] *= f;
      }
      const float mr = m[qt];
#pragma unroll
      for (int jj = 0; jj < 2; ++jj) {
        uint32_t w[4][NT];
#pragma unroll
        for (int i = 0; i < 4; ++i) {
          const floatx4 x = sv[qt][2 * jj + (i >> 1)];
          bf16_term_pairs<false>(__builtin_amdgcn_exp2f(fmaf(x[2 * (i & 1)], c, -mr)),
                                 __builtin_amdgcn_exp2f(fmaf(x[2 * (i & 1) + 1], c, -mr)), w[i]);
        }
#pragma unroll
        for (int y = 0; y < NT; ++y) pb[qt][y][jj] = __builtin_bit_cast(bf16x8, uint4{w[0][y], w[1][y], w[2][y], w[3][y]});
      }
    }
    int at = voff;
    asm volatile("" : "+v"(at));
    if constexpr (NT > 1) {
      // A chunk's products are summed from zero, smallest terms first, and added once: a
      // running sum over thousands of keys is rounded once a chunk, not with each of its six
      // products.
      static_assert(QT == 1, "one tile of rows");
#pragma unroll
      for (int dt = 0; dt < DT; dt += 2) {
        floatx4 part[2] = {{0.f, 0.f, 0.f, 0.f}, {0.f, 0.f, 0.f, 0.f}};
        bf16x8 va[2][2];
#pragma unroll
        for (int i = 0; i < 2; ++i)
#pragma unroll
          for (int jj = 0; jj < 2; ++jj) va[i][jj] = v_operand(st, at, jj, dt + i);
#pragma unroll
        for (int y = NT - 1; y >= 0; --y)
#pragma unroll
          for (int jj = 0; jj < 2; ++jj)
#pragma unroll
            for (int i = 0; i < 2; ++i)
              part[i] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(va[i][jj], pb[0][y][jj], part[i], 0, 0, 0);
        o[0][dt] += part[0];
        o[0][dt + 1] += part[1];
      }
      floatx4 part[2] = {{0.f, 0.f, 0.f, 0.f}, {0.f, 0.f, 0.f, 0.f}};
#pragma unroll
      for (int y = NT - 1; y >= 0; --y)
#pragma unroll
        for (int jj = 0; jj < 2; ++jj) part[jj] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(ones, pb[0][y][jj], part[jj], 0, 0, 0);
      lsum[0] += part[0] + part[1];
    } else {
#pragma unroll
      for (int jj = 0; jj < 2; ++jj) {
#pragma unroll
        for (int dt = 0; dt < DT; ++dt) {
          bf16x8 va = v_operand(st, at, jj, dt);
          if constexpr (decltype(careful)::value) {
            uint32_t w[4];
            __builtin_memcpy(w, &va, 16);
#pragma unroll
            for (int i = 0; i < 4; ++i) {
              if ((w[i] & 0x7f80u) == 0x7f80u) w[i] &= 0xffff0000u;
              if ((w[i] & 0x7f800000u) == 0x7f800000u) w[i] &= 0xffffu;
            }
            __builtin_memcpy(&va, w, 16);
          }
#pragma unroll
          for (int qt = 0; qt < QT; ++qt)
            o[qt][dt] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(va, pb[qt][0][jj], o[qt][dt], 0, 0, 0);
        }
#pragma unroll
        for (int qt = 0; qt < QT; ++qt)
          lsum[qt] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(ones, pb[qt][0][jj], lsum[qt], 0, 0, 0);
      }
      if constexpr (decltype(careful)::value) {
        // the infinite and NaN values that the products left out: added where they are
        // seen (a weight is positive), key by key
#pragma unroll
        for (int qt = 0; qt < QT; ++qt)
#pragma unroll
          for (int dt = 0; dt < DT; ++dt) asm volatile("s_nop 7\n\ts_nop 3" : "+v"(o[qt][dt]));
        for (int key = 0; key < kChKeys && k0 + key < k_hi; ++key) {
          const char* row = st + C::kTile + key * C::kRow + (gq & 1) * 8;
#pragma unroll
          for (int dt = 0; dt < DT; ++dt) {
            const uint2 w = *(const uint2*)(row + (((dt * 2 + (gq >> 1)) ^ C::swz_v(key)) * 16));
#pragma unroll
            for (int r = 0; r < 4; ++r) {
              const uint32_t x = ((r & 2 ? w.y : w.x) >> (16 * (r & 1))) << 16;
              if ((x & 0x7f800000u) == 0x7f800000u)
#pragma unroll
                for (int qt = 0; qt < QT; ++qt)
                  if (sees(k0 + key, qhi[qt])) o[qt][dt][r] += __uint_as_float(x);
            }
          }
        }
      }
    }
  };

  auto walk = [&](auto careful) __attribute__((always_inline)) {
    load_segment();
    // (the query loads are waited for here, not in the loop behind the copies)
#pragma unroll
    for (int qt = 0; qt < QT; ++qt)
#pragma unroll
      for (int y = 0; y < NT; ++y)
#pragma unroll
        for (int x = 0; x < KS; ++x) asm volatile("" : "+v"(qop[qt][y][x]));
    lds_barrier();
    if constexpr (Q8) {
      if (stager) {
        fetch(0);
        stage(0);
        if (n_chunks > 1) fetch(1);      // (kRuns keys at least are in the table)
      }
    } else {
      for (int ch = 0; ch < C::kStages - 1 && ch < n_chunks; ++ch) issue(ch);
    }
    // keys that every row of the wave sees (sinks not counted)
    const int all_lo = wave_hi1 - a.window + 1, all_hi = min(wave_hi0, k_hi - 1);
    for (int ch = 0; ch < n_chunks; ++ch) {
      if constexpr (!Q8) {
        // (the copies of up to two newer chunks may be outstanding)
        const int newer = n_chunks - 1 - ch;
        if (newer >= 2) wait_vm<2 * C::kCopies>();
        else if (newer == 1) wait_vm<C::kCopies>();
        else wait_vm<0>();
      }
      // every wave has written its part of chunk ch, and is done with chunk ch - 1,
      // whose stage is free
      lds_barrier();
      if constexpr (!Q8) {
        if (ch + C::kStages - 1 < n_chunks) {
          reach(ch + C::kStages - 1);
          issue(ch + C::kStages - 1);
        }
      }
      const int k0 = k_lo + ch * kChKeys;
      const char* st = smem[ch % C::kStages];
      // (no row of the wave sees a key past its last, nor one before its first window that
      // is no sink)
      const bool work = k0 <= wave_hi1 && (k0 + kChKeys > wave_hi0 - a.window + 1 || k0 < a.sink);
      const bool masked = k0 < all_lo || k0 + kChKeys - 1 > all_hi;
      if (work) {
        if (masked) phase_a(st, k0, std::true_type{});
        else phase_a(st, k0, std::false_type{});
        // (wait states before the products' results are read past the branches below)
#pragma unroll
        for (int qt = 0; qt < QT; ++qt) asm volatile("s_nop 7\n\ts_nop 3" : "+v"(sv[qt][3]));
      }
      if constexpr (Q8) {
        if (ch + 1 < n_chunks) {
          if (stager) stage(ch + 1);
          if (ch + 2 < n_chunks) {
            reach(ch + 2);
            if (stager) fetch(ch + 2);
          }
        }
      }
      if (work) {
        if (decltype(careful)::value && masked && odd_values(st)) phase_b(st, k0, careful);
        else phase_b(st, k0, std::false_type{});
      }
    }
  };
  if (n_chunks > 0) {
    walk(std::false_type{});
    if constexpr (!Q8) {
      // An infinite or NaN value that a row does not see has met its weight of 0 in the
      // products: where a result is not finite (codes are), all over again with such
      // values apart.  (Looked for in every chunk that some rows see keys of and others do
      // not, it took 12 of 113 us: 4 x 1024 queries in a window of 1024.)
      floatx4 zero[QT];
#pragma unroll
      for (int qt = 0; qt < QT; ++qt) {
        zero[qt] = floatx4{0.f, 0.f, 0.f, 0.f};
#pragma unroll
        for (int dt = 0; dt < DT; ++dt) {
          asm volatile("s_nop 7\n\ts_nop 3" : "+v"(o[qt][dt]));
#pragma unroll
          for (int r = 0; r < 4; ++r) zero[qt][r] = fmaf(o[qt][dt][r], 0.f, zero[qt][r]);
        }
      }
      bool odd = false;
#pragma unroll
      for (int qt = 0; qt < QT; ++qt)
#pragma unroll
        for (int r = 0; r < 4; ++r) odd |= !(zero[qt][r] == 0.f);
      if (__syncthreads_or(odd)) {
#pragma unroll
        for (int qt = 0; qt < QT; ++qt) {
          m[qt] = kMaxFloor;
          lsum[qt] = floatx4{0.f, 0.f, 0.f, 0.f};
#pragma unroll
          for (int dt = 0; dt < DT; ++dt) o[qt][dt] = floatx4{0.f, 0.f, 0.f, 0.f};
        }
        seg_end = k_lo;
        walk(std::true_type{});
      }
    }
  }

  // ---- lane holds O^T[dt*16 + 4*gq + r][query li] ----
#pragma unroll
  for (int qt = 0; qt < QT; ++qt) asm volatile("s_nop 7\n\ts_nop 3" : "+v"(o[qt][DT - 1]), "+v"(lsum[qt]));   // (as above)
  if (splits == 1) {
    // Through LDS, whose stages no wave reads any more: rows of a few lanes' 16 bytes each,
    // where the accumulators would give 8 bytes of 16 rows at a time (16 x 1024 queries in a
    // window of 1024: 395 us so, 380 through LDS).
    constexpr int kOut = D * (NT == 1 ? 2 : 4), kOutChunks = kOut / 16;       // bytes of a row, pieces
    constexpr int kSwz = (kOutChunks < 16 ? kOutChunks : 16) - 1;
    static_assert(W * QT * 16 * kOut <= C::kStages * 2 * C::kTile, "the waves' rows fit the stages");
    lds_barrier();
    char* const mine = smem[0] + wave * (QT * 16 * kOut);
#pragma unroll
    for (int qt = 0; qt < QT; ++qt) {
      const bool some = lsum[qt][0] != 0.f;                   // (no weight: zeros, whatever the values)
      const float inv = 1.f / lsum[qt][0];
      char* const row = mine + (qt * 16 + li) * kOut;
#pragma unroll
      for (int dt = 0; dt < DT; ++dt) {
        const floatx4 v = some ? o[qt][dt] * inv : floatx4{0.f, 0.f, 0.f, 0.f};
        if constexpr (NT == 1) {
          const bf16x2 p = {(__bf16)v[0], (__bf16)v[1]}, q = {(__bf16)v[2], (__bf16)v[3]};
          *(uint2*)(row + (((dt * 2 + (gq >> 1)) ^ (li & kSwz)) * 16) + (gq & 1) * 8) =
              uint2{__builtin_bit_cast(uint32_t, p), __builtin_bit_cast(uint32_t, q)};
        } else {
          *(floatx4*)(row + (((dt * 4 + gq) ^ (li & kSwz)) * 16)) = v;
        }
      }
    }
    asm volatile("s_waitcnt lgkmcnt(0)" ::: "memory");       // (a wave reads its own rows alone)
#pragma unroll
    for (int k = 0; k < QT * 16 * kOutChunks / 64; ++k) {
      const int i = (k * 64 + lane) / kOutChunks, piece = (k * 64 + lane) % kOutChunks;
      const int r = wrow0 + i;
      const uint4 v = *(const uint4*)(mine + i * kOut + ((piece ^ (i & 15 & kSwz)) * 16));
      if (r < R) {
        const int t = r / G;
        *(uint4*)((char*)a.out + (orow + (int64_t)t * g.Hq + (r - t * G)) * kOut + piece * 16) = v;
      }
    }
  } else {
#pragma unroll
    for (int qt = 0; qt < QT; ++qt) {
      const int r = wrow0 + qt * 16 + li;
      if (r >= R) continue;
      // (a split without keys is marked so: its sums are not written)
      const int64_t rec = (first_record + (int64_t)(u * a.n_rt + rb) * splits + split) * kRowsWg + (r - row0);
      if (gq == 0) *(floatx2*)(x.ml + 2 * rec) = floatx2{n_chunks > 0 ? m[qt] : kNegInf, lsum[qt][0]};
      if (n_chunks > 0)
#pragma unroll
        for (int dt = 0; dt < DT; ++dt) *(floatx4*)(x.o + rec * D + dt * 16 + 4 * gq) = o[qt][dt];
    }
  }
}

// The records of split row blocks joined: a workgroup per (layer, sequence, KV head, row
// block) and 64 rows, a wave per 4 rows.
constexpr int kJoinThreads = 1024, kJoinRows = 64;
template <int D, bool OUT_BF16>
__global__ __launch_bounds__(kJoinThreads) void window_join_kernel(WindowHead a, ChunkSplit x, int rows_wg) {
  constexpr int kDPerLane = D / 64, kRowsWave = kJoinRows / (kJoinThreads / 64);
  typedef float floatd __attribute__((ext_vector_type(kDPerLane)));
  const Dims& g = a.g;
  const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
  const uint32_t units = (uint32_t)(a.n_layers * g.Hkv);
  uint32_t rest = blockIdx.x;
  const int rb = rest % (uint32_t)a.n_rt;
  rest /= (uint32_t)a.n_rt;
  const uint32_t u = rest % units;
  const int j = rest / units;
  const int2 of = x.of_seq[j];
  if (of.x <= 1) return;
  const int ns = of.x, R = g.G * a.T;
  const int h = u % (uint32_t)g.Hkv, l = u / (uint32_t)g.Hkv;
  const int row0 = blockIdx.y * kJoinRows + wave * kRowsWave;            // of the block's
  const int64_t rec0 = (of.y + (int64_t)(u * a.n_rt + rb) * ns) * rows_wg + row0;
  float M[kRowsWave], L[kRowsWave], acc[kRowsWave][kDPerLane];
#pragma unroll
  for (int i = 0; i < kRowsWave; ++i) {
    M[i] = kMaxFloor, L[i] = 0.f;
#pragma unroll
    for (int e = 0; e < kDPerLane; ++e) acc[i][e] = 0.f;
  }
  for (int sp = 0; sp < ns; ++sp) {
    floatx2 ml[kRowsWave];
    floatd v[kRowsWave];
#pragma unroll
    for (int i = 0; i < kRowsWave; ++i) {
      const int64_t rec = rec0 + (int64_t)sp * rows_wg + i;
      ml[i] = *(const floatx2*)(x.ml + 2 * rec);
      __builtin_memcpy(&v[i], x.o + rec * D + lane * kDPerLane, sizeof(v[i]));
    }
#pragma unroll
    for (int i = 0; i < kRowsWave; ++i) {
      // (a split without keys wrote no sums; one whose weights are all 0 did, and its values may
      // not be finite, which an unsplit row would show)
      const bool in = ml[i][0] != kNegInf;
      const float mn = in ? fmaxf(M[i], ml[i][0]) : M[i];
      const float f0 = __builtin_amdgcn_exp2f(M[i] - mn), f1 = in ? __builtin_amdgcn_exp2f(ml[i][0] - mn) : 0.f;
      M[i] = mn;
      L[i] = L[i] * f0 + (in ? ml[i][1] * f1 : 0.f);
#pragma unroll
      for (int e = 0; e < kDPerLane; ++e) acc[i][e] = acc[i][e] * f0 + (in ? v[i][e] * f1 : 0.f);
    }
  }
#pragma unroll
  for (int i = 0; i < kRowsWave; ++i) {
    const int r = rb * rows_wg + row0 + i;
    if (r >= R) continue;
    const int t = r / g.G;
    const int64_t at = (((int64_t)l * a.n + j) * a.T + t) * g.Hq + h * g.G + (r - t * g.G);
#pragma unroll
    for (int e = 0; e < kDPerLane; ++e) {
      const float y = L[i] == 0.f ? 0.f : acc[i][e] / L[i];              // (a row that sees no key)
      if constexpr (OUT_BF16) ((__bf16*)a.out)[at * D + lane * kDPerLane + e] = (__bf16)y;
      else ((float*)a.out)[at * D + lane * kDPerLane + e] = y;
    }
  }
}

template <bool Q8, int NT, int QT>
hipError_t launch(int d, const WindowCall& a, const ChunkSplit& sp, unsigned grid, hipStream_t s) {
  if (d == 128) hipLaunchKernelGGL((window_chunk_kernel<Q8, NT, 128, QT>), dim3(grid), dim3(512), 0, s, a, sp);
  else hipLaunchKernelGGL((window_chunk_kernel<Q8, NT, 64, QT>), dim3(grid), dim3(512), 0, s, a, sp);
  return hipGetLastError();
}

// Records that a call's splits write: each split sequence has at most twice the workgroups
// that its share of the CUs is.
constexpr int kMostRecords = 2 * kCUs;

size_t records_bytes(const Geom& g, const WindowChunkPlan& x) { return (size_t)kMostRecords * x.rows_wg * (g.d + 2) * sizeof(float); }

}  // namespace

WindowChunkPlan window_chunk_plan(const Geom& g, int n, int n_layers, int T) {
  WindowChunkPlan x{};
  const int64_t units = (int64_t)n_layers * n * g.Hkv, R = (int64_t)g.G * T;
  x.qt = g.dtype == KARA_F32 || R <= 8 * 16 ? 1 : 2;
  x.rows_wg = 8 * 16 * x.qt;
  x.n_rb = (int)((R + x.rows_wg - 1) / x.rows_wg);
  x.blocks = units * x.n_rb;
  // (two to a CU and more: dealt out longest first)
  x.split = x.blocks < 2 * kCUs && n <= 512;
  return x;
}

// (whether keys may be split goes by the blocks, which a smaller call has fewer of)
size_t window_chunk_workspace(const Geom& g, int n, int n_layers, int T) {
  const WindowChunkPlan x = window_chunk_plan(g, n, n_layers, T);
  return records_bytes(g, x) + (size_t)std::min(n, 512) * sizeof(int2);
}

hipError_t launch_window_chunk(const Geom& g, const WindowCall& a, const WindowChunkPlan& x, bool q8, void* workspace,
                               hipStream_t s) {
  ChunkSplit sp{};
  if (x.split) {
    sp.most = a.n;
    sp.o = (float*)workspace;
    sp.ml = sp.o + (size_t)kMostRecords * x.rows_wg * g.d;
    sp.of_seq = (int2*)(sp.ml + (size_t)kMostRecords * x.rows_wg * 2);
  }
  const unsigned grid = (unsigned)(x.blocks + (x.split ? kCUs : 0));
  hipError_t e;
  if (g.dtype == KARA_F32) e = launch<true, 3, 1>(g.d, a, sp, grid, s);   // (over codes: rows of fp32 are split)
  else if (q8) e = x.qt == 1 ? launch<true, 1, 1>(g.d, a, sp, grid, s) : launch<true, 1, 2>(g.d, a, sp, grid, s);
  else e = x.qt == 1 ? launch<false, 1, 1>(g.d, a, sp, grid, s) : launch<false, 1, 2>(g.d, a, sp, grid, s);
  if (e != hipSuccess || !x.split) return e;
  const dim3 joins((unsigned)x.blocks, (unsigned)(x.rows_wg / kJoinRows));
#define KARA_WINDOW_JOIN(D, B) \
  hipLaunchKernelGGL((window_join_kernel<D, B>), joins, dim3(kJoinThreads), 0, s, (const WindowHead&)a, sp, x.rows_wg)
  if (g.d == 128) {
    if (g.dtype == KARA_F32) KARA_WINDOW_JOIN(128, false);
    else KARA_WINDOW_JOIN(128, true);
  } else {
    if (g.dtype == KARA_F32) KARA_WINDOW_JOIN(64, false);
    else KARA_WINDOW_JOIN(64, true);
  }
#undef KARA_WINDOW_JOIN
  return hipGetLastError();
}

}  // namespace kara

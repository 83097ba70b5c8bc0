// Attention of many query rows over the 4-bit cache (kara_q4_attention): a
// prompt's chunk over what is cached.  Bound by the matrix products.
//
// One workgroup of W waves owns 16 QT W query rows of one (layer, sequence, KV
// head), rows ordered (query, head in group), and walks the keys they see 64 at a
// time.  Its threads fetch a chunk's codes two chunks ahead into registers (16
// bytes, one block of 32 values with its scale, at a time), convert them in hardware
// to bf16 -- exactly -- and write them to the other of two LDS stages while the
// products of the present one run: a chunk is converted once for all rows, with one
// barrier.  From there the products are those of the recompute
// attention: S^T = K Q^T, weights as they stand the B operand of O^T += V^T P^T with
// V through the transposed LDS read, the row sums one more product with ones.
//
// NT: bf16 terms of a query and of a weight (1: bf16 calls; 3: fp32 ones).  bf16 calls
// so round a weight, in the output as in its sum, to bf16: 1.74e-3 of the result against
// 64 bits (4 x 512 queries over 2.5-8.7K) where whole weights give 1.61e-3, mostly the
// output's own rounding; a second term would double V's products.
//
// 16 sequences x 1024 queries over 2.5-8.7K cached, 32/8 heads, bf16: 1320 us, 1035
// TFLOP/s; fp32, 8 x 512: 894 us, 400 TFLOP/s of three products for each.
#include <algorithm>
#include <type_traits>

#include "kara_q4_device.h"

namespace kara {
namespace {

constexpr int kChKeys = 64;
constexpr float kLog2e = 1.4426950408889634f;
constexpr float kNegInf = -__builtin_huge_valf();
constexpr float kMaxFloor = -3.402823466e38f;
constexpr float kHeadroom = 8.f;

template <int D, int W>
struct ChCfg {
  static constexpr int kThreads = W * 64;
  static constexpr int kRow = D * 2;                 // bytes of a row in LDS
  static constexpr int kChunks = kRow / 16;
  static constexpr int kKS = D / 32;                 // products per dot product
  static constexpr int kDT = D / 16;                 // 16-row tiles of O^T
  static constexpr int kTile = kChKeys * kRow;       // a chunk of K, or of V
  static constexpr int kParts = D / kQ4Block;        // blocks of a row
  static constexpr int kStagers = 2 * kChKeys * kParts;   // blocks of a chunk to convert
  static constexpr int kPer = kStagers > kThreads ? kStagers / kThreads : 1;
  // XOR swizzles of a row's 16-byte chunks: those of the recompute attention
  static __device__ __forceinline__ int swz_k(int row) {
    if constexpr (D == 128) return ((row & 3) << 2) | ((row >> 2) & 3);
    return ((row & 3) << 1) | ((row >> 2) & 1);
  }
  static __device__ __forceinline__ int swz_v(int row) { return (2 * (D == 128 ? row : row >> 1)) & (kChunks - 1); }
};

typedef short v4i16 __attribute__((ext_vector_type(4)));
__device__ inline v4i16 read_tr(const char* p) {
  return __builtin_amdgcn_ds_read_tr16_b64_v4i16(
      (__attribute__((address_space(3))) v4i16*)(__attribute__((address_space(3))) char*)p);
}

template <int NT, int D, int QT, int W>
__global__ __launch_bounds__(W * 64, 2) void q4_chunk_kernel(Q4Split a) {
  using C = ChCfg<D, W>;
  constexpr int kRowsWg = W * 16 * QT;
  constexpr int KS = C::kKS, DT = C::kDT;
  __shared__ __attribute__((aligned(16))) char smem[2][2 * C::kTile];
  const Geom& g = a.g;
  const int tid = threadIdx.x, lane = tid & 63;
  const int wave = __builtin_amdgcn_readfirstlane(tid >> 6);
  const int gq = lane >> 4, li = lane & 15;

  // All row blocks and splits of a (layer, sequence, KV head) on one XCD, whose L2
  // then holds its codes once, where the units divide among the 8.
  uint32_t u, rest = blockIdx.x;
  const uint32_t per = (uint32_t)a.n_rt * (uint32_t)a.n_splits;
  const uint32_t units = (uint32_t)(a.n_layers * a.n * g.Hkv);
  if (units % 8 == 0) {
    u = rest / (8 * per) * 8 + rest % 8;
    rest = rest / 8 % per;
  } else {
    u = rest / per;
    rest = rest % per;
  }
  const int split = rest % (uint32_t)a.n_splits;
  const int rb = a.n_rt - 1 - (int)(rest / (uint32_t)a.n_splits);     // the blocks that see most keys first
  const int h = u % (uint32_t)g.Hkv;
  u /= (uint32_t)g.Hkv;
  int j = u % (uint32_t)a.n;
  const int l = u / (uint32_t)a.n;
  // Sequences by length.  Workgroups that wait for a place: the longest first.  Where
  // all are placed at once, two to a CU, the second half the shortest first, so that
  // long ones share a CU with short ones.
  if (a.n > 1 && a.n <= C::kThreads) {
    int* lens = (int*)smem[0];
    int mine = -1;
    if (tid < a.n) {
      const int s0 = a.seqs[tid];
      mine = s0 >= 0 && s0 < g.n_seqs ? a.seq_lens[s0] : 0;
      lens[tid] = mine;
    }
    __syncthreads();
    const int half = W == 8 ? a.n : (a.n + 1) / 2;
    const int want = j < half ? j : a.n - 1 - (j - half);
    if (tid < a.n) {
      int rank = 0;
      for (int o = 0; o < a.n; ++o) rank += lens[o] > mine || (lens[o] == mine && o < tid);
      if (rank == want) lens[a.n] = tid;
    }
    __syncthreads();
    j = __builtin_amdgcn_readfirstlane(lens[a.n]);
    __syncthreads();
  }
  const int s = a.seqs[j];
  const int G = g.G, T = a.T, R = G * T;
  const int len = s >= 0 && s < g.n_seqs ? a.seq_lens[s] : 0;
  const int row0 = rb * kRowsWg;
  const int64_t orow = ((int64_t)l * a.n + j) * T * g.Hq + h * G;
  const bool none = len <= 0 || len > a.max_len;
  const int first = len - T;                               // position of query 0
  const int last_pos = first + (min(row0 + kRowsWg, R) - 1) / G;
  const int k_lo = split * a.split_keys;
  const int k_hi = none ? 0 : min(last_pos + 1, k_lo + a.split_keys);
  const int n_chunks = k_hi > k_lo ? (k_hi - k_lo + kChKeys - 1) / kChKeys : 0;

  // ---- this wave's queries as B operands (lane: query li of each tile) ----
  const int wrow0 = row0 + wave * 16 * QT;
  bf16x8 qop[QT][NT][KS];
  int qpos[QT];
#pragma unroll
  for (int qt = 0; qt < QT; ++qt) {
    const int r = min(wrow0 + qt * 16 + li, R - 1);
    const int t = r / G;
    qpos[qt] = first + t;
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
  const int wave_first_pos = first + min(wrow0, R - 1) / G;
  const int wave_last_pos = first + min(wrow0 + 16 * QT - 1, R - 1) / G;

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

  // ---- staging: thread (K|V, key, block) ----
  constexpr int kHalf = C::kStagers / 2;              // blocks of K, or of V
  const bool stager = tid < C::kStagers;
  const int skey = (tid % kHalf) / C::kParts, sblk = tid % C::kParts;
  const int32_t* row_pages = a.bt + (int64_t)(none ? 0 : s) * g.max_blocks;
  // (keys past the last one repeat it, finite and masked for every query)
  auto pos_of = [&](int ch) __attribute__((always_inline)) { return min(k_lo + ch * kChKeys + skey, k_hi - 1); };
  // (a pool has fewer than 2^32 rows; the page of a chunk is read a chunk before its codes)
  const uint32_t page_rows = (uint32_t)g.Hkv * g.bs, head_row = (uint32_t)h * g.bs;
  uint4 cw[C::kPer];
  uint32_t cscale[C::kPer];
  int page = 0, slot = 0;
  auto look = [&](int ch) __attribute__((always_inline)) {
    const int pos = pos_of(ch), b = a.bs_shift >= 0 ? pos >> a.bs_shift : pos / g.bs;
    slot = pos - b * g.bs;
    page = row_pages[b];
  };
  auto fetch = [&]() __attribute__((always_inline)) {
    const uint64_t row = (uint32_t)min(max(page, 0), g.num_pages - 1) * page_rows + (head_row + slot);
#pragma unroll
    for (int i = 0; i < C::kPer; ++i) {
      const bool is_v = C::kPer == 2 ? i == 1 : tid >= kHalf;
      cw[i] = *(const uint4*)((const char*)(is_v ? a.vp.p[l] : a.kp.p[l]) + row * (D / 2) + sblk * 16);
      cscale[i] = ((const uint8_t*)(is_v ? a.vsp.p[l] : a.ksp.p[l]))[row * C::kParts + sblk];
    }
  };
  // A block's four octets go to LDS in an order that differs by row, so that the 16
  // lanes of four rows write 16 different chunks at a time: octet i ^ (row & 3) at
  // step i, its words exchanged beforehand.
  const int turn = skey & 3;
  auto stage = [&](int st) __attribute__((always_inline)) {
#pragma unroll
    for (int y = 0; y < C::kPer; ++y) {
      const bool is_v = C::kPer == 2 ? y == 1 : tid >= kHalf;
      char* const to = &smem[st][(is_v ? C::kTile : 0) + skey * C::kRow];
      const int swz = is_v ? C::swz_v(skey) : C::swz_k(skey & 15);
      const float scale = q4_scale(cscale[y]);
      uint32_t w0 = cw[y].x, w1 = cw[y].y, w2 = cw[y].z, w3 = cw[y].w;
      {
        const uint32_t a0 = turn & 1 ? w1 : w0, a1 = turn & 1 ? w0 : w1, a2 = turn & 1 ? w3 : w2, a3 = turn & 1 ? w2 : w3;
        w0 = turn & 2 ? a2 : a0, w1 = turn & 2 ? a3 : a1, w2 = turn & 2 ? a0 : a2, w3 = turn & 2 ? a1 : a3;
      }
      const uint32_t w[4] = {w0, w1, w2, w3};
#pragma unroll
      for (int i = 0; i < 4; ++i) {
        const bf16x8 v = q4_octet(w[i], scale);
        *(bf16x8*)(to + (((sblk * 4 + (i ^ turn)) ^ swz) * 16)) = v;
      }
    }
  };

  int koff[KS], voff[DT];
#pragma unroll
  for (int x = 0; x < KS; ++x) koff[x] = li * C::kRow + (((gq * KS + x) ^ C::swz_k(li)) * 16);
  {
    const int vrow = 4 * gq + (li >> 2);
#pragma unroll
    for (int dt = 0; dt < DT; ++dt)
      voff[dt] = C::kTile + vrow * C::kRow + (((dt * 2 + ((li & 3) >> 1)) ^ C::swz_v(vrow)) * 16) + (li & 1) * 8;
  }

  floatx4 sv[QT][4];
  auto phase_a = [&](const char* st, int k0, auto masked) __attribute__((always_inline)) {
#pragma unroll
    for (int kt = 0; kt < 4; ++kt) {
#pragma unroll
      for (int qt = 0; qt < QT; ++qt) sv[qt][kt] = floatx4{0.f, 0.f, 0.f, 0.f};
#pragma unroll
      for (int x = 0; x < KS; ++x) {
        const bf16x8 ka = *(const bf16x8*)(st + koff[x] + kt * 16 * C::kRow);
#pragma unroll
        for (int y = NT - 1; y >= 0; --y)
#pragma unroll
          for (int qt = 0; qt < QT; ++qt)
            sv[qt][kt] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(ka, qop[qt][y][x], sv[qt][kt], 0, 0, 0);
      }
    }
    if constexpr (decltype(masked)::value) {
#pragma unroll
      for (int qt = 0; qt < QT; ++qt)
#pragma unroll
        for (int kt = 0; kt < 4; ++kt)
#pragma unroll
          for (int r = 0; r < 4; ++r)
            if (k0 + kt * 16 + 4 * gq + r > min(qpos[qt], k_hi - 1)) sv[qt][kt][r] = kNegInf;
    }
  };
  auto phase_b = [&](const char* st) __attribute__((always_inline)) {
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
    auto v_operand = [&](int jj, int dt) __attribute__((always_inline)) {
      const v4i16 lo = read_tr(st + voff[dt] + (32 * jj) * C::kRow);
      const v4i16 hi = read_tr(st + voff[dt] + (32 * jj + 16) * C::kRow);
      bf16x8 va;
      __builtin_memcpy(&va, &lo, 8);
      __builtin_memcpy((char*)&va + 8, &hi, 8);
      return va;
    };
    if constexpr (NT > 1) {
      // A chunk's products are summed from zero, smallest terms first, and added once: a
      // running sum over thousands of keys is rounded once a chunk, not with each of its six
      // products (4 x 512 queries over 2.5-8.7K tokens: off by 4.3e-7 of the result where six
      // roundings a chunk leave 2.0e-6, 444 us against 424).
      static_assert(QT == 1, "one tile of rows");
#pragma unroll
      for (int dt = 0; dt < DT; dt += 2) {
        floatx4 part[2] = {{0.f, 0.f, 0.f, 0.f}, {0.f, 0.f, 0.f, 0.f}};
        bf16x8 va[2][2];
#pragma unroll
        for (int i = 0; i < 2; ++i)
#pragma unroll
          for (int jj = 0; jj < 2; ++jj) va[i][jj] = v_operand(jj, dt + i);
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
          const bf16x8 va = v_operand(jj, dt);
#pragma unroll
          for (int qt = 0; qt < QT; ++qt)
            o[qt][dt] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(va, pb[qt][0][jj], o[qt][dt], 0, 0, 0);
        }
#pragma unroll
        for (int qt = 0; qt < QT; ++qt)
          lsum[qt] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(ones, pb[qt][0][jj], lsum[qt], 0, 0, 0);
      }
    }
  };

  if (n_chunks > 0) {
    if (stager) {
      look(0);
      fetch();
      stage(0);
      if (n_chunks > 1) {
        look(1);
        fetch();
      }
      if (n_chunks > 2) look(2);
    }
    auto step = [&](int ch, auto masked) __attribute__((always_inline)) {
      // every wave has written its part of chunk ch, and is done with chunk ch - 1,
      // whose stage takes chunk ch + 1
      __syncthreads();
      const int k0 = k_lo + ch * kChKeys;
      const char* st = smem[ch & 1];
      const bool work = k0 <= wave_last_pos;
      if (work) {
        phase_a(st, k0, masked);
        // (wait states before the products' results are read past the branches below)
#pragma unroll
        for (int qt = 0; qt < QT; ++qt) asm volatile("s_nop 7\n\ts_nop 3" : "+v"(sv[qt][3]));
      }
      if (stager && ch + 1 < n_chunks) {
        stage((ch + 1) & 1);
        if (ch + 2 < n_chunks) fetch();
        if (ch + 3 < n_chunks) look(ch + 3);
      }
      if (work) phase_b(st);
    };
    // chunks in which every key is seen by every row of the wave, then the others
    const int whole = min(k_hi, wave_first_pos + 1) - k_lo;
    const int first_masked = min(n_chunks, max(whole, 0) / kChKeys);
    int ch = 0;
    for (; ch < first_masked; ++ch) step(ch, std::false_type{});
    for (; ch < n_chunks; ++ch) step(ch, std::true_type{});
  }

  // ---- lane holds O^T[dt*16 + 4*gq + r][query li] ----
#pragma unroll
  for (int qt = 0; qt < QT; ++qt) asm volatile("s_nop 7\n\ts_nop 3" : "+v"(o[qt][DT - 1]), "+v"(lsum[qt]));   // (as above)
#pragma unroll
  for (int qt = 0; qt < QT; ++qt) {
    const int r = wrow0 + qt * 16 + li;
    if (r >= R) continue;
    const int t = r / G;
    const int64_t at = orow + (int64_t)t * g.Hq + (r - t * G);
    if (a.n_splits == 1) {
      const float inv = lsum[qt][0] == 0.f ? 0.f : 1.f / lsum[qt][0];    // (a row that sees no key)
#pragma unroll
      for (int dt = 0; dt < DT; ++dt) {
        const floatx4 v = o[qt][dt] * inv;
        if (a.out_bf16) {
          const bf16x2 x = {(__bf16)v[0], (__bf16)v[1]}, y = {(__bf16)v[2], (__bf16)v[3]};
          *(uint2*)((__bf16*)a.out + at * D + dt * 16 + 4 * gq) =
              uint2{__builtin_bit_cast(uint32_t, x), __builtin_bit_cast(uint32_t, y)};
        } else {
          *(floatx4*)((float*)a.out + at * D + dt * 16 + 4 * gq) = v;
        }
      }
    } else if (!none && k_lo < len) {
      const int64_t rec = at * a.n_splits + split;
      if (gq == 0) *(floatx2*)(a.rec_ml + 2 * rec) = floatx2{m[qt], lsum[qt][0]};
#pragma unroll
      for (int dt = 0; dt < DT; ++dt) *(floatx4*)(a.rec_o + rec * D + dt * 16 + 4 * gq) = o[qt][dt];
    }
  }
}

template <int NT, int QT, int W>
hipError_t launch(const Q4Split& a, int64_t blocks, hipStream_t stream) {
  if (a.g.d == 128) hipLaunchKernelGGL((q4_chunk_kernel<NT, 128, QT, W>), dim3((unsigned)blocks), dim3(W * 64), 0, stream, a);
  else hipLaunchKernelGGL((q4_chunk_kernel<NT, 64, QT, W>), dim3((unsigned)blocks), dim3(W * 64), 0, stream, a);
  return hipGetLastError();
}

constexpr int kCUs = 256;

}  // namespace

// Rows per workgroup, key splits and blocks of a call.
Q4ChunkPlan q4_chunk_plan(const Geom& g, int n, int n_layers, int T, int max_len) {
  Q4ChunkPlan x{};
  const int64_t units = (int64_t)n_layers * n * g.Hkv, R = (int64_t)g.G * T;
  x.qt = g.dtype == KARA_F32 || R <= 8 * 16 ? 1 : 2;
  auto blocks = [&](int waves) { return units * ((R + waves * 16 * x.qt - 1) / (waves * 16 * x.qt)); };
  // Eight waves, a CU's worth of registers, convert a chunk once for 256 rows (bf16)
  // but stand one to a CU: a launch of half to all of the CUs' number ends with its
  // longest.  There four waves, two to a CU, lengths of 2.5-8.7K: 4 x 512 queries,
  // 256 blocks: 268 -> 215 us; 16 x 128: 272 -> 216; 5 x 512, 320 blocks: 270 -> 229;
  // 6 x 512, 384 blocks: 276 against 316.  (Lengths are not known here: 4 x 512 over
  // 8.7K each lose, 272 -> 291.  Below 128 blocks keys are split, to the same number
  // of workgroups either way.)
  x.waves = blocks(8) * 2 > kCUs && blocks(8) <= kCUs * 5 / 4 ? 4 : 8;
  x.rows_wg = x.waves * 16 * x.qt;
  x.n_rb = (int)((R + x.rows_wg - 1) / x.rows_wg);
  x.splits = 1;
  // (fewer workgroups than CUs: their keys are split, down to 512)
  if (x.waves == 8)
    while (x.splits < 16 && units * x.n_rb * x.splits * 2 <= kQ4ChunkWgs && max_len > 512 * x.splits) x.splits *= 2;
  x.split_keys = x.splits == 1 ? max_len : ((max_len + x.splits - 1) / x.splits + kChKeys - 1) / kChKeys * kChKeys;
  x.splits = (max_len + x.split_keys - 1) / x.split_keys;
  x.blocks = units * x.n_rb * x.splits;
  return x;
}

hipError_t launch_q4_chunk(Q4Split a, const Q4ChunkPlan& x, hipStream_t stream) {
  a.bs_shift = (a.g.bs & (a.g.bs - 1)) == 0 ? __builtin_ctz((unsigned)a.g.bs) : -1;
  if (a.g.dtype == KARA_F32) return x.waves == 8 ? launch<3, 1, 8>(a, x.blocks, stream) : launch<3, 1, 4>(a, x.blocks, stream);
  if (x.qt == 1) return x.waves == 8 ? launch<1, 1, 8>(a, x.blocks, stream) : launch<1, 1, 4>(a, x.blocks, stream);
  return x.waves == 8 ? launch<1, 2, 8>(a, x.blocks, stream) : launch<1, 2, 4>(a, x.blocks, stream);
}

}  // namespace kara

// kara_evict_observe: the softmax weights that many queries give to the cached
// keys, summed per key (include/kara_evict.h).  Two sweeps over q . k, as the
// weights need the rows' sums first: row statistics (each row's maximum and sum of
// exponentials), then column sums with K held and the queries streamed.  No V, no
// atomics: every key's sum is formed by one workgroup, in row order.
#include <algorithm>

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

struct ObserveArgs {
  Geom g;
  int n, T, n_new, max_len;
  int row_blocks, splits, split_keys;   // row statistics
  int key_blocks;                       // column sums
  const int32_t *seqs, *bt, *seq_lens;
  const void* q;                        // [n_layers][n][T][Hq][d]
  PoolPtrs k, ks;
  float* w[kMaxLayersPerLaunch];
  floatx2* stats;                       // [n_layers][n][Hkv][T * G][splits]: maximum (log2 units), sum
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
        bf16_term_pairs(__uint_as_float(v[i >> 1][2 * i & 3]), __uint_as_float(v[i >> 1][(2 * i & 3) + 1]), w[i]);
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

constexpr int kObsThreads = 256;
constexpr int kObsWaves = kObsThreads / 64;
constexpr int kChunk = 64;                  // rows staged at a time

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
__device__ __forceinline__ bool unit_of(const ObserveArgs& a, int64_t u, Unit* x) {
  const Geom& g = a.g;
  x->h = (int)(u % g.Hkv);
  x->j = (int)((u / g.Hkv) % a.n);
  x->l = (int)(u / ((int64_t)g.Hkv * a.n));
  x->s = a.seqs[x->j];
  x->len = x->s >= 0 && x->s < g.n_seqs ? a.seq_lens[x->s] : 0;
  return x->len > 0 && x->len <= a.max_len;
}

__device__ __forceinline__ uint64_t key_row(const Geom& g, const int32_t* row_pages, int h, int pos) {
  const int b = pos / g.bs;
  const int page = min(max(row_pages[b], 0), g.num_pages - 1);
  return (uint64_t)(((int64_t)page * g.Hkv + h) * g.bs + (pos - b * g.bs));
}

// ---- row statistics: one workgroup per (unit, 128 query rows, split of the keys);
// a wave holds 32 rows, the keys pass through LDS 64 at a time
constexpr int kStatRows = kObsWaves * 32;

template <int KSRC, int NK, int QSRC, int NQ, int D>
__global__ __launch_bounds__(kObsThreads) void observe_stats_kernel(ObserveArgs a) {
  constexpr int KS = D / 32, kOct = D / 8, kPer = kChunk * kOct / kObsThreads;
  __shared__ ChunkLds<NK, D> lds;
  const Geom& g = a.g;
  const int tid = threadIdx.x, lane = tid & 63;
  const int wave = __builtin_amdgcn_readfirstlane(tid >> 6);
  const int gq = lane >> 4, li = lane & 15;
  const int split = blockIdx.x % a.splits;
  const int rb = (blockIdx.x / a.splits) % a.row_blocks;
  const int64_t u = blockIdx.x / (a.splits * a.row_blocks);
  Unit x;
  if (!unit_of(a, u, &x)) return;
  const int G = g.G, R = G * a.T;
  const int row0 = rb * kStatRows;
  const int first = x.len - a.T;                       // position of query 0
  const int last_pos = first + (min(row0 + kStatRows, R) - 1) / G;
  const int k_lo = split * a.split_keys;
  const int k_hi = min(min(x.len, last_pos + 1), k_lo + a.split_keys);
  const int32_t* row_pages = a.bt + (int64_t)x.s * g.max_blocks;
  const int wrow0 = row0 + wave * 32;
  const int wfirst = first + min(wrow0, R - 1) / G, wlast = first + min(wrow0 + 31, R - 1) / G;

  bf16x8 qa[2][NQ][KS];
  int qpos[2];
#pragma unroll
  for (int t = 0; t < 2; ++t) {
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
  float m[2] = {kMaxFloor, kMaxFloor}, sum[2] = {0.f, 0.f};    // of this lane's keys
  const float c = g.scale * kLog2e;

  Octet<KSRC> pre[kPer];
  auto fetch = [&](int k0) __attribute__((always_inline)) {
#pragma unroll
    for (int i = 0; i < kPer; ++i) {
      const int slot = i * kObsThreads + tid;
      const int pos = min(k0 + slot / kOct, k_hi - 1);         // (past the end: the last key, masked)
      pre[i].load(a.k.p[x.l], a.ks.p[x.l], key_row(g, row_pages, x.h, pos), slot % kOct, D);
    }
  };
  if (k_lo < k_hi) {
    fetch(k_lo);
    int buf = 0;
    for (int k0 = k_lo; k0 < k_hi; k0 += kChunk, buf ^= 1) {
#pragma unroll
      for (int i = 0; i < kPer; ++i) {
        const int slot = i * kObsThreads + tid, row = slot / kOct, o = slot % kOct;
        bf16x8 t[NK];
        pre[i].terms(t);
#pragma unroll
        for (int y = 0; y < NK; ++y) __builtin_memcpy(&lds.b[buf][y][row * D * 2 + ((o ^ swz<D>(row & 15)) * 16)], &t[y], 16);
      }
      if (k0 + kChunk < k_hi) fetch(k0 + kChunk);
      __syncthreads();
      if (k0 <= wlast) {
        const bool masked = k0 + kChunk > min(k_hi, wfirst + 1);
        floatx4 sv[2][4];
#pragma unroll
        for (int kt = 0; kt < 4; ++kt) {
          bf16x8 ka[NK][KS];
          read_tile<NK, D>(lds.b[buf], kt * 16, gq, li, ka);
#pragma unroll
          for (int t = 0; t < 2; ++t) sv[t][kt] = dot_tile<NK, NQ, KS>(ka, qa[t]);
        }
        // (wait states before the results are read past a branch)
        asm volatile("s_nop 7\n\ts_nop 3" : "+v"(sv[0][3]), "+v"(sv[1][3]));
#pragma unroll
        for (int t = 0; t < 2; ++t) {
          if (masked) {
#pragma unroll
            for (int kt = 0; kt < 4; ++kt)
#pragma unroll
              for (int r = 0; r < 4; ++r)
                if (k0 + kt * 16 + 4 * gq + r >= min(k_hi, qpos[t] + 1)) sv[t][kt][r] = kNegInf;
          }
          float mx = sv[t][0][0];
#pragma unroll
          for (int kt = 0; kt < 4; ++kt)
#pragma unroll
            for (int r = 0; r < 4; ++r) mx = fmaxf(mx, sv[t][kt][r]);
          const float mn = fmaxf(m[t], mx * c);
          float add = 0.f;
#pragma unroll
          for (int kt = 0; kt < 4; ++kt)
#pragma unroll
            for (int r = 0; r < 4; ++r) add += __builtin_amdgcn_exp2f(fmaf(sv[t][kt][r], c, -mn));
          sum[t] = fmaf(sum[t], __builtin_amdgcn_exp2f(m[t] - mn), add);
          m[t] = mn;
        }
      }
    }
  }
#pragma unroll
  for (int t = 0; t < 2; ++t) {
    float M = fmaxf(m[t], __shfl_xor(m[t], 16, 64));
    M = fmaxf(M, __shfl_xor(M, 32, 64));
    float L = sum[t] * __builtin_amdgcn_exp2f(m[t] - M);
    L += __shfl_xor(L, 16, 64);
    L += __shfl_xor(L, 32, 64);
    const int r = wrow0 + t * 16 + li;
    if (gq == 0 && r < R) a.stats[(u * R + r) * a.splits + split] = floatx2{M, L};
  }
}

// ---- column sums: one workgroup per (unit, 128 keys); a wave holds 32 keys, the
// query rows that see them pass through LDS 64 at a time
constexpr int kSumKeys = kObsWaves * 32;

template <int KSRC, int NK, int QSRC, int NQ, int D>
__global__ __launch_bounds__(kObsThreads) void observe_sum_kernel(ObserveArgs a) {
  constexpr int KS = D / 32, kOct = D / 8, kPer = kChunk * kOct / kObsThreads;
  __shared__ ChunkLds<NQ, D> lds;
  __shared__ float row_m[2][kChunk], row_i[2][kChunk];
  const Geom& g = a.g;
  const int tid = threadIdx.x, lane = tid & 63;
  const int wave = __builtin_amdgcn_readfirstlane(tid >> 6);
  const int gq = lane >> 4, li = lane & 15;
  const int kb = blockIdx.x % a.key_blocks;
  const int64_t u = blockIdx.x / a.key_blocks;
  Unit x;
  if (!unit_of(a, u, &x)) return;
  const int key0 = kb * kSumKeys;
  if (key0 >= x.len) return;
  int dup = 0;
  for (int o = tid; o < x.j; o += kObsThreads) dup |= a.seqs[o] == x.s;
  if (__syncthreads_or(dup)) return;                   // an earlier listing counts
  const int G = g.G, R = G * a.T;
  const int first = x.len - a.T;
  const int32_t* row_pages = a.bt + (int64_t)x.s * g.max_blocks;
  const int wkey0 = key0 + wave * 32;

  bf16x8 ka[2][NK][KS];
#pragma unroll
  for (int t = 0; t < 2; ++t) {
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
  floatx4 acc[2] = {floatx4{0.f, 0.f, 0.f, 0.f}, floatx4{0.f, 0.f, 0.f, 0.f}};
  const float c = g.scale * kLog2e;
  // the first row that sees this workgroup's first key
  const int r_lo = max(0, max(key0, 0) - first) * G;

  Octet<QSRC> pre[kPer];
  float pm = 0.f, pi = 0.f;
  auto fetch = [&](int r0) __attribute__((always_inline)) {
#pragma unroll
    for (int i = 0; i < kPer; ++i) {
      const int slot = i * kObsThreads + tid;
      const int r = min(r0 + slot / kOct, R - 1), qt = r / G;
      const uint64_t row = (((uint64_t)x.l * a.n + x.j) * a.T + qt) * g.Hq + x.h * G + (r - qt * G);
      pre[i].load(a.q, nullptr, row, slot % kOct, D);
    }
    if (tid < kChunk) {
      pm = 0.f, pi = 0.f;
      if (r0 + tid < R) {
        const floatx2* st = a.stats + (u * R + r0 + tid) * a.splits;
        pm = kMaxFloor;
        for (int i = 0; i < a.splits; ++i) pm = fmaxf(pm, st[i][0]);
        float L = 0.f;
        for (int i = 0; i < a.splits; ++i) L += st[i][1] * __builtin_amdgcn_exp2f(st[i][0] - pm);
        pi = 1.f / L;
      }
    }
  };
  if (r_lo < R) {
    fetch(r_lo);
    int buf = 0;
    for (int r0 = r_lo; r0 < R; r0 += kChunk, buf ^= 1) {
#pragma unroll
      for (int i = 0; i < kPer; ++i) {
        const int slot = i * kObsThreads + tid, row = slot / kOct, o = slot % kOct;
        bf16x8 t[NQ];
        pre[i].terms(t);
#pragma unroll
        for (int y = 0; y < NQ; ++y) __builtin_memcpy(&lds.b[buf][y][row * D * 2 + ((o ^ swz<D>(row & 15)) * 16)], &t[y], 16);
      }
      if (tid < kChunk) row_m[buf][tid] = pm, row_i[buf][tid] = pi;
      if (r0 + kChunk < R) fetch(r0 + kChunk);
      __syncthreads();
#pragma unroll
      for (int rt = 0; rt < 4; ++rt) {
        const int last = first + min(r0 + rt * 16 + 15, R - 1) / G;
        if (r0 + rt * 16 >= R || last < wkey0) continue;          // (uniform in the wave)
        bf16x8 qb[NQ][KS];
        read_tile<NQ, D>(lds.b[buf], rt * 16, gq, li, qb);
        const float rm = row_m[buf][rt * 16 + li], ri = row_i[buf][rt * 16 + li];
        const int pos = r0 + rt * 16 + li < R ? first + (r0 + rt * 16 + li) / G : -1;    // (past the last row: sees none)
        floatx4 sv[2];
#pragma unroll
        for (int t = 0; t < 2; ++t) sv[t] = dot_tile<NK, NQ, KS>(ka[t], qb);
        asm volatile("s_nop 7\n\ts_nop 3" : "+v"(sv[0]), "+v"(sv[1]));
#pragma unroll
        for (int t = 0; t < 2; ++t)
#pragma unroll
          for (int r = 0; r < 4; ++r) {
            const float p = __builtin_amdgcn_exp2f(fmaf(sv[t][r], c, -rm));
            // (a row that sees none of these keys may have no sum: its weight is dropped, not multiplied by 0)
            acc[t][r] += wkey0 + t * 16 + 4 * gq + r > pos ? 0.f : p * ri;
          }
      }
    }
  }
#pragma unroll
  for (int t = 0; t < 2; ++t)
#pragma unroll
    for (int r = 0; r < 4; ++r) {
      float v = acc[t][r];
#pragma unroll
      for (int y = 1; y < 16; y <<= 1) v += __shfl_xor(v, y, 64);
      const int pos = wkey0 + t * 16 + 4 * gq + r;
      if (li != 0 || pos >= x.len) continue;
      const int b = pos / g.bs, page = row_pages[b];
      if (page < 0 || page >= g.num_pages) continue;
      float* to = a.w[x.l] + ((int64_t)page * g.Hkv + x.h) * g.bs + (pos - b * g.bs);
      *to = pos >= x.len - a.n_new ? v : *to + v;
    }
}

bool grid_ok(int64_t blocks) { return blocks > 0 && blocks < ((int64_t)1 << 24); }

// Splits of the keys for the row statistics: enough workgroups for the chip where
// rows are few, none shorter than 512 keys.
int stat_splits(int64_t blocks, int max_len) {
  int splits = 1;
  while (splits < 16 && blocks * splits < 1024 && max_len > splits * 2 * 512) splits *= 2;
  return splits;
}

struct Plan {
  int row_blocks, splits, split_keys, key_blocks;
  int64_t units;
  size_t bytes;
};

Plan plan_of(const Geom& g, int n, int n_layers, int T, int max_len) {
  Plan x{};
  x.units = (int64_t)n_layers * n * g.Hkv;
  const int64_t R = (int64_t)g.G * T;
  x.row_blocks = (int)((R + kStatRows - 1) / kStatRows);
  x.splits = stat_splits(x.units * x.row_blocks, max_len);
  x.split_keys = ((max_len + x.splits - 1) / x.splits + kChunk - 1) / kChunk * kChunk;
  x.key_blocks = (max_len + kSumKeys - 1) / kSumKeys;
  x.bytes = (size_t)(x.units * R * x.splits) * sizeof(floatx2);
  return x;
}

template <int KSRC, int NK, int QSRC, int NQ, int D>
hipError_t launch(const ObserveArgs& a, const Plan& x, hipStream_t stream) {
  hipLaunchKernelGGL((observe_stats_kernel<KSRC, NK, QSRC, NQ, D>), dim3((unsigned)(x.units * x.row_blocks * x.splits)),
                     dim3(kObsThreads), 0, stream, a);
  const hipError_t e = hipGetLastError();
  if (e != hipSuccess) return e;
  hipLaunchKernelGGL((observe_sum_kernel<KSRC, NK, QSRC, NQ, D>), dim3((unsigned)(x.units * x.key_blocks)),
                     dim3(kObsThreads), 0, stream, a);
  return hipGetLastError();
}

template <int D>
hipError_t launch_d(const ObserveArgs& a, const Plan& x, bool codes, hipStream_t stream) {
  const bool f32 = a.g.dtype == KARA_F32;
  if (codes) return f32 ? launch<kCodeRows, 1, kF32Rows, 3, D>(a, x, stream) : launch<kCodeRows, 1, kBf16Rows, 1, D>(a, x, stream);
  return f32 ? launch<kF32Rows, 3, kF32Rows, 3, D>(a, x, stream) : launch<kBf16Rows, 1, kBf16Rows, 1, D>(a, x, stream);
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
  // (a launch of 1024 row blocks or more does not split; a smaller one has at most
  // twice 1024 of them, records and all)
  const int64_t R = (int64_t)g.G * n_query;
  const int64_t rows = (int64_t)n_layers * n * g.Hkv * R;
  *bytes = (size_t)(rows + (int64_t)2048 * kStatRows) * sizeof(floatx2);
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
  const Plan x = plan_of(a.g, n, n_layers, n_query, max_len);
  if (!workspace || workspace_bytes < x.bytes) return KARA_ERR_WORKSPACE;
  if (!grid_ok(x.units * x.row_blocks * x.splits) || !grid_ok(x.units * x.key_blocks)) return KARA_ERR_UNSUPPORTED;
  a.n = n;
  a.T = n_query;
  a.n_new = n_new;
  a.max_len = max_len;
  a.row_blocks = x.row_blocks;
  a.splits = x.splits;
  a.split_keys = x.split_keys;
  a.key_blocks = x.key_blocks;
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
  const hipError_t e = a.g.d == 128 ? launch_d<128>(a, x, k_scales != nullptr, (hipStream_t)stream)
                                    : launch_d<64>(a, x, k_scales != nullptr, (hipStream_t)stream);
  return hip_status(e);
}

}  // extern "C"

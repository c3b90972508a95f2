// Attention weight that each cached position receives from the queries of a call, for
// gfx950:
//
//   W[j] (+)= sum over rows r that see key j of 2^(q_r k_j c - l_r),
//   c = log2(e) / sqrt(D), l_r = log2(e) lse_r,
//
// the probabilities recomputed from the log-sum-exp that attention returned.  A block
// holds 128 or 256 keys of one kv head as matrix operands in registers and takes the
// query rows past them, 64 at a time through LDS, so a key is read once for every
// split of the rows and the sums stay in registers: S = Q K^T with a key per
// lane (32x32 products), the 16 rows a lane has of each product added up there, the two
// lanes of a key joined at the end.  No atomics: the same call gives the same bits.
//
// Where a call has few keys and many rows, its rows are cut into splits that leave
// partials, added in their order by weights_merge_kernel.
//
// What bounds it: with many rows the issue of instructions.  Of 234K cycles a SIMD, 2048
// tokens of 32 heads past 6007 shared keys take 99K in the matrix unit and 126K in the
// others (an exponential for each pair of row and key is 8 cycles, its sum and
// scale more), and the two hardly overlap though nothing waits between them: 127 us a call, 810
// TFLOP/s of the products.  More keys a block share a row's reads from LDS (KN = 1: 158 us); a
// third or fourth wave a SIMD does not fit the registers.  With few rows the latency of a block: its
// keys, then its tiles of rows one after the other (one token each of 64 sequences past 4321
// keys, four tiles in a block of the prefix, one of four rows in a block of own keys: 11.9 us).
//
// fp32 caches: the same on 32x32x2 products, four for each 16-byte vector (elements e of
// the two lanes' vectors together make a product's depth of two; the order of the head's
// elements in a sum is free).
#include "fcg_device.hpp"
#include "kernels.hpp"

namespace fcg {

namespace {

typedef __bf16 wt_bf16x8 __attribute__((ext_vector_type(8)));
typedef float wt_f32x16 __attribute__((ext_vector_type(16)));

template <typename T>
__device__ __forceinline__ wt_f32x16 mma(const uint4& a, const uint4& b, wt_f32x16 c);
template <>
__device__ __forceinline__ wt_f32x16 mma<bf16_t>(const uint4& a, const uint4& b, wt_f32x16 c) {
  return __builtin_amdgcn_mfma_f32_32x32x16_bf16(__builtin_bit_cast(wt_bf16x8, a), __builtin_bit_cast(wt_bf16x8, b), c,
                                                 0, 0, 0);
}
template <>
__device__ __forceinline__ wt_f32x16 mma<float>(const uint4& a, const uint4& b, wt_f32x16 c) {
  c = __builtin_amdgcn_mfma_f32_32x32x2f32(__uint_as_float(a.x), __uint_as_float(b.x), c, 0, 0, 0);
  c = __builtin_amdgcn_mfma_f32_32x32x2f32(__uint_as_float(a.y), __uint_as_float(b.y), c, 0, 0, 0);
  c = __builtin_amdgcn_mfma_f32_32x32x2f32(__uint_as_float(a.z), __uint_as_float(b.z), c, 0, 0, 0);
  return __builtin_amdgcn_mfma_f32_32x32x2f32(__uint_as_float(a.w), __uint_as_float(b.w), c, 0, 0, 0);
}

constexpr int kTileRows = 64;  // query rows of an LDS tile

// The plan of a call: in device memory, or by value.
template <bool VALUE>
struct Plan {};
template <>
struct Plan<false> {
  const WeightItem* items;
  const WeightRank* ranks;
  __device__ __forceinline__ WeightItem item(int b) const { return items[b]; }
  __device__ __forceinline__ WeightRank rank(int r) const { return ranks[r]; }
};
template <>
struct Plan<true> {
  WeightArgs a;
  __device__ __forceinline__ WeightItem item(int b) const {
    if (b < a.n_pre) return cut(a.pre, b);
    // the group is the last one whose first item is at most b
    static_assert(kWgtGroups == 64, "one group per lane");
    const int lane = threadIdx.x & 63;
    const WeightGroup mine = a.group[min(lane, a.n_group - 1)];
    const uint64_t below = __builtin_amdgcn_ballot_w64(lane < a.n_group && mine.item0 <= b);
    const int r = 63 - __builtin_clzll(below);
    WeightGroup x;
    x.seq = __builtin_amdgcn_readlane(mine.seq, r);
    x.lo = __builtin_amdgcn_readlane(mine.lo, r);
    x.hi = __builtin_amdgcn_readlane(mine.hi, r);
    x.row0 = __builtin_amdgcn_readlane(mine.row0, r);
    x.rows = __builtin_amdgcn_readlane(mine.rows, r);
    x.item0 = __builtin_amdgcn_readlane(mine.item0, r);
    x.kb0 = __builtin_amdgcn_readlane(mine.kb0, r);
    return cut(x, b);
  }
  __device__ __forceinline__ WeightItem cut(const WeightGroup& x, int b) const {
    const int ns = (x.rows + a.split_rows - 1) / a.split_rows, kb = (b - x.item0) / ns, s = b - x.item0 - kb * ns;
    WeightItem it;
    it.seq = x.seq;
    it.k0 = x.lo + kb * a.block;
    it.k1 = min(x.hi, it.k0 + a.block);
    it.row0 = x.row0 + s * a.split_rows;
    it.n_row = min(a.split_rows, x.rows - s * a.split_rows);
    it.kb = x.kb0 + kb;
    it.split = s;
    it.n_split = ns;
    return it;
  }
  __device__ __forceinline__ WeightRank rank(int r) const { return a.rank[r]; }
};

}  // namespace

template <typename T, int D, bool PAGED, int KN, bool VALUE>
__global__ void __launch_bounds__(256, 2) attend_weights_kernel(WeightCall wc, Plan<VALUE> plan, CacheView cv) {
  constexpr int NC = D * (int)sizeof(T) / 16;  // 16-byte chunks of a row
  constexpr int KS = NC / 2;                   // a pair of lanes takes two chunks a step
  constexpr int SW = NC < 16 ? NC : 16;        // rows' chunks are XORed with the row modulo this
  constexpr int PF = NC / 4;                   // chunks of a tile that a thread brings in
  // whole tiles' products beside exponentials: fp32 products leave these room anyway, and small
  // calls gain more from a third block on a compute unit
  constexpr bool PIPE = sizeof(T) == 2 && KN == 2;
  __shared__ __align__(16) uint4 s_q[2][kTileRows * NC];
  __shared__ __align__(16) float s_l[2][kTileRows];
  __shared__ __align__(16) int s_pos[2][kTileRows];

  const WeightItem it = plan.item(blockIdx.y);
  const int hk = blockIdx.x;
  const int t = threadIdx.x, lane = t & 63, lc = lane & 31, lh = lane >> 5;
  const int w = __builtin_amdgcn_readfirstlane(t >> 6);
  const int g = 1 << wc.g_shift;

  // this wave's keys, 32 for each of KN: lane lc (and lc + 32) the key key0 + 32 i + lc
  uint4 kf[KN][KS];
  const int key0 = it.k0 + 32 * KN * w;
#pragma unroll
  for (int i = 0; i < KN; ++i) {
    const int key = min(key0 + 32 * i + lc, it.k1 - 1);
    const T* row = reinterpret_cast<const T*>(cv.k) + kv_offset<PAGED>(cv, wc.layer, it.seq, hk, key);
#pragma unroll
    for (int s = 0; s < KS; ++s) kf[i][s] = ld16(reinterpret_cast<const char*>(row) + (2 * s + lh) * 16);
  }

  const int n_tile = (it.n_row + kTileRows - 1) / kTileRows;
  // Four threads bring in a row, each every fourth chunk.  Two tiles ahead the rows' tokens,
  // one tile ahead the rows: neither load waits for the other inside a tile.  Rows past the
  // item's repeat its last one and see no key.
  const int tr = t >> 2, tc = t & 3;
  uint4 pf[PF];
  WeightRank rank, at;
  float pl = 0.f;
  auto find = [&](int ti) __attribute__((always_inline)) {
    rank = plan.rank((it.row0 + min(ti * kTileRows + tr, it.n_row - 1)) >> wc.g_shift);
  };
  auto fetch = [&](int ti) __attribute__((always_inline)) {
    const int r = ti * kTileRows + tr, row = it.row0 + min(r, it.n_row - 1);
    const int head = (hk << wc.g_shift) + (row & (g - 1));
    at = WeightRank{rank.tok, r < it.n_row ? rank.pos : -1};
    const char* src = reinterpret_cast<const char*>(reinterpret_cast<const T*>(wc.q.p) + (int64_t)at.tok * wc.q.token +
                                                    (int64_t)head * wc.q.head) + tc * 16;
#pragma unroll
    for (int j = 0; j < PF; ++j) pf[j] = ld16_any(src + j * 64);
    if (tc == 0) pl = wc.lse[(int64_t)at.tok * wc.n_q_heads + head];
  };
  const int qoff = tr * NC + (tc ^ (tr % SW));  // chunk 4 j + tc of the row lies at qoff ^ 4 j
  auto put = [&](int b) __attribute__((always_inline)) {
#pragma unroll
    for (int j = 0; j < PF; ++j) s_q[b][qoff ^ (4 * j)] = pf[j];
    if (tc == 0) {
      s_l[b][tr] = pl * 1.4426950408889634f;
      s_pos[b][tr] = at.pos;
    }
  };
  find(0);
  fetch(0);
  find(1);
  put(0);
  __syncthreads();

  const float scale = 1.4426950408889634f / sqrtf((float)D);
  float sum[KN][4];
#pragma unroll
  for (int i = 0; i < KN; ++i) sum[i][0] = sum[i][1] = sum[i][2] = sum[i][3] = 0.f;
  // A tile of which some row is missing or does not see some key of this wave.
  auto parts = [&](int b, int left) __attribute__((always_inline)) {
#pragma unroll
    for (int sub = 0; sub < kTileRows / 32; ++sub) {
      if (sub * 32 >= left || key0 >= it.k1) break;  // (wave-uniform) no rows, or no keys of this wave
      const int r0 = sub * 32;
      wt_f32x16 st[KN];
#pragma unroll
      for (int s = 0; s < KS; ++s) {
        const uint4 qf = s_q[b][(r0 + lc) * NC + ((2 * s + lh) ^ (lc % SW))];
#pragma unroll
        for (int i = 0; i < KN; ++i) st[i] = mma<T>(qf, kf[i][s], s ? st[i] : wt_f32x16{});
      }
      // element 4 q + e of st is row r0 + 8 q + 4 lh + e; a row sees keys up to its position,
      // and rows of a tile are sorted by it (rows past the item's, with -1, come last)
      float l[16];
#pragma unroll
      for (int q = 0; q < 4; ++q) {
        const float4 x = *reinterpret_cast<const float4*>(&s_l[b][r0 + 8 * q + 4 * lh]);
        l[4 * q] = x.x;
        l[4 * q + 1] = x.y;
        l[4 * q + 2] = x.z;
        l[4 * q + 3] = x.w;
      }
      const bool edge = min(s_pos[b][r0], s_pos[b][r0 + 31]) < key0 + 32 * KN - 1;
#pragma unroll
      for (int i = 0; i < KN; ++i) {
        float p[16];
#pragma unroll
        for (int e = 0; e < 16; ++e) p[e] = __builtin_amdgcn_exp2f(fmaf(st[i][e], scale, -l[e]));
        if (__builtin_amdgcn_readfirstlane(edge)) {
          const int key = key0 + 32 * i + lc;
#pragma unroll
          for (int q = 0; q < 4; ++q) {
            const int4 x = *reinterpret_cast<const int4*>(&s_pos[b][r0 + 8 * q + 4 * lh]);
            p[4 * q] = key <= x.x ? p[4 * q] : 0.f;
            p[4 * q + 1] = key <= x.y ? p[4 * q + 1] : 0.f;
            p[4 * q + 2] = key <= x.z ? p[4 * q + 2] : 0.f;
            p[4 * q + 3] = key <= x.w ? p[4 * q + 3] : 0.f;
          }
        }
#pragma unroll
        for (int n = 8; n >= 1; n /= 2)
#pragma unroll
          for (int e = 0; e < n; ++e) p[e] += p[e + n];
        sum[i][0] += p[0];
      }
    }
  };
  // A whole tile that sees all of this wave's keys: a product's steps beside the
  // exponentials of the one before (the matrix unit works while the others are issued), row
  // operands and log-sum-exps of the next 32 rows read in the place of those just used.
  constexpr int UN = kTileRows / 32 * KN;  // products
  auto whole = [&](int b) __attribute__((always_inline)) {
    if constexpr (PIPE) {
    uint4 qf[KS];
    float l[16];
    wt_f32x16 st[2];
    auto row_frag = [&](int sub, int s) __attribute__((always_inline)) {
      return s_q[b][(sub * 32 + lc) * NC + ((2 * s + lh) ^ (lc % SW))];
    };
    auto row_lse = [&](int sub, int q) __attribute__((always_inline)) {
      const float4 x = *reinterpret_cast<const float4*>(&s_l[b][sub * 32 + 8 * q + 4 * lh]);
      l[4 * q] = x.x;
      l[4 * q + 1] = x.y;
      l[4 * q + 2] = x.z;
      l[4 * q + 3] = x.w;
    };
#pragma unroll
    for (int s = 0; s < KS; ++s) qf[s] = row_frag(0, s);
#pragma unroll
    for (int q = 0; q < 4; ++q) row_lse(0, q);
#pragma unroll
    for (int u = 0; u <= UN; ++u) {  // product u (32 rows u / KN, keys u % KN) and the exponentials of u - 1
      const int sub = u / KN, i = u % KN, before = (u + KN - 1) % KN;
      float p[16];
#pragma unroll
      for (int s = 0; s < KS; ++s) {
        if (u < UN) {
          st[u & 1] = mma<T>(qf[s], kf[i][s], s ? st[u & 1] : wt_f32x16{});
          if (i == KN - 1 && sub + 1 < kTileRows / 32) qf[s] = row_frag(sub + 1, s);
        }
        if (u) {
#pragma unroll
          for (int e = s * 16 / KS; e < (s + 1) * 16 / KS; ++e) {
            p[e] = __builtin_amdgcn_exp2f(fmaf(st[(u & 1) ^ 1][e], scale, -l[e]));
            if (e % 4 == 3) {
              sum[before][e / 4] += (p[e - 3] + p[e - 2]) + (p[e - 1] + p[e]);
              if (before == KN - 1 && u < UN) row_lse(sub, e / 4);
            }
          }
        }
        __builtin_amdgcn_sched_barrier(0);
      }
    }
    }
  };
  for (int ti = 0; ti < n_tile; ++ti) {
    const int b = ti & 1;
    if (ti + 1 < n_tile) {
      fetch(ti + 1);
      find(ti + 2);
    }
    const int left = it.n_row - ti * kTileRows;
    const bool full = PIPE && left >= kTileRows && key0 < it.k1 && s_pos[b][0] >= key0 + 32 * KN - 1;
    if (__builtin_amdgcn_readfirstlane(full)) whole(b);
    else parts(b, left);
    if (ti + 1 < n_tile) put(b ^ 1);
    __syncthreads();
  }
#pragma unroll
  for (int i = 0; i < KN; ++i) {
    const uint32_t mine = __float_as_uint((sum[i][0] + sum[i][1]) + (sum[i][2] + sum[i][3]));
    const auto x = __builtin_amdgcn_permlane32_swap(mine, mine, false, false);
    const float total = __uint_as_float(x[0]) + __uint_as_float(x[1]);
    const int key = key0 + 32 * i + lc;
    if (lh || key >= it.k1) continue;
    if (it.n_split > 1) {
      wc.part[(((int64_t)it.split * wc.n_kb + it.kb) * cv.n_kv_heads + hk) * (128 * KN) + key - it.k0] = total;
    } else {
      float* dst = wc.weights + ((int64_t)it.seq * cv.n_kv_heads + hk) * cv.max_tokens + key;
      *dst = wc.add ? *dst + total : total;
    }
  }
}

// The splits of each block of keys added up: one block of threads a block of keys (its
// first item, b, tells which) and kv head.
template <bool VALUE>
__global__ void __launch_bounds__(256) weights_merge_kernel(WeightCall wc, Plan<VALUE> plan, CacheView cv, int block) {
  const WeightItem it = plan.item(blockIdx.y);
  const int key = it.k0 + threadIdx.x;
  if (it.split || it.n_split == 1 || key >= it.k1) return;
  const float* p = wc.part + ((int64_t)it.kb * cv.n_kv_heads + blockIdx.x) * block + threadIdx.x;
  float total = 0.f;
#pragma unroll 8
  for (int s = 0; s < it.n_split; ++s) total += p[(int64_t)s * wc.n_kb * cv.n_kv_heads * block];
  float* dst = wc.weights + ((int64_t)it.seq * cv.n_kv_heads + blockIdx.x) * cv.max_tokens + key;
  *dst = wc.add ? *dst + total : total;
}

namespace {

int check(hipError_t e) { return e == hipSuccess ? 0 : (int)e; }

template <bool VALUE>
int launch(int dtype, const WeightCall& wc, const Plan<VALUE>& plan, int n_items, int block, const CacheView& cv,
           hipStream_t s) {
  const dim3 grid(cv.n_kv_heads, n_items);
#define WK(T, DD, PG, KN) hipLaunchKernelGGL((attend_weights_kernel<T, DD, PG, KN, VALUE>), grid, dim3(256), 0, s, wc, plan, cv)
#define WKN(T, DD, PG) { if (block == 256) WK(T, DD, PG, (weights_most_keys(sizeof(T), DD) / 128)); else WK(T, DD, PG, 1); }
#define WKP(T, DD) { if (cv.page_size) WKN(T, DD, true) else WKN(T, DD, false) }
  if (dtype == 0) { if (cv.head_dim == 64) WKP(float, 64) else WKP(float, 128) }
  else { if (cv.head_dim == 64) WKP(bf16_t, 64) else WKP(bf16_t, 128) }
#undef WKP
#undef WKN
#undef WK
  if (int rc = check(hipGetLastError())) return rc;
  if (wc.part) {
    hipLaunchKernelGGL((weights_merge_kernel<VALUE>), grid, dim3(block), 0, s, wc, plan, cv, block);
    return check(hipGetLastError());
  }
  return 0;
}

}  // namespace

int launch_attend_weights(int dtype, const WeightCall& call, const WeightArgs* args, const WeightItem* items,
                          const WeightRank* ranks, int n_items, int block, const CacheView& cv, hipStream_t s) {
  if (args) return launch<true>(dtype, call, Plan<true>{*args}, n_items, block, cv, s);
  return launch<false>(dtype, call, Plan<false>{items, ranks}, n_items, block, cv, s);
}

}  // namespace fcg

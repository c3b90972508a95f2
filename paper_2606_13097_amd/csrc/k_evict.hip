// Eviction by weight for gfx950: of each sequence, layer and kv head the positions that
// stay are selected, and their rows moved to positions 0, 1, 2, .. of a sequence, keys
// turned by the distance they move.
//
// Selection (evict_select_kernel, one block for each item, kv head and layer): the
// weights as ordered 32-bit keys (the ends that always stay above all others), the
// threshold found 8 to 11 bits at a time by histograms in LDS, then the positions
// above it, and as many equal to it as are left, lowest first, written in order by counts
// over waves.  A row of up to 16K positions stays in registers over all of it (block sizes:
// see the launch); a longer one is read anew in each pass (56 rows of up to 20K: 40 us; twice the
// weights a thread would still fit the registers, of which 68 are in use).  Bound by
// its chain of passes, not by the weights it reads (256 rows of 4321: 12 us, 0.4 TB/s; eight
// copies of each bin, so that adds meet less often: no difference).  More blocks of the launch
// fill the table of turns: (cos, sin) of every distance, so that the rows that move the same
// distance, in whatever layer and head, share them (one sincos for each row and pair took as
// long as the memory).
//
// Moving: into another sequence, 64 rows of a layer and head a block, keys and values
// together, every load before the first store.  Bound by the memory: 1111 of 4321 bf16 rows
// of 32 layers and 8 heads 60 us, 5 TB/s; 16 sequences of 4 layers, half of their rows or so,
// 142 us.  The rows go past the caches: the calls took 81 us and 187 us through them, 78 and
// 180 with the stores past them, 76.5 and 173.5 with the loads too.  (Data asked for before the
// turns, and five blocks a compute unit by register count: no difference.  Turns computed by
// the copy for calls of few rows: 5.5 us against 3.9, for one launch's table less.)
//
// In place a row only moves down, so a later row never reads what an earlier one wrote; a
// block takes a layer's and head's keys or values in order, 128 rows a step, and stores a
// step's rows once all its waves have read theirs: 1111 of 4321 bf16 rows of 32 layers and 8
// heads 66 us, 4.6 TB/s, bound by that chain of steps, with accesses through the caches.
#include "fcg_device.hpp"
#include "kernels.hpp"

namespace fcg {

namespace {

constexpr int kSelKeys = 16;  // keys of a thread in registers

// order of a weight: larger ones above, -0 as 0, NaN below everything
__device__ __forceinline__ uint32_t order_of(float x) {
  const uint32_t u = __float_as_uint(x + 0.f);
  const uint32_t k = u >> 31 ? ~u : u | 0x80000000u;
  return x != x ? 0u : k;
}
constexpr uint32_t kAlways = 0xFFFFFFFFu;

// inclusive sum over the lanes of a wave up to this one: within rows of 16 lanes by DPP
// shifts, then the sums of the rows before by its broadcasts of lanes 15, 47 and 31
template <int CTRL, int ROWS>
__device__ __forceinline__ int dpp_add(int v) {
  return v + __builtin_amdgcn_update_dpp(0, v, CTRL, ROWS, 0xF, false);
}
__device__ __forceinline__ int scan_wave(int v) {
  v = dpp_add<0x111, 0xF>(v);  // row_shr:1
  v = dpp_add<0x112, 0xF>(v);
  v = dpp_add<0x114, 0xF>(v);
  v = dpp_add<0x118, 0xF>(v);
  v = dpp_add<0x142, 0xA>(v);     // row_bcast:15 to rows 1 and 3
  return dpp_add<0x143, 0xC>(v);  // row_bcast:31 to rows 2 and 3
}

// The item of chunk (or block) b: the last one whose first chunk is at most b.
__device__ __forceinline__ int find_item(const EvictArgs& a, int b) {
  static_assert(kEvictItems == 64, "one item per lane");
  const int lane = threadIdx.x & 63;
  const int first = a.item[min(lane, a.n - 1)].chunk0;
  const uint64_t below = __builtin_amdgcn_ballot_w64(lane < a.n && first <= b);
  return 63 - __builtin_clzll(below);
}
__device__ __forceinline__ int32_t* kept_row(const EvictCall& ec, int item, int Hkv, int hk, int layer) {
  return ec.kept + (((int64_t)layer * ec.n_items + ec.item0 + item) * Hkv + hk) * ec.kept_stride;
}

}  // namespace

// BITS of the keys a pass
template <int kSelThreads, int BITS>
__global__ void __launch_bounds__(kSelThreads) evict_select_kernel(EvictCall ec, EvictArgs a, RopeArgs ra, int n_rows,
                                                                   int n_seqs, int Hkv, int max_tokens, int n_turn) {
  constexpr int kSelSeg = kSelThreads * kSelKeys, kSelWaves = kSelThreads / 64, kBins = 1 << BITS;
  constexpr int PASSES = (32 + BITS - 1) / BITS, PER = kBins / kSelThreads;  // bins of a thread
  static_assert(PER >= 1 && PER <= 2, "one or two bins a thread");
  __shared__ int s_hist[kBins];
  __shared__ __align__(16) int s_wave[kSelWaves];
  __shared__ int s_gt[kSelKeys * kSelWaves], s_eq[kSelKeys * kSelWaves];
  __shared__ int s_bin, s_above;
  const int t = threadIdx.x, lane = t & 63, w = t >> 6;

  if ((int)blockIdx.x >= n_rows) {  // the table of turns
    const int half = ra.rot / 2;
    const int64_t end = (int64_t)n_turn * half, step = (int64_t)(gridDim.x - n_rows) * kSelThreads;
    for (int64_t i = (int64_t)(blockIdx.x - n_rows) * kSelThreads + t; i < end; i += step) {
      float cs, sn;
      const int d = (int)(i / half);
      rope_cs_turns((double)d, ra.turns[i - (int64_t)d * half], &cs, &sn);
      ec.turns[i] = make_float2(cs, sn);
    }
    return;
  }
  const int hk = blockIdx.x % Hkv, x = blockIdx.x / Hkv, item = x % a.n, layer = x / a.n;
  const EvictItem it = a.item[item];
  const float* src = ec.weights + (((int64_t)layer * n_seqs + it.src) * Hkv + hk) * max_tokens;
  float* dst = ec.weights + (((int64_t)layer * n_seqs + it.dst) * Hkv + hk) * max_tokens;
  int32_t* kept = kept_row(ec, item, Hkv, hk, layer);
  const int n = it.len, keep = it.keep;
  const int first = min(keep, ec.first), recent = min(keep - first, ec.recent);

  float v[kSelKeys];
  uint32_t key[kSelKeys];
  // (uniform) some thread's element e of the segment is in the row
  auto used = [&](int seg, int e) __attribute__((always_inline)) { return seg * kSelSeg + e * kSelThreads < n; };
  auto load = [&](int seg) __attribute__((always_inline)) {
#pragma unroll
    for (int e = 0; e < kSelKeys; ++e) {
      const int i = seg * kSelSeg + e * kSelThreads + t;
      if (used(seg, e)) v[e] = i < n ? src[i] : 0.f;
    }
#pragma unroll
    for (int e = 0; e < kSelKeys; ++e) {
      const int i = seg * kSelSeg + e * kSelThreads + t;
      if (used(seg, e)) key[e] = i < first || i >= n - recent ? kAlways : order_of(v[e]);
    }
  };
  const int n_seg = keep ? (n + kSelSeg - 1) / kSelSeg : 0;
  // threshold: the keep-th largest key; `equal` of those equal to it stay
  uint32_t top = 0, mask = 0;
  int equal = keep;
  if (n_seg) load(0);
  if (n_seg && keep < n) {
    for (int pass = 0; pass < PASSES; ++pass) {
      const int hi = 32 - pass * BITS, shift = max(hi - BITS, 0), bits = hi - shift;
      for (int j = t; j < kBins; j += kSelThreads) s_hist[j] = 0;
      __syncthreads();
      for (int seg = 0; seg < n_seg; ++seg) {
        if (n_seg > 1) load(seg);
#pragma unroll
        for (int e = 0; e < kSelKeys; ++e) {
          if (!used(seg, e)) break;
          const int i = seg * kSelSeg + e * kSelThreads + t;
          const uint32_t k = key[e];
          if (i < n && (k & mask) == top) atomicAdd(&s_hist[k >> shift & ((1u << bits) - 1)], 1);
        }
      }
      __syncthreads();
      // bins from the highest down, one or two a thread: the one in which the count passes `equal`
      const int b1 = kBins - 1 - PER * t, h1 = s_hist[b1], h0 = PER == 2 ? s_hist[b1 - 1] : 0;
      const int up = scan_wave(h1 + h0);
      if (lane == 63) s_wave[w] = up;
      __syncthreads();
      int above = up - h1 - h0;
#pragma unroll
      for (int j = 0; j < kSelWaves; ++j) above += j < w ? s_wave[j] : 0;
      if (above < equal && above + h1 >= equal) {
        s_bin = b1;
        s_above = above;
      } else if (above + h1 < equal && above + h1 + h0 >= equal) {
        s_bin = b1 - 1;
        s_above = above + h1;
      }
      __syncthreads();
      equal -= s_above;
      top |= (uint32_t)s_bin << shift;
      mask |= ((1u << bits) - 1) << shift;
      __syncthreads();
    }
  }
  // what stays, in order of position
  int gt0 = 0, eq0 = 0;
  for (int seg = 0; seg < n_seg; ++seg) {
    if (n_seg > 1) load(seg);
    uint32_t is_gt = 0, is_eq = 0;
#pragma unroll
    for (int e = 0; e < kSelKeys; ++e) {
      if (!used(seg, e)) {  // (counts of the places past the row)
        if (t < kSelWaves) s_gt[e * kSelWaves + t] = s_eq[e * kSelWaves + t] = 0;
        continue;
      }
      const int i = seg * kSelSeg + e * kSelThreads + t;
      const uint32_t k = key[e];
      const bool all = keep >= n;
      const bool gt = i < n && (all || k > top), eq = i < n && !all && k == top;
      is_gt |= (uint32_t)gt << e;
      is_eq |= (uint32_t)eq << e;
      const uint64_t bg = __builtin_amdgcn_ballot_w64(gt), be = __builtin_amdgcn_ballot_w64(eq);
      if (lane == 0) {
        s_gt[e * kSelWaves + w] = __builtin_popcountll(bg);
        s_eq[e * kSelWaves + w] = __builtin_popcountll(be);
      }
    }
    __syncthreads();  // (and every weight of the segment has been read)
    if (w < 2) {      // running counts: of those above by wave 0, of the equal ones by wave 1
      int* s = w ? s_eq : s_gt;
      int base = w ? eq0 : gt0;
#pragma unroll
      for (int j = 0; j < kSelKeys * kSelWaves; j += 64) {
        const int c = s[j + lane], up = scan_wave(c);
        s[j + lane] = base + up - c;
        base += __builtin_amdgcn_readlane(up, 63);
      }
      if (lane == 0) s_wave[w] = base;
    }
    __syncthreads();
#pragma unroll
    for (int e = 0; e < kSelKeys; ++e) {
      if (!used(seg, e)) break;
      const bool gt = is_gt >> e & 1, eq = is_eq >> e & 1;
      const uint64_t bg = __builtin_amdgcn_ballot_w64(gt), be = __builtin_amdgcn_ballot_w64(eq);
      const int g = s_gt[e * kSelWaves + w] + __builtin_amdgcn_mbcnt_hi(bg >> 32, __builtin_amdgcn_mbcnt_lo((uint32_t)bg, 0));
      const int q = s_eq[e * kSelWaves + w] + __builtin_amdgcn_mbcnt_hi(be >> 32, __builtin_amdgcn_mbcnt_lo((uint32_t)be, 0));
      if (gt || (eq && q < equal)) {
        const int to = g + min(q, equal);
        kept[to] = seg * kSelSeg + e * kSelThreads + t;
        dst[to] = v[e];
      }
    }
    gt0 = s_wave[0];
    eq0 = s_wave[1];
    __syncthreads();
  }
  for (int i = min(keep, n) + t; i < max_tokens; i += kSelThreads) dst[i] = 0.f;
}

namespace {

// The lanes of a row: which two vectors this lane moves, and their turn.
template <typename T, int D, bool PAIRS>
struct Lane {
  static constexpr int VEC = Store<T>::VEC;
  static constexpr int NCH = D / (2 * VEC);  // lanes of a row
  int c, lo, hi;
  bool turn_a, turn_b;
  __device__ __forceinline__ Lane(int t, int half) {
    const int rchunks = half / VEC;
    c = t % NCH;
    turn_a = c < (PAIRS ? 2 * rchunks : rchunks);
    turn_b = PAIRS ? NCH + c < 2 * rchunks : turn_a;
    lo = (!PAIRS && c >= rchunks ? rchunks + c : c) * VEC;
    hi = (!PAIRS && c < rchunks ? rchunks + c : NCH + c) * VEC;
  }
  // (cos, sin) of the pairs of this lane: NT vectors of two
  static constexpr int NT = VEC / 2;
  __device__ __forceinline__ void load(const float2* row, float4* cs) const {
    constexpr int P = PAIRS ? VEC / 2 : VEC;
    if (turn_a) {
#pragma unroll
      for (int j = 0; j < P / 2; ++j) cs[j] = *reinterpret_cast<const float4*>(row + c * P + 2 * j);
    }
    if (PAIRS && turn_b) {
#pragma unroll
      for (int j = 0; j < P / 2; ++j) cs[P / 2 + j] = *reinterpret_cast<const float4*>(row + (NCH + c) * P + 2 * j);
    }
  }
  // turned back by the distance
  __device__ __forceinline__ void turn(uint4* a, uint4* b, const float4* cs) const {
    float xa[VEC], xb[VEC], ya[VEC], yb[VEC];
    if (!turn_a) return;
    Store<T>::unpack(*a, xa);
    Store<T>::unpack(*b, xb);
    auto cos_of = [&](int i) __attribute__((always_inline)) { return i & 1 ? cs[i / 2].z : cs[i / 2].x; };
    auto sin_of = [&](int i) __attribute__((always_inline)) { return i & 1 ? cs[i / 2].w : cs[i / 2].y; };
    if constexpr (PAIRS) {
      constexpr int P = VEC / 2;
#pragma unroll
      for (int e = 0; e < P; ++e) {
        ya[2 * e] = fmaf(xa[2 * e], cos_of(e), xa[2 * e + 1] * sin_of(e));
        ya[2 * e + 1] = fmaf(xa[2 * e + 1], cos_of(e), -xa[2 * e] * sin_of(e));
      }
      *a = Store<T>::pack(ya);
      if (!turn_b) return;
#pragma unroll
      for (int e = 0; e < P; ++e) {
        yb[2 * e] = fmaf(xb[2 * e], cos_of(P + e), xb[2 * e + 1] * sin_of(P + e));
        yb[2 * e + 1] = fmaf(xb[2 * e + 1], cos_of(P + e), -xb[2 * e] * sin_of(P + e));
      }
      *b = Store<T>::pack(yb);
    } else {
#pragma unroll
      for (int e = 0; e < VEC; ++e) {
        ya[e] = fmaf(xa[e], cos_of(e), xb[e] * sin_of(e));
        yb[e] = fmaf(xb[e], cos_of(e), -xa[e] * sin_of(e));
      }
      *a = Store<T>::pack(ya);
      *b = Store<T>::pack(yb);
    }
  }
};

}  // namespace

// into another sequence
template <typename T, int D, bool PAIRS, bool PAGED>
__global__ void __launch_bounds__(256) evict_copy_kernel(EvictCall ec, EvictArgs a, CacheView cv, int half) {
  typedef Lane<T, D, PAIRS> L;
  constexpr int RP = 256 / L::NCH, PASSES = kEvictRows / RP;
  const int item = find_item(a, blockIdx.x), hk = blockIdx.y, layer = blockIdx.z;
  const EvictItem it = a.item[item];
  const int j0 = (blockIdx.x - it.chunk0) * kEvictRows;
  const int32_t* kept = kept_row(ec, item, cv.n_kv_heads, hk, layer);
  const L ln(threadIdx.x, half);
  const int row = threadIdx.x / L::NCH;
  uint4 ka[PASSES], kb[PASSES], va[PASSES], vb[PASSES];
  float4 cs[PASSES][L::NT];
  int from[PASSES];
#pragma unroll
  for (int p = 0; p < PASSES; ++p) from[p] = kept[min(j0 + p * RP + row, it.keep - 1)];
#pragma unroll
  for (int p = 0; p < PASSES; ++p) {
    const int j = min(j0 + p * RP + row, it.keep - 1);
    const T* k = reinterpret_cast<const T*>(cv.k) + kv_offset<PAGED>(cv, layer, it.src, hk, from[p]);
    const T* v = v_row<PAGED, T>(cv, layer, it.src, hk, from[p]);
    ka[p] = ld16_nt(k + ln.lo);
    kb[p] = ld16_nt(k + ln.hi);
    va[p] = ld16_nt(v + ln.lo);
    vb[p] = ld16_nt(v + ln.hi);
    ln.load(ec.turns + (int64_t)(from[p] - j) * half, cs[p]);
  }
#pragma unroll
  for (int p = 0; p < PASSES; ++p) {
    const int j = j0 + p * RP + row;
    if (j >= it.keep) continue;
    const int64_t at = kv_offset<PAGED>(cv, layer, it.dst, hk, j);
    T* k = reinterpret_cast<T*>(cv.k) + at;
    T* v = reinterpret_cast<T*>(cv.v) + at;
    if (from[p] != j) ln.turn(&ka[p], &kb[p], cs[p]);
    st16_nt(k + ln.lo, ka[p]);
    st16_nt(k + ln.hi, kb[p]);
    st16_nt(v + ln.lo, va[p]);
    st16_nt(v + ln.hi, vb[p]);
  }
}

// in place: blockIdx.y even the keys, odd the values of a head
template <typename T, int D, bool PAIRS, bool PAGED>
__global__ void __launch_bounds__(256) evict_inplace_kernel(EvictCall ec, EvictArgs a, CacheView cv, int half) {
  typedef Lane<T, D, PAIRS> L;
  constexpr int RP = 256 / L::NCH, PASSES = 128 / RP > 1 ? 128 / RP : 1, STEP = RP * PASSES;
  const int hk = blockIdx.y >> 1, layer = blockIdx.z;
  const bool keys = !(blockIdx.y & 1);
  const EvictItem it = a.item[blockIdx.x];
  const int32_t* kept = kept_row(ec, blockIdx.x, cv.n_kv_heads, hk, layer);
  T* base = reinterpret_cast<T*>(keys ? cv.k : cv.v);
  const L ln(threadIdx.x, half);
  const int row = threadIdx.x / L::NCH;
  uint4 x[PASSES], y[PASSES];
  float4 cs[PASSES][L::NT];
  int from[PASSES];
  auto load = [&](int j0) __attribute__((always_inline)) {
#pragma unroll
    for (int p = 0; p < PASSES; ++p) from[p] = kept[min(j0 + p * RP + row, it.keep - 1)];
#pragma unroll
    for (int p = 0; p < PASSES; ++p) {
      const T* r = base + kv_offset<PAGED>(cv, layer, it.src, hk, from[p]);
      x[p] = ld16(r + ln.lo);
      y[p] = ld16(r + ln.hi);
      if (keys) ln.load(ec.turns + (int64_t)(from[p] - min(j0 + p * RP + row, it.keep - 1)) * half, cs[p]);
    }
  };
  int j0 = 0;
  while (j0 + STEP <= it.keep && kept[j0 + STEP - 1] == j0 + STEP - 1) j0 += STEP;  // these stay where they are
  if (j0 < it.keep) load(j0);
  for (; j0 < it.keep; j0 += STEP) {
    wait_vm0();       // this step's rows are read,
    __syncthreads();  // by every wave; rows of later steps lie past all that is written now
    uint4 sx[PASSES], sy[PASSES];
    int was[PASSES];
#pragma unroll
    for (int p = 0; p < PASSES; ++p) {
      if (keys) ln.turn(&x[p], &y[p], cs[p]);
      sx[p] = x[p];
      sy[p] = y[p];
      was[p] = from[p];
    }
    if (j0 + STEP < it.keep) load(j0 + STEP);
#pragma unroll
    for (int p = 0; p < PASSES; ++p) {
      const int j = j0 + p * RP + row;
      if (j >= it.keep || was[p] == j) continue;
      T* r = base + kv_offset<PAGED>(cv, layer, it.dst, hk, j);
      st16(r + ln.lo, sx[p]);
      st16(r + ln.hi, sy[p]);
    }
  }
}

namespace {

int check(hipError_t e) { return e == hipSuccess ? 0 : (int)e; }

}  // namespace

int launch_evict_select(const EvictCall& ec, const EvictArgs& args, const RopeArgs& ra, int n_layers, int n_seqs, int Hkv,
                        int max_tokens, int n_turn, hipStream_t s) {
  const int n_rows = args.n * Hkv * n_layers;
  int longest = 0;
  for (int i = 0; i < args.n; ++i) longest = args.item[i].len > longest ? args.item[i].len : longest;
  // The smallest block that holds the longest row in its registers, of 256 threads for short
  // rows only (us a call with blocks of 256, 512 and 1024 threads: 14 sequences of up to 317
  // positions, 28 layers of 4 kv heads, 25, 32, 62; 4 of 1000, 16 layers of 8, 35, 35, 44; 1
  // of 2000, 32 layers, 25.3, 24.5, 26.3; 8 of 4000, 16 layers, 73, 74, 92; 1 of 8000, 32 layers,
  // 65, 33.0, 33.4; 1 of 15000, 104, 67, 41).
  const int threads = longest <= 1024 ? 256 : longest <= 512 * kSelKeys ? 512 : 1024;
  const int64_t entries = (int64_t)n_turn * (ra.rot / 2);
  const int64_t want = (entries + threads - 1) / threads;
  const int n_tab = (int)(want < 4096 ? want : 4096);
#define SEL(TH, BITS)                                                                                              \
  hipLaunchKernelGGL((evict_select_kernel<TH, BITS>), dim3(n_rows + n_tab), dim3(TH), 0, s, ec, args, ra, n_rows, n_seqs, \
                     Hkv, max_tokens, n_turn)
  if (threads == 256) SEL(256, 8);
  else if (threads == 512) SEL(512, 9);
  else SEL(1024, 11);
#undef SEL
  return check(hipGetLastError());
}

int launch_evict_move(int dtype, bool pairs, bool in_place, const EvictCall& ec, const EvictArgs& args, int n_chunks,
                      const CacheView& cv, int half, int n_layers, hipStream_t s) {
  const dim3 grid = in_place ? dim3(args.n, 2 * cv.n_kv_heads, n_layers) : dim3(n_chunks, cv.n_kv_heads, n_layers);
#define EV(T, DD, PR, PG)                                                                                              \
  {                                                                                                                    \
    if (in_place) hipLaunchKernelGGL((evict_inplace_kernel<T, DD, PR, PG>), grid, dim3(256), 0, s, ec, args, cv, half); \
    else hipLaunchKernelGGL((evict_copy_kernel<T, DD, PR, PG>), grid, dim3(256), 0, s, ec, args, cv, half);            \
  }
#define EVG(T, DD, PR) { if (cv.page_size) EV(T, DD, PR, true) else EV(T, DD, PR, false) }
#define EVP(T, DD) { if (pairs) EVG(T, DD, true) else EVG(T, DD, false) }
  if (dtype == 0) { if (cv.head_dim == 64) EVP(float, 64) else EVP(float, 128) }
  else { if (cv.head_dim == 64) EVP(bf16_t, 64) else EVP(bf16_t, 128) }
#undef EVP
#undef EVG
#undef EV
  return check(hipGetLastError());
}

}  // namespace fcg

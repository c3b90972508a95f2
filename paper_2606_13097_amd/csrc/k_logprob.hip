// Log probabilities of given tokens, entropy and the most likely tokens from rows of
// logits, and the gradient of the logits, for gfx950.
//
//   lse = ln sum e^x,  logprob_t = x_t - lse,  H = -sum p ln p,  p = e^(x - lse).
//
// One pass over a row: with a reference r near the row's maximum,
//   S = sum e^(x - r),  U = sum e^(x - r) (x - r),  lse = r + ln S,  H = ln S - U / S.
// x - r is formed first, so large logits cost no digits.  A thread keeps its reference until
// an element's e^(x - r) passes 8, so few steps rescale, and yet a token that has nearly all of
// the probability is the reference itself: its term is 1, S is at least 1 and U at most 0, so
// that no log probability is above 0 and no entropy below.  (A reference that trails by d costs
// ln S and U / S d units of 2^-24: a reference moved at 2^40 had entropies of such rows off
// by 2e-6, of any sign.)  A vector's terms are added to each other before they meet the sum,
// so that fewer and larger addends are rounded against a peak.
//
// The most likely tokens: order is (value, then lower index), as one 64-bit key.  A block
// holds a chunk of its row in registers (4 vectors a thread); a lower bound on the k-th
// largest key is the k-th largest of the maxima of 64 or 128 groups of threads (later chunks:
// the k-th found so far), and the few elements at or above it go to a list in LDS, of which
// k are kept by counting.  If too many pass (a row of equal logits), the bound is taken
// anew from the threads' own largest keys: at most (k - 1) 32 + 1 elements reach that.
//
// Few rows are cut into splits, whose partials a second launch joins.
//
// What bounds it: many rows the memory (3001 fp32 rows of 50021: 95 us, 6.3 TB/s; each logit is
// read once, with 8 vectors a thread in flight where no alternatives are kept); blocks of 256
// threads, several to a compute unit, so that one's exponentials (8 cycles each) run beside
// another's loads (141 us with blocks of 1024).  Few rows the chain of a row: load,
// reduce, bound, list, partial, second launch (1 row of 128K bf16 with 20 alternatives 7.3 + 4.7
// us; 64 rows, one chunk a block, 11.9 + 4.8).  Many bf16 rows lie between: as many
// exponentials in half the bytes (3001 rows of 50021 70 us, 4.3 TB/s; 1501 of 100003 with 20
// alternatives 95 us, 3.1 TB/s).
//
// The gradient reads and writes each logit once and is bound by that: 1501 bf16 rows of 100003,
// 108 us, 5.5 TB/s (the fastest copies 6.2).  Times of many rows are of calls one after the other;
// a profiler's kernel times of the two are 115 and 114 us.
#include <type_traits>

#include "fcg_device.hpp"
#include "kernels.hpp"

namespace fcg {

namespace {

constexpr int kThreads = 256, kWaves = kThreads / 64;
constexpr int kListCap = kLogpTop + (kLogpTop - 1) * 32 + 1;  // keys kept, and those of one chunk
constexpr float kC = 1.4426950408889634f, kLn2 = 0.6931471805599453f;
constexpr float kMove = 3 * kLn2;  // a reference moves when an element is further above it
constexpr float kLeast = -3.4028235e38f;  // the reference of nothing
constexpr float kBound = -1e20f;  // a difference in a product: 0 times -inf is NaN

__device__ __forceinline__ uint32_t order_of(float x) {
  const uint32_t u = __float_as_uint(x + 0.f);
  const uint32_t k = u >> 31 ? ~u : u | 0x80000000u;
  return x != x ? 0u : k;
}
__device__ __forceinline__ float value_of(uint32_t k) {
  return k ? __uint_as_float(k >> 31 ? k ^ 0x80000000u : ~k) : __uint_as_float(0x7FC00000u);
}
__device__ __forceinline__ uint64_t key_of(float x, int i) { return (uint64_t)order_of(x) << 32 | (uint32_t)~i; }

constexpr uint32_t kLowest = 0x007FFFFFu;  // order_of(-inf)

// S and U about a reference
struct Stat {
  float r, s, u;
};
__device__ __forceinline__ Stat join(const Stat& a, const Stat& b) {
  const float r = fmaxf(a.r, b.r);
  const float da = fmaxf(a.r - r, kBound), db = fmaxf(b.r - r, kBound);
  const float fa = __builtin_amdgcn_exp2f(da * kC), fb = __builtin_amdgcn_exp2f(db * kC);
  return Stat{r, fmaf(a.s, fa, b.s * fb), fmaf(fmaf(a.s, da, a.u), fa, fmaf(b.s, db, b.u) * fb)};
}
__device__ __forceinline__ float max_wave(float v) {
  v = max_lanes32(v);
  const auto b = __builtin_amdgcn_permlane32_swap(__float_as_uint(v), __float_as_uint(v), false, false);
  return fmaxf(__uint_as_float(b[0]), __uint_as_float(b[1]));
}
__device__ __forceinline__ float sum_wave(float v) {
  v = sum_lanes32(v);
  const auto b = __builtin_amdgcn_permlane32_swap(__float_as_uint(v), __float_as_uint(v), false, false);
  return __uint_as_float(b[0]) + __uint_as_float(b[1]);
}
// over the lanes of a wave: every lane's brought to the largest reference, then added
__device__ __forceinline__ Stat join_wave(const Stat& a) {
  const float r = max_wave(a.r), d = fmaxf(a.r - r, kBound), f = __builtin_amdgcn_exp2f(d * kC);
  return Stat{r, sum_wave(a.s * f), sum_wave(fmaf(a.s, d, a.u) * f)};
}

// what a row's statistics give
struct Row {
  float r, ln_s, lse;
  bool empty;
  __device__ __forceinline__ explicit Row(const Stat& a) {
    empty = a.s == 0.f;
    r = a.r;
    ln_s = empty ? 0.f : log2f(a.s) * kLn2;
    lse = empty ? -INFINITY : r + ln_s;
  }
  __device__ __forceinline__ float logprob(float x) const { return empty ? -INFINITY : (x - r) - ln_s; }
  __device__ __forceinline__ float entropy(const Stat& a) const {
    return empty ? 0.f : ln_s - a.u / a.s;
  }
};

// A row's target and its logit, asked for early: two memory round trips.
template <typename T>
struct Target {
  int t;
  float x;
  __device__ __forceinline__ Target(const LogpArgs& la, int row) : t(la.logprob ? la.targets[row] : -1), x(0.f) {}
  __device__ __forceinline__ void load(const LogpArgs& la, int row) {
    if (t >= la.vocab) t = -1;
    if (t >= 0) x = Store<T>::load1(reinterpret_cast<const T*>(la.x) + (int64_t)row * la.stride + t);
  }
};
template <typename T>
__device__ __forceinline__ void finish(const LogpArgs& la, int row, const Stat& st, const Target<T>& tg) {
  const Row rw(st);
  if (la.lse) la.lse[row] = rw.lse;
  if (la.entropy) la.entropy[row] = rw.entropy(st);
  if (la.logprob) la.logprob[row] = tg.t < 0 ? 0.f : rw.logprob(tg.x);
}
__device__ __forceinline__ void put_top(const LogpArgs& la, int row, int j, uint64_t key, const Stat& st) {
  const Row rw(st);
  la.top_id[(int64_t)row * la.n_top + j] = (int)~(uint32_t)key;
  if (la.top_logprob) la.top_logprob[(int64_t)row * la.n_top + j] = rw.logprob(value_of((uint32_t)(key >> 32)));
}

// A vector without its first n elements, -inf behind the others.
template <typename T>
__device__ __forceinline__ uint4 shifted(const uint4& v, int n) {
  const uint64_t none = sizeof(T) == 2 ? 0xFF80FF80FF80FF80ull : 0xFF800000FF800000ull;
  const uint64_t lo = (uint64_t)v.y << 32 | v.x, hi = (uint64_t)v.w << 32 | v.z;
  const int bits = n * (int)sizeof(T) * 8;
  uint64_t a, b;
  if (bits >= 128) a = b = none;
  else if (bits >= 64) {
    a = bits == 64 ? hi : hi >> (bits - 64) | none << (128 - bits);
    b = none;
  } else {
    a = bits ? lo >> bits | hi << (64 - bits) : lo;
    b = bits ? hi >> bits | none << (64 - bits) : hi;
  }
  return make_uint4((uint32_t)a, (uint32_t)(a >> 32), (uint32_t)b, (uint32_t)(b >> 32));
}
// elements i .. of a row shorter than a vector
template <typename T>
__device__ __forceinline__ uint4 few(const T* x, int i, int n) {
  float f[Store<T>::VEC];
#pragma unroll
  for (int e = 0; e < Store<T>::VEC; ++e) f[e] = i + e < n ? Store<T>::load1(x + i + e) : -INFINITY;
  return Store<T>::pack(f);
}

// The n keys in s: those of rank < k to out, largest first, by counting; threads of the block.
__device__ __forceinline__ void rank_keys(const uint64_t* s, int n, uint64_t* out, int k, int threads) {
  for (int i = threadIdx.x; i < n; i += threads) {
    const uint64_t mine = s[i];
    int above = 0;
#pragma unroll 8
    for (int j = 0; j < n; ++j) above += s[j] > mine;
    if (above < k) out[above] = mine;
  }
}

}  // namespace

// STREAM: more than the last-level cache holds, read past it.
template <typename T, bool TOP, bool STREAM>
__global__ void __launch_bounds__(kThreads, 4) logprob_kernel(LogpArgs la) {
  constexpr int kVecs = TOP ? 4 : 8;  // vectors of a thread in a chunk
  constexpr int VEC = Store<T>::VEC, CHUNK = kThreads * kVecs * VEC;
  __shared__ Stat s_stat[kWaves];
  __shared__ uint64_t s_list[TOP ? kListCap : 1], s_top[TOP ? kLogpTop : 1], s_bound;
  __shared__ uint64_t s_own[TOP ? kThreads : 1];
  __shared__ int s_n;

  const int t = threadIdx.x, lane = t & 63, w = t >> 6;
  const int row = blockIdx.x / la.splits, split = blockIdx.x - row * la.splits;
  const int e0 = split * la.split_len, e1 = min(la.vocab, e0 + la.split_len);
  const T* x = reinterpret_cast<const T*>(la.x) + (int64_t)row * la.stride;
  const int k = la.n_top;

  uint4 cur[kVecs], next[kVecs];
  // (uniform) some thread's vector j of the chunk is in the part
  auto used = [&](int chunk, int j) __attribute__((always_inline)) {
    return e0 + chunk * CHUNK + j * kThreads * VEC < e1;
  };
  // (vectors that pass the part's end read its last elements: see fix; no branches, so that
  // the compiler can count which loads it waits for)
  auto load = [&](uint4* v, int chunk) __attribute__((always_inline)) {
#pragma unroll
    for (int j = 0; j < kVecs; ++j) {
      const int i = e0 + chunk * CHUNK + (j * kThreads + t) * VEC;
      v[j] = STREAM ? ld16_nt_any(x + min(i, e1 - VEC)) : ld16_any(x + min(i, e1 - VEC));
    }
  };
  // in the last chunk: the elements in their places, -inf past the end
  auto fix = [&](uint4* v, int chunk) __attribute__((always_inline)) {
    if (e1 < VEC) return;
#pragma unroll
    for (int j = 0; j < kVecs; ++j) {
      if (!used(chunk, j)) break;
      const int i = e0 + chunk * CHUNK + (j * kThreads + t) * VEC;
      if (i + VEC > e1) v[j] = shifted<T>(v[j], min(i + VEC - e1, VEC));
    }
  };
  float r = kLeast, s0 = 0.f, s1 = 0.f, u0 = 0.f, u1 = 0.f;
  if (TOP && t == 0) {
    s_n = 0;
    s_bound = 0;
  }
  int have = 0;  // keys in s_list
  const int n_chunk = (e1 - e0 + CHUNK - 1) / CHUNK;
  Target<T> target(la, row);
  if (e1 >= VEC) {
    load(cur, 0);
  } else {
#pragma unroll
    for (int j = 0; j < kVecs; ++j) cur[j] = few<T>(x, (j * kThreads + t) * VEC, e1);
  }
  if (la.splits == 1) target.load(la, row);
  auto take = [&](int ch, auto last) __attribute__((always_inline)) {
    auto in_use = [&](int j) __attribute__((always_inline)) { return !decltype(last)::value || used(ch, j); };
    float vmax[kVecs], tmax = -INFINITY;
#pragma unroll
    for (int j = 0; j < kVecs; ++j) {
      vmax[j] = -INFINITY;
      if (!in_use(j)) continue;
      float f[VEC];
      Store<T>::unpack(cur[j], f);
      float m = f[0];
#pragma unroll
      for (int e = 1; e < VEC; ++e) m = fmaxf(m, f[e]);
      vmax[j] = m;
      tmax = fmaxf(tmax, m);
      if (m > r + kMove) {
        const float to = fminf(m, -kLeast), d = fmaxf(r - to, kBound), g = __builtin_amdgcn_exp2f(d * kC);
        u0 = fmaf(s0, d, u0) * g;
        u1 = fmaf(s1, d, u1) * g;
        s0 *= g;
        s1 *= g;
        r = to;
      }
      float sum[VEC];
#pragma unroll
      for (int e = 0; e < VEC; ++e) {
        const float d = f[e] - r, p = __builtin_amdgcn_exp2f(d * kC);
        sum[e] = p;
        (e & 1 ? u1 : u0) = fmaf(p, fmaxf(d, kBound), e & 1 ? u1 : u0);
      }
#pragma unroll
      for (int n = VEC / 2; n; n /= 2)
#pragma unroll
        for (int e = 0; e < n; ++e) sum[e] += sum[e + n];
      (j & 1 ? s1 : s0) += sum[0];
    }

    if constexpr (TOP) {
      const int at = e0 + ch * CHUNK;
      if (have < k) {  // a bound from the groups' maxima: of 4 threads, of 2 where 64 groups leave too low a one
        const bool fine = k > 32;
        const int groups = fine ? kThreads / 2 : kThreads / 4;
        float gm = fmaxf(tmax, dpp_f32<kDppXor1>(tmax));
        if (!fine) gm = fmaxf(gm, dpp_f32<kDppXor2>(gm));
        const int gi = fine ? t / 2 : t / 4;
        if (gi * (kThreads / groups) == t) s_own[gi] = key_of(gm, gi);
        __syncthreads();
        if (t < groups) {
          const uint64_t mine = s_own[t];
          int above = 0;
#pragma unroll 16
          for (int j = 0; j < groups; ++j) above += s_own[j] > mine;
          // (below -inf there is NaN, which the maxima passed over)
          if (above == k - 1) s_bound = mine >> 32 > kLowest ? mine >> 32 << 32 : 0;
        }
      }
      __syncthreads();
      auto each = [&](uint64_t bound, auto&& f) __attribute__((always_inline)) {
        const float least = bound >> 32 > kLowest ? value_of((uint32_t)(bound >> 32)) : -INFINITY;
#pragma unroll
        for (int j = 0; j < kVecs; ++j) {
          const int i = at + (j * kThreads + t) * VEC;
          if (!in_use(j)) break;
          if (vmax[j] < least || i >= e1) continue;  // (NaN: not less)
          float v[VEC];
          Store<T>::unpack(cur[j], v);
#pragma unroll
          for (int e = 0; e < VEC; ++e) {
            const uint64_t key = key_of(v[e], i + e);
            if (i + e < e1 && key >= bound) f(key);
          }
        }
      };
      auto append = [&](uint64_t key) __attribute__((always_inline)) {
        const int to = have + atomicAdd(&s_n, 1);
        if (to < kListCap) s_list[to] = key;
      };
      each(s_bound, append);
      __syncthreads();
      int total = have + s_n;
      if (total > kListCap) {  // (block-uniform) a bound from each thread's largest key
        const uint64_t was = s_bound;
        uint64_t best = 0;
        each(was, [&](uint64_t key) __attribute__((always_inline)) { best = key > best ? key : best; });
        s_own[t] = best;
        __syncthreads();
        if (t == 0) s_n = 0;
        int above = 0;
#pragma unroll 8
        for (int j = 0; j < kThreads; ++j) above += s_own[j] > best;
        if (best && above == k - 1) s_bound = best;
        __syncthreads();
        each(s_bound, append);
        __syncthreads();
        total = min(have + s_n, kListCap);
      }
      if (total > have) {
        rank_keys(s_list, total, s_top, k, kThreads);
        __syncthreads();
        have = min(total, k);
        if (t < have) s_list[t] = s_top[t];
        if (t == 0) {
          s_n = 0;
          if (have == k) s_bound = s_top[k - 1];
        }
      }
      __syncthreads();
    }
  };
  for (int ch = 0; ch + 1 < n_chunk; ++ch) {
    load(next, ch + 1);
    take(ch, std::false_type{});
#pragma unroll
    for (int j = 0; j < kVecs; ++j) cur[j] = next[j];
  }
  fix(cur, n_chunk - 1);
  take(n_chunk - 1, std::true_type{});

  // the block's statistics
  Stat st = join_wave(Stat{r, s0 + s1, u0 + u1});
  if (lane == 0) s_stat[w] = st;
  __syncthreads();
  st = s_stat[0];
#pragma unroll
  for (int j = 1; j < kWaves; ++j) st = join(st, s_stat[j]);

  if (la.splits > 1) {
    if (t == 0) la.part[blockIdx.x] = make_float4(st.r, st.s, st.u, 0.f);
    if (TOP && t < k) la.part_top[(int64_t)blockIdx.x * k + t] = t < have ? s_list[t] : 0;
    return;
  }
  if (t == 0) finish<T>(la, row, st, target);
  if (TOP && t < k) put_top(la, row, t, s_list[t], st);
}

// The splits of a row joined, in their order.
template <typename T>
__global__ void __launch_bounds__(256) logprob_merge_kernel(LogpArgs la) {
  constexpr int KEYS = kLogpSplits * kLogpTop;
  __shared__ uint64_t s_first[2 * kLogpTop], s_list[KEYS], s_top[kLogpTop], s_bound;
  __shared__ int s_n;
  const int row = blockIdx.x, t = threadIdx.x, lane = t & 63, k = la.n_top, n = la.splits * k;
  static_assert(kLogpSplits <= 64, "a split a lane");
  const uint64_t* keys = la.part_top + (int64_t)row * n;
  Target<T> target(la, row);
  Stat st{kLeast, 0.f, 0.f};
  if (lane < la.splits) {
    const float4 p = la.part[(int64_t)row * la.splits + lane];
    st = Stat{p.x, p.y, p.z};
  }
  uint64_t mine[KEYS / 256];  // (empty places, 0, lie below every key)
#pragma unroll
  for (int j = 0; j < KEYS / 256; ++j)
    if (j * 256 < n) mine[j] = j * 256 + t < n ? keys[j * 256 + t] : 0;
  target.load(la, row);
  st = join_wave(st);
  if (t == 0) finish<T>(la, row, st, target);
  if (!k) return;
  // A lower bound on the row's k-th key: the k-th of the splits' first few, k in all or a
  // few more (a split's own k-th lies far below where there are many splits).
  const int m = (k + la.splits - 1) / la.splits, q = m * la.splits;
  static_assert(kLogpSplits <= kLogpTop, "q < 2 kLogpTop");
#pragma unroll
  for (int j = 0; j < KEYS / 256; ++j) {
    const int i = j * 256 + t, split = i / k, at = i - split * k;
    if (j * 256 < n && i < n && at < m) s_first[split * m + at] = mine[j];
  }
  if (t == 0) s_n = 0;
  __syncthreads();
  if (t < q) {
    const uint64_t own = s_first[t];
    int above = 0;
#pragma unroll 8
    for (int j = 0; j < q; ++j) above += s_first[j] > own || (s_first[j] == own && j < t);  // (several empty places)
    if (above == k - 1) s_bound = own;
  }
  __syncthreads();
#pragma unroll
  for (int j = 0; j < KEYS / 256; ++j)
    if (j * 256 < n && j * 256 + t < n && mine[j] >= s_bound && mine[j]) s_list[atomicAdd(&s_n, 1)] = mine[j];
  __syncthreads();
  rank_keys(s_list, s_n, s_top, k, 256);
  __syncthreads();
  if (t < k) put_top(la, row, t, s_top[t], st);
}

// dx = p (g_lse - g_logprob - g_entropy (ln p + H)), and g_logprob more at the target
template <typename T>
__global__ void __launch_bounds__(256) logprob_grad_kernel(LogpGradArgs ga, int64_t block0) {
  constexpr int VEC = Store<T>::VEC;
  const int64_t b = block0 + blockIdx.x;
  const int row = (int)(b / ga.chunks), chunk = (int)(b - (int64_t)row * ga.chunks);
  const T* x = reinterpret_cast<const T*>(ga.x) + (int64_t)row * ga.stride;
  T* dx = reinterpret_cast<T*>(ga.dx) + (int64_t)row * ga.d_stride;
  uint4 v[kLogpGradVecs];
  const int i0 = (chunk * kLogpGradVecs * 256 + (int)threadIdx.x) * VEC;
#pragma unroll
  for (int j = 0; j < kLogpGradVecs; ++j) {
    const int i = i0 + j * 256 * VEC;
    if (i + VEC <= ga.vocab) v[j] = ld16_any(x + i);
  }
  const int tgt = ga.targets ? ga.targets[row] : -1;
  const float gl = ga.g_logprob && tgt >= 0 && tgt < ga.vocab ? ga.g_logprob[row] : 0.f;
  const float gh = ga.g_entropy ? ga.g_entropy[row] : 0.f, gs = ga.g_lse ? ga.g_lse[row] : 0.f;
  const float lse = ga.lse[row], ent = ga.g_entropy ? ga.entropy[row] : 0.f;
  const float a = gs - gl - gh * ent;
  auto grad = [&](float f, int i) __attribute__((always_inline)) -> float {
    const float lp = f - lse, p = __builtin_amdgcn_exp2f(lp * kC);
    float d = p * fmaf(-gh, lp, a);
    d = f == -INFINITY || p == 0.f ? 0.f : d;  // (a row of nothing but -inf has no gradient)
    return i == tgt ? d + gl : d;
  };
#pragma unroll
  for (int j = 0; j < kLogpGradVecs; ++j) {
    const int i = i0 + j * 256 * VEC;
    if (i + VEC <= ga.vocab) {
      float f[VEC];
      Store<T>::unpack(v[j], f);
#pragma unroll
      for (int e = 0; e < VEC; ++e) f[e] = grad(f[e], i + e);
      st16_any(dx + i, Store<T>::pack(f));
    }
  }
  const int e = ga.vocab / VEC * VEC + (int)threadIdx.x;  // what is left of the row, an element a lane
  if (chunk == ga.chunks - 1 && e < ga.vocab) Store<T>::store1(dx + e, grad(Store<T>::load1(x + e), e));
}

namespace {

int check(hipError_t e) { return e == hipSuccess ? 0 : (int)e; }

}  // namespace

int launch_logprobs(int dtype, const LogpArgs& args, hipStream_t s) {
  const dim3 grid(args.n * args.splits);
#define LP(T, TOP, ST) hipLaunchKernelGGL((logprob_kernel<T, TOP, ST>), grid, dim3(kThreads), 0, s, args)
#define LPS(T, TOP) { if (args.stream) LP(T, TOP, true); else LP(T, TOP, false); }
  if (dtype == 0) { if (args.n_top) LPS(float, true) else LPS(float, false) }
  else { if (args.n_top) LPS(bf16_t, true) else LPS(bf16_t, false) }
#undef LPS
#undef LP
  if (int rc = check(hipGetLastError())) return rc;
  if (args.splits == 1) return 0;
  if (dtype == 0) hipLaunchKernelGGL((logprob_merge_kernel<float>), dim3(args.n), dim3(256), 0, s, args);
  else hipLaunchKernelGGL((logprob_merge_kernel<bf16_t>), dim3(args.n), dim3(256), 0, s, args);
  return check(hipGetLastError());
}

int launch_logprobs_grad(int dtype, const LogpGradArgs& args, hipStream_t s) {
  const int64_t blocks = (int64_t)args.n * args.chunks;
  for (int64_t b = 0; b < blocks; b += kGridX) {
    const dim3 grid((uint32_t)(blocks - b < kGridX ? blocks - b : kGridX));
    if (dtype == 0) hipLaunchKernelGGL((logprob_grad_kernel<float>), grid, dim3(256), 0, s, args, b);
    else hipLaunchKernelGGL((logprob_grad_kernel<bf16_t>), grid, dim3(256), 0, s, args, b);
    if (int rc = check(hipGetLastError())) return rc;
  }
  return 0;
}

}  // namespace fcg

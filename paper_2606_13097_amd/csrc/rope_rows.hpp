// Rows of queries, keys and values in blocks: what rotary encoding into tensors or
// into a cache (k_rope.hip) and the same behind a norm of each row (k_norm_rope.hip)
// share.  A block moves one pass of rows (kRopePass pairs of vectors, a pair for each
// lane) of up to 16 tokens at consecutive indices (and, appending, at consecutive
// positions of one sequence), of one layer or of every gridDim.z-th; which vectors a
// lane takes is explained in k_rope.hip.
#pragma once

#include "fcg_device.hpp"
#include "kernels.hpp"

namespace fcg {

// sum over each group of N lanes (4, 8 or 16), every lane ending with it
template <int N>
__device__ __forceinline__ float sum_lanes(float v) {
  static_assert(N == 4 || N == 8 || N == 16, "lanes of a row");
  v += dpp_f32<kDppXor1>(v);
  v += dpp_f32<kDppXor2>(v);
  if (N >= 8) v += dpp_f32<kDppHalfMirror>(v);
  if (N >= 16) v += dpp_f32<kDppMirror>(v);
  return v;
}

// 1 / sqrt(mean of squares + eps) of a row, from the sum of squares of the lane's part
template <typename T, int D>
__device__ __forceinline__ float norm_scale(float sum, float eps) {
  return 1.f / sqrtf(sum_lanes<D / (2 * Store<T>::VEC)>(sum) * (1.f / D) + eps);
}

// The norm of a lane's two vectors of a row:
//   x -> (offset + weight) x / sqrt(mean of x^2 + eps),
// the mean over the head's D elements, in fp32, rounded only after the turn.
template <typename T, bool NORM>
struct NormLane {
  static constexpr bool on = false;
  __device__ __forceinline__ NormLane(const NormArgs<NORM>&, int, int, int, int) {}
  __device__ __forceinline__ void load(int) {}
};
template <typename T>
struct NormLane<T, true> {
  static constexpr int VEC = Store<T>::VEC;
  const T* w;  // the head's weights of layer 0, or null
  int64_t layer;
  float eps, offset;
  int lo, hi;
  bool on;
  uint4 wa, wb;
  __device__ __forceinline__ NormLane(const NormArgs<true>& n, int kind, int head, int lo_, int hi_) : lo(lo_), hi(hi_) {
    // (fields chosen from scalar registers: a view chosen by address is loaded lane by lane,
    // field after field, before the first row)
    const NormView q = n.q, k = n.k;
    const bool is_q = kind == 0;
    on = kind != 2 && (is_q ? q.on : k.on);
    const int64_t step = is_q ? q.head : k.head;
    const T* first = reinterpret_cast<const T*>(is_q ? q.w : k.w);
    w = on && first ? first + head * step : nullptr;
    layer = is_q ? q.layer : k.layer;
    eps = is_q ? q.eps : k.eps;
    offset = w ? is_q ? q.offset : k.offset : 1.f;
    wa = wb = make_uint4(0, 0, 0, 0);
  }
  __device__ __forceinline__ void load(int l) {
    if (!w) return;
    wa = ld16_any(w + l * layer + lo);
    wb = ld16_any(w + l * layer + hi);
  }
  template <int D>
  __device__ __forceinline__ void apply(float* xa, float* xb) const {
    float sum = 0.f;
#pragma unroll
    for (int e = 0; e < VEC; ++e) sum = fmaf(xa[e], xa[e], sum);
#pragma unroll
    for (int e = 0; e < VEC; ++e) sum = fmaf(xb[e], xb[e], sum);
    const float r = norm_scale<T, D>(sum, eps);
    if (!on) return;
    float fa[VEC], fb[VEC];
    Store<T>::unpack(wa, fa);
    Store<T>::unpack(wb, fb);
#pragma unroll
    for (int e = 0; e < VEC; ++e) {
      xa[e] *= r * (offset + fa[e]);
      xb[e] *= r * (offset + fb[e]);
    }
  }
};

constexpr int kApply = 0, kAppendArgs = 1, kAppendList = 2;

template <int MODE>
struct Where {};
template <>
struct Where<kApply> {
  const int32_t* pos;
};
template <>
struct Where<kAppendArgs> {
  AppendArgs a;
  int32_t n_runs;
};
template <>
struct Where<kAppendList> {
  const AppendGroup* groups;
};

// group b of a plan by value: its run is the last one whose first group is at
// most b; every lane of a wave holds one run, so one vector load finds it
__device__ __forceinline__ AppendGroup find_group(const Where<kAppendArgs>& w, int b, int tb) {
  static_assert(kAppRuns == 64, "one run per lane");
  const int lane = threadIdx.x & 63;
  const AppendRun mine = w.a.run[min(lane, w.n_runs - 1)];
  const uint64_t below = __builtin_amdgcn_ballot_w64(lane < w.n_runs && mine.grp0 <= b);
  const int r = 63 - __builtin_clzll(below);
  const int tok0 = __builtin_amdgcn_readlane(mine.tok0, r), seq = __builtin_amdgcn_readlane(mine.seq, r);
  const int pos0 = __builtin_amdgcn_readlane(mine.pos0, r), n = __builtin_amdgcn_readlane(mine.n, r);
  const int grp0 = __builtin_amdgcn_readlane(mine.grp0, r), pg = __builtin_amdgcn_readlane(mine.page0, r);
  const int j = (b - grp0) * tb;
  AppendGroup g;
  g.tok0 = tok0 + j;
  g.seq = seq;
  g.pos0 = pos0 + j;
  g.n = min(tb, n - j);
  g.enter = pg < 0;
  const int e = (pg & 0x7FFFFFFF) + (g.pos0 >> 4) - (pos0 >> 4);
  g.page_a = w.a.page[min(e, kAppPages - 1)];
  g.page_b = w.a.page[min(e + 1, kAppPages - 1)];
  g.pad = 0;
  return g;
}

// The rows of one block.  NORM: queries and keys are normalised first (NormLane), each by the lanes that hold its row.
template <typename T, int D, bool PAIRS, int MODE, bool PAGED, bool NORM>
__device__ __forceinline__ void rope_rows(const Where<MODE>& where, const RopeRows& rows, const CacheView& cv, int layer0,
                                          const RopeArgs& ra, const float2* __restrict__ tab,
                                          const NormArgs<NORM>& norm) {
  constexpr int VEC = Store<T>::VEC;
  constexpr int NCH = D / (2 * VEC);  // vector pairs of a row
  __shared__ __align__(16) float2 s_cs[kAppMaxTb * kRopePairs];

  const int t = threadIdx.x;
  AppendGroup g;
  if constexpr (MODE == kApply) {
    g.tok0 = blockIdx.x * rows.tb;
    g.n = min(rows.tb, rows.n_tok - g.tok0);
  } else if constexpr (MODE == kAppendArgs) {
    g = find_group(where, blockIdx.x, rows.tb);
  } else {
    g = where.groups[blockIdx.x];
  }
  const int half = ra.rot / 2;
  const int H = rows.Hq + rows.Hk + rows.Hv;
  const int r0 = blockIdx.y * rows.slice_rows;
  const int nrow = min(rows.slice_rows, g.n * H - r0);  // rows of this block, token-major
  if (nrow <= 0) return;  // (block-uniform) a slice past a short group's rows
  const int total = nrow * NCH;
  auto tl_of = [&](int r) __attribute__((always_inline)) {  // r / H
    return H == 1 ? r : (int)__umulhi((unsigned)r, rows.h_magic);
  };
  const int tl0 = tl_of(r0);
  const int rchunks = half / VEC;  // vector pairs that turn

  if constexpr (MODE != kApply && PAGED) {
    if (g.enter && blockIdx.y == 0 && blockIdx.z == 0 && t == 0) {
      int32_t* row = const_cast<int32_t*>(cv.page_table) + (int64_t)g.seq * 2 * cv.n_lp + (g.pos0 >> 4);
      row[0] = g.page_a;
      row[cv.n_lp] = -1;
      if (((g.pos0 + g.n - 1) >> 4) != (g.pos0 >> 4)) {
        row[1] = g.page_b;
        row[cv.n_lp + 1] = -1;
      }
    }
  }

  // This lane's vectors: vector pair c of a row (token tl of the group, q, k or v,
  // head); lanes past the rows repeat the last one and store nothing.
  const bool mine = t < total;
  const int i = min(t, total - 1), c = i % NCH, r = r0 + i / NCH;
  const int tl = tl_of(r), hh = r - tl * H;
  const int kind = hh < rows.Hq ? 0 : hh < rows.Hq + rows.Hk ? 1 : 2;
  const int head = hh - (kind == 0 ? 0 : kind == 1 ? rows.Hq : rows.Hq + rows.Hk);
  const bool turn = kind != 2 && c < (PAIRS ? 2 * rchunks : rchunks);  // the first vector, for halves both
  // element offsets of the two vectors in the row
  const int lo = (!PAIRS && kind != 2 && c >= rchunks ? rchunks + c : c) * VEC;
  const int hi = (!PAIRS && kind != 2 && c < rchunks ? rchunks + c : NCH + c) * VEC;
  auto row_of = [&](const RowView& v) __attribute__((always_inline)) {  // of layer 0
    return reinterpret_cast<const T*>(v.p) + (int64_t)(g.tok0 + tl) * v.token + (int64_t)head * v.head;
  };
  const T* src = row_of(kind == 0 ? rows.q : kind == 1 ? rows.k : rows.v);
  const int64_t src_layer = kind == 0 ? rows.q.layer : kind == 1 ? rows.k.layer : rows.v.layer;
  const bool to_cache = MODE != kApply && kind != 0;
  T* dst;
  int64_t dst_layer;
  if (!to_cache) {
    dst = const_cast<T*>(row_of(kind == 0 ? rows.q_out : rows.k_out));
    dst_layer = kind == 0 ? rows.q_out.layer : rows.k_out.layer;
  } else {
    const int pos = g.pos0 + tl;
    int64_t off = (int64_t)layer0 * cv.layer_stride;
    if (PAGED) {
      const int page = (pos >> 4) == (g.pos0 >> 4) ? g.page_a : g.page_b;
      off += (((int64_t)page * cv.n_kv_heads + head) * 16 + (pos & 15)) * D;
    } else {
      off += (((int64_t)g.seq * cv.n_kv_heads + head) * cv.max_tokens + pos) * D;
    }
    dst = reinterpret_cast<T*>(kind == 1 ? cv.k : cv.v) + off;
    dst_layer = cv.layer_stride;
  }
  uint4 a, b;
  NormLane<T, NORM> nl(norm, kind, head, lo, hi);
  auto load = [&](int layer) __attribute__((always_inline)) {
    const T* p = src + layer * src_layer;
    if (rows.stream) {  // (uniform) more than the last-level cache holds
      a = ld16_nt_any(p + lo);
      b = ld16_nt_any(p + hi);
    } else {
      a = ld16_any(p + lo);
      b = ld16_any(p + hi);
    }
    nl.load(layer);
  };
  load(blockIdx.z);

  // the (cos, sin) of the rows' tokens
  const int n_cs = (tl_of(r0 + nrow - 1) - tl0 + 1) * half;
  for (int j = t; j < n_cs; j += 256) {
    const int tj = tl0 + j / half, pr = j % half;
    float cs, sn;
    if (MODE != kApply && tab) {
      const float2 e = tab[(int64_t)(g.pos0 + tj) * half + pr];
      cs = e.x;
      sn = e.y;
    } else {
      int pos;
      if constexpr (MODE == kApply) pos = where.pos[g.tok0 + tj];
      else pos = g.pos0 + tj;
      rope_cs_turns((double)pos, ra.turns[pr], &cs, &sn);
      cs *= ra.m;
      sn *= ra.m * rows.sign;
    }
    s_cs[j] = make_float2(cs, sn);
  }
  __syncthreads();

  const float2* cs = s_cs + (tl - tl0) * half + c * (PAIRS ? VEC / 2 : VEC);  // of the lane's first pair
  for (int layer = blockIdx.z; layer < rows.n_layers; layer += gridDim.z) {
    uint4 ya = a, yb = b;
    float xa[VEC], xb[VEC];
    if constexpr (NORM) {
      Store<T>::unpack(ya, xa);
      Store<T>::unpack(yb, xb);
      nl.template apply<D>(xa, xb);
      if (nl.on && !turn) ya = Store<T>::pack(xa);
      if (nl.on && (!turn || PAIRS)) yb = Store<T>::pack(xb);
    }
    if (layer + (int)gridDim.z < rows.n_layers) load(layer + gridDim.z);
    if (turn) {
      float za[VEC], zb[VEC];
      if constexpr (!NORM) {
        Store<T>::unpack(ya, xa);
        Store<T>::unpack(yb, xb);
      }
      if constexpr (PAIRS) {
        constexpr int P = VEC / 2;  // pairs of a vector
#pragma unroll
        for (int e = 0; e < P; ++e) {
          za[2 * e] = fmaf(xa[2 * e], cs[e].x, -xa[2 * e + 1] * cs[e].y);
          za[2 * e + 1] = fmaf(xa[2 * e + 1], cs[e].x, xa[2 * e] * cs[e].y);
        }
        ya = Store<T>::pack(za);
        if (NCH + c < 2 * rchunks) {
#pragma unroll
          for (int e = 0; e < P; ++e) {
            const float2 c2 = cs[NCH * P + e];
            zb[2 * e] = fmaf(xb[2 * e], c2.x, -xb[2 * e + 1] * c2.y);
            zb[2 * e + 1] = fmaf(xb[2 * e + 1], c2.x, xb[2 * e] * c2.y);
          }
          yb = Store<T>::pack(zb);
        }
      } else {
#pragma unroll
        for (int e = 0; e < VEC; ++e) {
          za[e] = fmaf(xa[e], cs[e].x, -xb[e] * cs[e].y);
          zb[e] = fmaf(xb[e], cs[e].x, xa[e] * cs[e].y);
        }
        ya = Store<T>::pack(za);
        yb = Store<T>::pack(zb);
      }
    }
    if (!mine) continue;
    T* p = dst + layer * dst_layer;
    // Caller tensors are read next: plain stores leave them in the last-level cache (keys
    // of 32 layers of 713 tokens, new inputs each pass: 20 us and 30 with a kernel that reads
    // them, past the caches 16 and 33; fp32 gradients of 4.7K tokens 23 and 41, 17 and 51).
    // Cache rows, and results larger than that cache, go past the L2: whoever reads them next
    // runs on any XCD (8 layers of 11K tokens into pages 447 -> 432 us, 32 layers of 129 into
    // a contiguous cache 21.0 -> 20.3).
    if (to_cache) {
      st16_nt(p + lo, ya);
      st16_nt(p + hi, yb);
    } else if (rows.stream) {
      st16_nt_any(p + lo, ya);
      st16_nt_any(p + hi, yb);
    } else {
      st16_any(p + lo, ya);
      st16_any(p + hi, yb);
    }
  }
}

}  // namespace fcg

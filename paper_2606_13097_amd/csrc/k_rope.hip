// Rotary encoding of rows in any of the rotary forms, into a caller's tensor
// (rope apply) or into a cache (append), for gfx950.
//
//   (a, b) -> (m (a cos - b sin), m (b cos + a sin)),  angle p w_i,
// for the pairs (i, i + R/2) or (2i, 2i + 1) of the first R dimensions of a
// head; the others are copied.  The backward pass negates the angle.
//
// A block moves one pass of rows (kRopePass pairs of vectors, a pair for each
// lane) of up to 16 tokens at consecutive indices (and, appending, at consecutive
// positions of one sequence), of one layer or of every gridDim.z-th.  The (cos,
// sin) of its tokens' pairs are computed once into LDS while the first rows' loads
// are in flight, and shared by heads and layers; with several layers, the next
// one's rows are requested before the last one's are turned and stored.  A lane
// moves two 16-byte vectors of a row, chosen so that every form turns registers
// only and that neighbouring lanes move neighbouring vectors: for halves, vectors
// c and c + R / 2 / VEC hold both ends of VEC pairs; for neighbours each vector
// holds whole pairs, and a lane takes vectors c and c + D / 2 / VEC; what passes
// unturned is cut in halves likewise.  (With 2c and 2c + 1 each access covered
// every other 16 bytes.)  Caller rows start at any element (unaligned 16-byte
// accesses); cache rows are aligned.
//
// What bounds it: many tokens, the memory (bf16, D 128: keys of 32 layers of 713
// tokens of 8 heads, 93 MB read and written, 15.5 us on the same buffers again and
// 17.6 on new ones, a copy of as many bytes 13.6 and 19.3; keys, values and queries of
// 8 layers of 11K tokens into pages, 2.2 GB, 390 us, 5.6 TB/s, a copy 5.2); few, the
// chain of argument fetch, position, rows and stores (3 us for one token).
#include "fcg_device.hpp"
#include "kernels.hpp"

namespace fcg {

namespace {

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

}  // namespace

template <typename T, int D, bool PAIRS, int MODE, bool PAGED>
__global__ void __launch_bounds__(256) rope_rows_kernel(Where<MODE> where, RopeRows rows, CacheView cv, int layer0,
                                                        RopeArgs ra, const float2* __restrict__ tab) {
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
  auto load = [&](int layer) __attribute__((always_inline)) {
    const T* p = src + layer * src_layer;
    if (rows.stream) {  // (uniform) more than the last-level cache holds
      a = ld16_nt_any(p + lo);
      b = ld16_nt_any(p + hi);
    } else {
      a = ld16_any(p + lo);
      b = ld16_any(p + hi);
    }
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
    if (layer + (int)gridDim.z < rows.n_layers) load(layer + gridDim.z);
    if (turn) {
      float xa[VEC], xb[VEC], za[VEC], zb[VEC];
      Store<T>::unpack(ya, xa);
      Store<T>::unpack(yb, xb);
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

namespace {

int check(hipError_t e) { return e == hipSuccess ? 0 : (int)e; }

template <int MODE, bool PAGED>
void launch_rows(int dtype, int D, bool pairs, dim3 grid, const Where<MODE>& where, const RopeRows& rows,
                 const CacheView& cv, int layer0, const RopeArgs& ra, const float2* tab, hipStream_t s) {
#define RR(T, DD, PR)                                                                                              \
  hipLaunchKernelGGL((rope_rows_kernel<T, DD, PR, MODE, PAGED>), grid, dim3(256), 0, s, where, rows, cv, layer0, ra, \
                     tab)
#define RRP(T, DD) { if (pairs) RR(T, DD, true); else RR(T, DD, false); }
  if (dtype == 0) { if (D == 64) RRP(float, 64) else RRP(float, 128) }
  else { if (D == 64) RRP(bf16_t, 64) else RRP(bf16_t, 128) }
#undef RRP
#undef RR
}

}  // namespace

int launch_rope_apply(int dtype, int D, bool pairs, const RopeRows& rows, const int32_t* pos, const RopeArgs& ra,
                      hipStream_t s) {
  const int H = rows.Hq + rows.Hk;
  const dim3 grid((rows.n_tok + rows.tb - 1) / rows.tb, (rows.tb * H + rows.slice_rows - 1) / rows.slice_rows,
                  rows.grid_layers);
  launch_rows<kApply, false>(dtype, D, pairs, grid, Where<kApply>{pos}, rows, CacheView{}, 0, ra, nullptr, s);
  return check(hipGetLastError());
}

int launch_append(int dtype, bool pairs, const RopeRows& rows, const AppendArgs& args, int n_runs,
                  const AppendGroup* groups, int n_groups, const CacheView& cv, int layer0, const RopeArgs& ra,
                  const float2* tab, hipStream_t s) {
  const int H = rows.Hq + rows.Hk + rows.Hv;
  const dim3 grid(n_groups, (rows.tb * H + rows.slice_rows - 1) / rows.slice_rows, rows.grid_layers);
#define AP(PG)                                                                                                     \
  {                                                                                                                \
    if (groups)                                                                                                    \
      launch_rows<kAppendList, PG>(dtype, cv.head_dim, pairs, grid, Where<kAppendList>{groups}, rows, cv, layer0, ra, \
                                   tab, s);                                                                        \
    else                                                                                                           \
      launch_rows<kAppendArgs, PG>(dtype, cv.head_dim, pairs, grid, Where<kAppendArgs>{args, n_runs}, rows, cv, layer0, \
                                   ra, tab, s);                                                                    \
  }
  if (cv.page_size) AP(true) else AP(false)
#undef AP
  return check(hipGetLastError());
}

}  // namespace fcg

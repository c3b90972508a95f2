// Norms of query and key rows with their rotary turn in one pass, and the gradient of
// both, for gfx950.
//
//   y = R(p) n,  n = (o + w) x s,  s = 1 / sqrt(mean(x^2) + eps),
//
// R(p) the turn of k_rope.hip (with its factor m), the mean over the head's D elements.
// With g the gradient of y:
//   dn = R(p)^T g,  dw = sum over rows of dn x s,
//   dx = s (dn (o + w) - x s mean(dn (o + w) x s)).
// All of it in fp32, rounded once.
//
// Forward: the blocks of rope_rows.hpp; the D / (2 VEC) lanes that hold a row add up its
// squares by DPP, so the norm costs no memory round trip and no LDS beside the turn.  Bound by
// the memory: 4.4K tokens of 32 + 8 bf16 heads of 128, 18.7 us, 5.1 TB/s (the fastest copies 6.2);
// one token appended 4.4 us, a launch.
//
// Backward: a block takes chunks of 16 to 64 tokens, as many as it holds a row of each, whose
// (cos, sin) are computed once into LDS, and up to kNormHeads heads of them; a lane holds the
// same two vectors of every row it takes, so it adds up its part of dw in registers; the lanes
// of a wave that hold the same vectors join theirs by lane exchanges, after each head (or, with
// one weight vector for all, once), into the wave's own sums in LDS: no barrier.  The blocks'
// partials are added by a second launch in a fixed order: no atomics, so the same call gives
// the same bits.  4.4K tokens of 16 + 4 fp32 heads: 30 + 4 us, 4.7 TB/s in the first; bound by
// the memory and, for a quarter of the time, the angles and the joins.  In bf16 every range of
// heads computes as many angles for half the bytes: 32 + 8 heads 44 + 5 us, 3.1 TB/s.
#include "rope_rows.hpp"

namespace fcg {

template <typename T, int D, bool PAIRS, int MODE, bool PAGED>
__global__ void __launch_bounds__(256) norm_rope_kernel(Where<MODE> where, RopeRows rows, CacheView cv, int layer0,
                                                        RopeArgs ra, const float2* __restrict__ tab,
                                                        NormArgs<true> norm) {
  rope_rows<T, D, PAIRS, MODE, PAGED, true>(where, rows, cv, layer0, ra, tab, norm);
}

// sum over the lanes of a wave that are equal modulo N (4, 8 or 16)
template <int N>
__device__ __forceinline__ float sum_same(float v) {
  if (N <= 8) v += dpp_f32<0x128>(v);  // row_ror:8
  if (N <= 4) v += dpp_f32<0x124>(v);  // row_ror:4
  return sum_rows4(v);
}

template <typename T, int D, bool PAIRS>
__global__ void __launch_bounds__(256) norm_rope_grad_kernel(NormGradArgs args, RopeArgs ra) {
  constexpr int VEC = Store<T>::VEC;
  constexpr int NCH = D / (2 * VEC);  // lanes of a row
  constexpr int TK = 256 / NCH;       // tokens of a chunk, a row of each at a time
  static_assert(TK == norm_tokens(D, sizeof(T)), "as the host counts them");
  __shared__ __align__(16) float2 s_cs[TK * D / 2];
  __shared__ __align__(16) float s_dw[4][kNormHeads * D];  // each wave's dw

  const int t = threadIdx.x, c = t % NCH, tr = t / NCH, lane = t & 63, w = t >> 6;
  const int bs = blockIdx.x < args.blocks_q ? 0 : 1, b = blockIdx.x - (bs ? args.blocks_q : 0);
  const NormSide& sd = args.side[bs];
  const int layer = blockIdx.y;
  const int hb = b / sd.spread, tc = b - hb * sd.spread;  // head range; first chunk of tokens
  const int h0 = hb * sd.heads_per, nh = min(sd.heads_per, sd.heads - h0);
  const bool own_w = sd.w_heads > 1;  // a weight vector for each head
  const bool has_dw = sd.dw != nullptr;
  const int half = ra.rot / 2, rchunks = half / VEC;
  const bool turn_a = c < (PAIRS ? 2 * rchunks : rchunks), turn_b = PAIRS ? NCH + c < 2 * rchunks : turn_a;
  const int lo = (!PAIRS && c >= rchunks ? rchunks + c : c) * VEC;
  const int hi = (!PAIRS && c < rchunks ? rchunks + c : NCH + c) * VEC;
  const float inv_d = 1.f / D;

  float dwa[VEC], dwb[VEC];
#pragma unroll
  for (int e = 0; e < VEC; ++e) dwa[e] = dwb[e] = 0.f;
  if (has_dw)
    for (int j = lane; j < (own_w ? nh : 1) * D; j += 64) s_dw[w][j] = 0.f;

  // the lanes' parts of dw into the wave's sums of a weight vector
  auto join = [&](float* dst) __attribute__((always_inline)) {
#pragma unroll
    for (int e = 0; e < VEC; ++e) {
      const float a = sum_same<NCH>(dwa[e]), b = sum_same<NCH>(dwb[e]);
      if (lane < NCH) {
        dst[lo + e] += a;
        dst[hi + e] += b;
      }
      dwa[e] = dwb[e] = 0.f;
    }
  };

  const int n_chunk = (args.n_tok + TK - 1) / TK;
  for (int ch = tc; ch < n_chunk; ch += sd.spread) {
    const int tok0 = ch * TK, n = min(TK, args.n_tok - tok0);
    const bool mine = tr < n;
    uint4 xa, xb, ga, gb, wa = make_uint4(0, 0, 0, 0), wb = wa;
    auto row_of = [&](const RowView& v, int step) __attribute__((always_inline)) {
      const int tok = tok0 + min(tr, n - 1);
      return reinterpret_cast<const T*>(v.p) + (int64_t)layer * v.layer + (int64_t)tok * v.token +
             (int64_t)(h0 + step) * v.head;
    };
    auto load = [&](int step) __attribute__((always_inline)) {
      const T *x = row_of(sd.x, step), *g = row_of(sd.gy, step);
      xa = ld16_any(x + lo);
      xb = ld16_any(x + hi);
      ga = ld16_any(g + lo);
      gb = ld16_any(g + hi);
      // (beside the rows: a load asked for later is waited for with all before it)
      if (sd.norm.w && (step == 0 || own_w)) {
        const T* wt = reinterpret_cast<const T*>(sd.norm.w) + layer * sd.norm.layer +
                      (int64_t)(h0 + step) * sd.norm.head;
        wa = ld16_any(wt + lo);
        wb = ld16_any(wt + hi);
      }
    };
    load(0);
    __syncthreads();  // the chunk before has been read
    for (int j = t; j < n * half; j += 256) {
      float cs, sn;
      rope_cs_turns((double)args.pos[tok0 + j / half], ra.turns[j % half], &cs, &sn);
      s_cs[j] = make_float2(cs * ra.m, sn * ra.m);
    }
    __syncthreads();
    for (int step = 0; step < nh; ++step) {  // a head
      float x[2 * VEC], g[2 * VEC], f[2 * VEC];
      Store<T>::unpack(xa, x);
      Store<T>::unpack(xb, x + VEC);
      Store<T>::unpack(ga, g);
      Store<T>::unpack(gb, g + VEC);
      Store<T>::unpack(wa, f);
      Store<T>::unpack(wb, f + VEC);
      if (step + 1 < nh) load(step + 1);
      // dn = R^T g
      const float2* cs = s_cs + min(tr, n - 1) * half + c * (PAIRS ? VEC / 2 : VEC);
      if constexpr (PAIRS) {
        constexpr int P = VEC / 2;
        if (turn_a) {
#pragma unroll
          for (int e = 0; e < P; ++e) {
            const float a = g[2 * e], b2 = g[2 * e + 1];
            g[2 * e] = fmaf(a, cs[e].x, b2 * cs[e].y);
            g[2 * e + 1] = fmaf(b2, cs[e].x, -a * cs[e].y);
          }
        }
        if (turn_b) {
#pragma unroll
          for (int e = 0; e < P; ++e) {
            const float2 c2 = cs[NCH * P + e];
            const float a = g[VEC + 2 * e], b2 = g[VEC + 2 * e + 1];
            g[VEC + 2 * e] = fmaf(a, c2.x, b2 * c2.y);
            g[VEC + 2 * e + 1] = fmaf(b2, c2.x, -a * c2.y);
          }
        }
      } else if (turn_a) {
#pragma unroll
        for (int e = 0; e < VEC; ++e) {
          const float a = g[e], b2 = g[VEC + e];
          g[e] = fmaf(a, cs[e].x, b2 * cs[e].y);
          g[VEC + e] = fmaf(b2, cs[e].x, -a * cs[e].y);
        }
      }
      if (sd.norm.on) {  // (uniform)
        float sum = 0.f;
#pragma unroll
        for (int e = 0; e < 2 * VEC; ++e) sum = fmaf(x[e], x[e], sum);
        const float s = norm_scale<T, D>(sum, sd.norm.eps);
#pragma unroll
        for (int e = 0; e < 2 * VEC; ++e) x[e] *= s;
        if (has_dw && mine) {
#pragma unroll
          for (int e = 0; e < VEC; ++e) {
            dwa[e] = fmaf(g[e], x[e], dwa[e]);
            dwb[e] = fmaf(g[VEC + e], x[VEC + e], dwb[e]);
          }
        }
        if (sd.norm.w) {
#pragma unroll
          for (int e = 0; e < 2 * VEC; ++e) g[e] *= sd.norm.offset + f[e];
        }
        float dot = 0.f;
#pragma unroll
        for (int e = 0; e < 2 * VEC; ++e) dot = fmaf(g[e], x[e], dot);
        dot = sum_lanes<NCH>(dot) * inv_d;
#pragma unroll
        for (int e = 0; e < 2 * VEC; ++e) g[e] = s * fmaf(-x[e], dot, g[e]);
      }
      if (mine) {
        T* p = const_cast<T*>(row_of(sd.dx, step));
        st16_any(p + lo, Store<T>::pack(g));
        st16_any(p + hi, Store<T>::pack(g + VEC));
      }
      if (has_dw && own_w) join(s_dw[w] + step * D);
    }
  }
  if (!has_dw) return;
  float* part = args.part + sd.part0;
  if (!own_w) join(s_dw[w]);
  __syncthreads();
  for (int j = t; j < (own_w ? nh : 1) * D; j += 256) {
    const int64_t group = (int64_t)layer * sd.w_heads + (own_w ? h0 + j / D : 0);
    part[(group * sd.parts + (own_w ? tc : b)) * D + j % D] = (s_dw[0][j] + s_dw[1][j]) + (s_dw[2][j] + s_dw[3][j]);
  }
}

// dw [group][D] = sum of the group's partials, in their order: 16 columns a block, the
// partials shared by 16 lanes a column.
__global__ void __launch_bounds__(256) norm_weight_sum_kernel(NormGradArgs args, int D, int64_t group0,
                                                              int64_t groups_q) {
  __shared__ float s_sum[16][17];
  const int64_t at = group0 + blockIdx.y;
  const int bs = at < groups_q ? 0 : 1;
  const int64_t group = at - (bs ? groups_q : 0);
  const NormSide& sd = args.side[bs];
  const int col = threadIdx.x & 15, r = threadIdx.x >> 4, j = blockIdx.x * 16 + col;
  const float* p = args.part + sd.part0 + group * sd.parts * D + j;
  float sum = 0.f;
#pragma unroll 8
  for (int i = r; i < sd.parts; i += 16) sum += p[(int64_t)i * D];
  s_sum[r][col] = sum;
  __syncthreads();
  if (r) return;
  sum = 0.f;
#pragma unroll
  for (int i = 0; i < 16; ++i) sum += s_sum[i][col];
  sd.dw[group * D + j] = sum;
}

namespace {

int check(hipError_t e) { return e == hipSuccess ? 0 : (int)e; }

template <int MODE, bool PAGED>
void launch_rows(int dtype, int D, bool pairs, dim3 grid, const Where<MODE>& where, const RopeRows& rows,
                 const CacheView& cv, int layer0, const RopeArgs& ra, const float2* tab, const NormArgs<true>& norm,
                 hipStream_t s) {
#define RR(T, DD, PR)                                                                                              \
  hipLaunchKernelGGL((norm_rope_kernel<T, DD, PR, MODE, PAGED>), grid, dim3(256), 0, s, where, rows, cv, layer0, ra, \
                     tab, norm)
#define RRP(T, DD) { if (pairs) RR(T, DD, true); else RR(T, DD, false); }
  if (dtype == 0) { if (D == 64) RRP(float, 64) else RRP(float, 128) }
  else { if (D == 64) RRP(bf16_t, 64) else RRP(bf16_t, 128) }
#undef RRP
#undef RR
}

}  // namespace

int launch_norm_rope(int dtype, int D, bool pairs, const RopeRows& rows, const int32_t* pos, const RopeArgs& ra,
                     const NormArgs<true>& norm, hipStream_t s) {
  const int H = rows.Hq + rows.Hk;
  const dim3 grid((rows.n_tok + rows.tb - 1) / rows.tb, (rows.tb * H + rows.slice_rows - 1) / rows.slice_rows,
                  rows.grid_layers);
  launch_rows<kApply, false>(dtype, D, pairs, grid, Where<kApply>{pos}, rows, CacheView{}, 0, ra, nullptr, norm, s);
  return check(hipGetLastError());
}

int launch_append_norm(int dtype, bool pairs, const RopeRows& rows, const AppendArgs& args, int n_runs,
                       const AppendGroup* groups, int n_groups, const CacheView& cv, int layer0, const RopeArgs& ra,
                       const float2* tab, const NormArgs<true>& norm, hipStream_t s) {
  const int H = rows.Hq + rows.Hk + rows.Hv;
  const dim3 grid(n_groups, (rows.tb * H + rows.slice_rows - 1) / rows.slice_rows, rows.grid_layers);
#define AP(PG)                                                                                                       \
  {                                                                                                                  \
    if (groups)                                                                                                      \
      launch_rows<kAppendList, PG>(dtype, cv.head_dim, pairs, grid, Where<kAppendList>{groups}, rows, cv, layer0, ra, \
                                   tab, norm, s);                                                                    \
    else                                                                                                             \
      launch_rows<kAppendArgs, PG>(dtype, cv.head_dim, pairs, grid, Where<kAppendArgs>{args, n_runs}, rows, cv,      \
                                   layer0, ra, tab, norm, s);                                                        \
  }
  if (cv.page_size) AP(true) else AP(false)
#undef AP
  return check(hipGetLastError());
}

int launch_norm_rope_grad(int dtype, int D, bool pairs, const NormGradArgs& args, const RopeArgs& ra, hipStream_t s) {
  const NormSide &q = args.side[0], &k = args.side[1];
  const dim3 grid(q.head_blocks * q.spread + k.head_blocks * k.spread, args.n_layers);
#define GK(T, DD, PR) hipLaunchKernelGGL((norm_rope_grad_kernel<T, DD, PR>), grid, dim3(256), 0, s, args, ra)
#define GKP(T, DD) { if (pairs) GK(T, DD, true); else GK(T, DD, false); }
  if (args.n_tok) {
    if (dtype == 0) { if (D == 64) GKP(float, 64) else GKP(float, 128) }
    else { if (D == 64) GKP(bf16_t, 64) else GKP(bf16_t, 128) }
    if (int rc = check(hipGetLastError())) return rc;
  }
#undef GKP
#undef GK
  const int64_t gq = q.dw ? (int64_t)args.n_layers * q.w_heads : 0, gk = k.dw ? (int64_t)args.n_layers * k.w_heads : 0;
  constexpr int64_t kGridY = 65535;
  for (int64_t g0 = 0; g0 < gq + gk; g0 += kGridY) {
    const int n = (int)(gq + gk - g0 < kGridY ? gq + gk - g0 : kGridY);
    hipLaunchKernelGGL(norm_weight_sum_kernel, dim3(D / 16, n), dim3(256), 0, s, args, D, g0, gq);
    if (int rc = check(hipGetLastError())) return rc;
  }
  return 0;
}

}  // namespace fcg

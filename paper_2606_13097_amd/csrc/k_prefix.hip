// Attention of a batch over one shared prefix on gfx950 matrix cores: query rows
// of several sequences meet each key tile of the prefix together, so the prefix
// is read once for all of them, and each sequence's rows then meet its own keys.
//
// An item (one block per kv head) attends up to 128 query rows (fp32: 64) over
// prefix positions [a0, a1) and positions [b0, b1) of one sequence, the latter up
// to each row's own position; what several items leave for a row is merged by
// prefix_merge_kernel (log-sum-exp).  Rows are sorted by (sequence, position),
// row = rank * g + query head of the group, whatever their sequences: the
// prefix part needs no more.
//
// Blocks have four waves.  Wide items: wave w owns rows 32 w .. 32 w + 31, and
// the waves share 64-key tiles (two in LDS, the next one in flight).  Narrow
// items (at most 16 rows: a decode step's own keys): the waves take 16-key tiles
// in turn, each through an LDS ring of its own, without barriers, and merge at
// the end.  In both, S^T = K Q^T and O^T += V^T P^T: lane l holds scores and
// output of query row l % 16, the probabilities pass from accumulator to operand
// without leaving their lane, and the online softmax (base 2) exchanges only
// maxima between the four lanes of a row.  Rows of keys arrive by LDS DMA, whole
// rows, chunks XOR-swizzled against bank conflicts.
//
// Tiles start on multiples of their length in position, so the 16 keys that one
// wave brings in lie on one page, whose entry is one scalar load.  Keys of a tile
// outside the range re-read a key inside it and are masked; a position that is not
// attended is never read.
#include "fcg_device.hpp"
#include "kernels.hpp"

namespace fcg {

namespace {

typedef __bf16 px_bf16x8 __attribute__((ext_vector_type(8)));
typedef short px_i16x4 __attribute__((ext_vector_type(4)));
typedef float px_f32x4 __attribute__((ext_vector_type(4)));
typedef __bf16 px_bf16x2 __attribute__((ext_vector_type(2)));
typedef float px_f32x2 __attribute__((ext_vector_type(2)));

__device__ __forceinline__ px_f32x4 mma32(const uint4& a, const uint4& b, const px_f32x4& c) {
  return __builtin_amdgcn_mfma_f32_16x16x32_bf16(__builtin_bit_cast(px_bf16x8, a), __builtin_bit_cast(px_bf16x8, b), c,
                                                 0, 0, 0);
}
__device__ __forceinline__ px_f32x4 mma16(const uint2& a, const uint2& b, const px_f32x4& c) {
  return __builtin_amdgcn_mfma_f32_16x16x16bf16_1k(__builtin_bit_cast(px_i16x4, a), __builtin_bit_cast(px_i16x4, b), c,
                                                   0, 0, 0);
}
// two fp32 -> packed bf16, round to nearest even
__device__ __forceinline__ uint32_t px_cvt(float lo, float hi) {
  return __builtin_bit_cast(uint32_t, __builtin_convertvector((px_f32x2){lo, hi}, px_bf16x2));
}

// One range of keys: positions [lo, hi) of a sequence (hi > lo).
struct Keys {
  int seq, lo, hi;
};

// Where the 16 keys from position p0 (a multiple of 16) of a sequence lie.
// Positions are clamped into [lo, hi) by the caller, so the page is mapped.
template <typename T, int D, bool PAGED>
struct Rows16 {
  const T *k, *v;  // row of position p0
};
template <typename T, int D, bool PAGED>
__device__ __forceinline__ Rows16<T, D, PAGED> rows16(const CacheView& cv, int layer, int seq, int hk, int p0) {
  const T* ck = reinterpret_cast<const T*>(cv.k);
  const T* cvv = reinterpret_cast<const T*>(cv.v);
  Rows16<T, D, PAGED> r;
  if (!PAGED) {
    const int64_t off = kv_offset<false>(cv, layer, seq, hk, p0);
    r.k = ck + off;
    r.v = cvv + off;
    return r;
  }
  typedef const __attribute__((address_space(4))) int32_t* cptr;  // wave-uniform: through the scalar cache
  const cptr row = (cptr)(uintptr_t)(cv.page_table + (int64_t)seq * 2 * cv.n_lp);
  const int page = row[p0 >> 4];
  const int64_t off = (int64_t)layer * cv.layer_stride + ((int64_t)page * cv.n_kv_heads + hk) * 16 * D;
  r.k = ck + off;
  r.v = cvv + off;
  if (cv.v_alias) {
    const int a = row[cv.n_lp + (p0 >> 4)];
    if (a >= 0)
      r.v = reinterpret_cast<const T*>(cv.lib_v) + (((int64_t)layer * cv.n_kv_heads + hk) * cv.lib_cap + a) * D;
  }
  return r;
}

__device__ __forceinline__ const char* row_ptr(const RowView& v, int64_t esize, int tok, int head) {
  return reinterpret_cast<const char*>(v.p) + ((int64_t)tok * v.token + (int64_t)head * v.head) * esize;
}

constexpr float kLn2 = 0.6931471805599453f;

// Masked keys of a tile have probability 0, but 0 * V is NaN where V is infinite
// or NaN, and one matrix operand serves rows that see the key and rows that do
// not.  So tiles with masked keys enter the product with such elements replaced by
// zeros (*bad: there were some), and the rows that see them get them afterwards:
// a positive weight times an infinity or NaN is that value itself.
__device__ __forceinline__ uint32_t finite2(uint32_t x, bool* bad) {
  const bool hi = (x & 0x7F800000u) == 0x7F800000u, lo = (x & 0x7F80u) == 0x7F80u;
  *bad = *bad || hi || lo;
  return x & (hi ? 0x0000FFFFu : 0xFFFFFFFFu) & (lo ? 0xFFFF0000u : 0xFFFFFFFFu);
}
__device__ __forceinline__ float not_finite(float x) { return fabsf(x) < INFINITY ? 0.f : x; }

}  // namespace

// ------------------------------------------------------------------ bf16

template <int D, bool PAGED>
__global__ void __launch_bounds__(256, 2) prefix_attend_kernel(PrefixCall pc, CacheView cv) {
  constexpr int KS = D / 32;        // 32-deep steps over the head dimension
  constexpr int DT = D / 16;        // 16-wide output tiles
  constexpr int NC = D / 8;         // 16-byte chunks of a row
  constexpr int RI = 64 / NC;       // rows of one DMA instruction
  constexpr int KI = 16 / RI;       // instructions for 16 rows
  constexpr int HALF_T = kPfxTile * D;  // elements of a tile's keys (values)
  __shared__ __align__(16) bf16_t s_kv[2][2 * HALF_T];
  __shared__ float s_wm[4][16], s_wl[4][16];

  const PrefixItem it = pc.items[blockIdx.x];
  const int hk = blockIdx.y;
  const int t = threadIdx.x, lane = t & 63, lr = lane & 15, lq = lane >> 4;
  const int w = __builtin_amdgcn_readfirstlane(t >> 6);
  const int Hkv = cv.n_kv_heads;
  const int g = pc.g;
  const float qscale = 1.4426950408889634f / sqrtf((float)D);

  // lane offsets (bytes) of the DMA instructions for 16 rows, interior tiles
  auto k_off = [&](int j, int r) __attribute__((always_inline)) -> uint32_t {
    const int rr = j * RI + lane / NC;
    return (uint32_t)(r * D + ((lane % NC) ^ (rr % NC)) * 8) * 2;
  };
  auto v_off = [&](int j, int r) __attribute__((always_inline)) -> uint32_t {
    const int rr = j * RI + lane / NC;
    return (uint32_t)(r * D + ((lane % NC) ^ (2 * (rr % (NC / 2)))) * 8) * 2;
  };
  // 16 keys from position p0 of range ks into LDS, keys at lk, values at lv
  auto issue16 = [&](const Keys& ks, int p0, uint32_t lk, uint32_t lv) __attribute__((always_inline)) {
    // a group of 16 with no key inside the range re-reads the nearest one
    const int q0 = min(max(p0, ks.lo & ~15), (ks.hi - 1) & ~15);
    const Rows16<bf16_t, D, PAGED> b = rows16<bf16_t, D, PAGED>(cv, pc.layer, ks.seq, hk, q0);
    const int rlo = max(ks.lo - q0, 0), rhi = min(ks.hi - 1 - q0, 15);
    const void *bk = uniform_ptr(b.k), *bv = uniform_ptr(b.v);
#pragma unroll
    for (int j = 0; j < KI; ++j) dma16s(bk, k_off(j, min(max(j * RI + lane / NC, rlo), rhi)), lk + j * 1024);
#pragma unroll
    for (int j = 0; j < KI; ++j) dma16s(bv, v_off(j, min(max(j * RI + lane / NC, rlo), rhi)), lv + j * 1024);
  };
  constexpr int DPT = 2 * KI;  // DMA instructions of one issue16

  // the two ranges, tiles of `len` keys starting on multiples of len
  const Keys ka{pc.prefix_seq, it.a0, it.a1}, kb{it.seq, it.b0, it.b1};
  auto tiles_of = [&](const Keys& ks, int len) { return ks.hi > ks.lo ? (ks.hi - 1) / len - ks.lo / len + 1 : 0; };

  // this lane's query row `r` of the item
  auto load_q = [&](int r, uint4* qf, int* rpos, int* rtok, int* rhead) __attribute__((always_inline)) {
    const int row = it.row0 + (r < it.n_row ? r : 0);
    const PrefixRank m = pc.ranks[row / g];
    *rpos = m.pos;
    *rtok = m.tok;
    *rhead = hk * g + row % g;
    const char* src = row_ptr(pc.q, 2, m.tok, *rhead);
#pragma unroll
    for (int ks = 0; ks < KS; ++ks) qf[ks] = ld16_any(src + (ks * 32 + lq * 8) * 2);
  };

  // write a row's result: the output, or the slot's partial
  auto emit8 = [&](int r, int rtok, int rhead, int dim, float x0, float x1, float x2, float x3, float m,
                   float l) __attribute__((always_inline)) {
    if (pc.direct) {
      const float inv = l == 0.f ? 0.f : 1.f / l;
      const uint2 y = make_uint2(px_cvt(x0 * inv, x1 * inv), px_cvt(x2 * inv, x3 * inv));
      char* dst = const_cast<char*>(row_ptr(pc.out, 2, rtok, rhead)) + dim * 2;
      __builtin_memcpy(dst, &y, 8);
      if (dim == 0 && pc.lse)
        pc.lse[(int64_t)rtok * (Hkv * g) + rhead] = l == 0.f ? -INFINITY : (m + log2f(l)) * kLn2;
    } else {
      // partial outputs in bf16: the merge weights them in fp32, and its result is bf16
      const int64_t pr = ((int64_t)it.slot * Hkv + hk) * pc.rows + it.row0 + r;
      st8_nt(reinterpret_cast<bf16_t*>(pc.part_o) + pr * D + dim, px_cvt(x0, x1), px_cvt(x2, x3));
      if (dim == 0) {
        pc.part_ml[pr * 2 + 0] = m;
        pc.part_ml[pr * 2 + 1] = l;
      }
    }
  };

  if (it.n_row > 16) {
    // ---------------------------------------------------------------- wide
    constexpr int RT = 2;
    const int na = tiles_of(ka, kPfxTile), nb = tiles_of(kb, kPfxTile), nt = na + nb;
    // tile ti: its range and first position
    auto issue = [&](int ti) __attribute__((always_inline)) {
      const bool own = ti >= na;
      const Keys ks = own ? kb : ka;
      const int p0 = (ks.lo / kPfxTile + (own ? ti - na : ti)) * kPfxTile + 16 * w;
      bf16_t* buf = s_kv[ti & 1];
      issue16(ks, p0, lds_addr(buf) + w * (16 * D * 2), lds_addr(buf + HALF_T) + w * (16 * D * 2));
    };
    if (nt) issue(0);
    uint4 qf[RT][KS];
    int rpos[RT], rtok[RT], rhead[RT];
#pragma unroll
    for (int rt = 0; rt < RT; ++rt)
      load_q(16 * (RT * w + rt) + lr, qf[rt], &rpos[rt], &rtok[rt], &rhead[rt]);
    float mrow[RT], lsum[RT];
    px_f32x4 acc[RT][DT];
#pragma unroll
    for (int rt = 0; rt < RT; ++rt) {
      mrow[rt] = -INFINITY;
      lsum[rt] = 0.f;
#pragma unroll
      for (int dt = 0; dt < DT; ++dt) acc[rt][dt] = px_f32x4{0.f, 0.f, 0.f, 0.f};
    }
    const bool busy = 16 * RT * w < it.n_row;  // some row of this wave
    // the compiler cannot see the tile loads: its wait for these must not fall into the loop
#pragma unroll
    for (int rt = 0; rt < RT; ++rt) {
#pragma unroll
      for (int s = 0; s < KS; ++s) asm volatile("" ::"v"(__builtin_bit_cast(u32x4_t, qf[rt][s])));
      asm volatile("" ::"v"(rpos[rt]), "v"(rtok[rt]));
    }
#pragma unroll 1
    for (int ti = 0; ti < nt; ++ti) {
      wait_vm<0>();   // this wave's loads of the tile have landed ...
      lds_barrier();  // ... and every wave's; every wave is done with the tile before
      if (ti + 1 < nt) issue(ti + 1);
      if (!busy) continue;
      const bool own = ti >= na;
      const Keys ks = own ? kb : ka;
      const int p0 = (ks.lo / kPfxTile + (own ? ti - na : ti)) * kPfxTile;
      const bf16_t* K = s_kv[ti & 1];
      const bf16_t* V = K + HALF_T;
      px_f32x4 st[RT][4];
#pragma unroll
      for (int kt = 0; kt < 4; ++kt) {
        uint4 kf[KS];
#pragma unroll
        for (int s = 0; s < KS; ++s) kf[s] = ld16(&K[((kt * 16 + lr) * NC + ((s * 4 + lq) ^ (lr % NC))) * 8]);
#pragma unroll
        for (int rt = 0; rt < RT; ++rt) {
          px_f32x4 c = {0.f, 0.f, 0.f, 0.f};
#pragma unroll
          for (int s = 0; s < KS; ++s) c = mma32(kf[s], qf[rt][s], c);
          st[rt][kt] = c;
        }
      }
      const bool edge = own || p0 < ks.lo || p0 + kPfxTile > ks.hi;  // masked keys: block-uniform
      if (edge) {
#pragma unroll
        for (int rt = 0; rt < RT; ++rt) {
          // key p0 + 16 kt + 4 lq + e is visible iff lo <= 16 kt + e <= hi
          const int lo = ks.lo - p0 - 4 * lq;
          const int hi = (own ? min(rpos[rt], ks.hi - 1) : ks.hi - 1) - p0 - 4 * lq;
#pragma unroll
          for (int kt = 0; kt < 4; ++kt)
#pragma unroll
            for (int e = 0; e < 4; ++e)
              st[rt][kt][e] = 16 * kt + e >= lo && 16 * kt + e <= hi ? st[rt][kt][e] : -INFINITY;
        }
      }
      uint4 pb[RT][2];
#pragma unroll
      for (int rt = 0; rt < RT; ++rt) {
        float tmax = -INFINITY;
#pragma unroll
        for (int kt = 0; kt < 4; ++kt)
#pragma unroll
          for (int e = 0; e < 4; ++e) tmax = fmaxf(tmax, st[rt][kt][e]);
        tmax = max_rows4(tmax) * qscale;
        // the reference moves only when a row's max grows by more than 2^8: the
        // probabilities stay below 2^8, harmless in fp32 and bf16
        if (__builtin_amdgcn_ballot_w64(tmax > mrow[rt] + 8.f)) {
          const float mnew = fmaxf(mrow[rt], tmax);
          const float alpha = mrow[rt] == -INFINITY ? 0.f : __builtin_amdgcn_exp2f(mrow[rt] - mnew);
          mrow[rt] = mnew;
          lsum[rt] *= alpha;
#pragma unroll
          for (int dt = 0; dt < DT; ++dt) acc[rt][dt] *= alpha;
        }
        const float mref = mrow[rt] == -INFINITY ? 0.f : mrow[rt];
        float pv[4][4], ps = 0.f;
#pragma unroll
        for (int kt = 0; kt < 4; ++kt)
#pragma unroll
          for (int e = 0; e < 4; ++e) {
            pv[kt][e] = __builtin_amdgcn_exp2f(fmaf(st[rt][kt][e], qscale, -mref));
            ps += pv[kt][e];
          }
        lsum[rt] += ps;
#pragma unroll
        for (int s = 0; s < 2; ++s)
          pb[rt][s] = make_uint4(px_cvt(pv[2 * s][0], pv[2 * s][1]), px_cvt(pv[2 * s][2], pv[2 * s][3]),
                                 px_cvt(pv[2 * s + 1][0], pv[2 * s + 1][1]), px_cvt(pv[2 * s + 1][2], pv[2 * s + 1][3]));
      }
      // fragment i = 2 dt + s: lane (lr, lq) needs V[32 s + 4 lq + e][16 dt + lr] and the
      // same 16 keys later; in the transpose read lane lr addresses row 4 lq + lr / 4
      const int vr = 4 * lq + (lr >> 2), vsw = 2 * (vr % (NC / 2));
      auto vfrag = [&](int i) __attribute__((always_inline)) -> uint4 {
        const int vc = (2 * (i >> 1) + ((lr & 3) >> 1)) ^ vsw;
        const bf16_t* row = &V[((32 * (i & 1) + vr) * NC + vc) * 8 + (lr & 1) * 4];
        const uint2 lo = ld_tr8(row), hi = ld_tr8(row + 16 * D);
        return make_uint4(lo.x, lo.y, hi.x, hi.y);
      };
      if (!edge) {
        uint4 va = vfrag(0);
#pragma unroll
        for (int i = 0; i < 2 * DT; ++i) {
          const uint4 vn = i + 1 < 2 * DT ? vfrag(i + 1) : va;
#pragma unroll
          for (int rt = 0; rt < RT; ++rt) acc[rt][i >> 1] = mma32(va, pb[rt][i & 1], acc[rt][i >> 1]);
          va = vn;
        }
      } else {
        bool bad = false;
#pragma unroll
        for (int i = 0; i < 2 * DT; ++i) {
          uint4 va = vfrag(i);
          va = make_uint4(finite2(va.x, &bad), finite2(va.y, &bad), finite2(va.z, &bad), finite2(va.w, &bad));
#pragma unroll
          for (int rt = 0; rt < RT; ++rt) acc[rt][i >> 1] = mma32(va, pb[rt][i & 1], acc[rt][i >> 1]);
        }
        if (__builtin_amdgcn_ballot_w64(bad)) {
#pragma unroll 1
          for (int p = max(p0, ks.lo); p < min(p0 + kPfxTile, ks.hi); ++p) {
            const int kk = p - p0, sw = 2 * (kk % (NC / 2));
#pragma unroll
            for (int dt = 0; dt < DT; ++dt) {
              const uint2 x = *reinterpret_cast<const uint2*>(&V[(kk * NC + ((2 * dt + (lq >> 1)) ^ sw)) * 8 + (lq & 1) * 4]);
              const float v[4] = {lo_bf16(x.x), hi_bf16(x.x), lo_bf16(x.y), hi_bf16(x.y)};
#pragma unroll
              for (int rt = 0; rt < RT; ++rt)
#pragma unroll
                for (int e = 0; e < 4; ++e) acc[rt][dt][e] += !own || p <= rpos[rt] ? not_finite(v[e]) : 0.f;
            }
          }
        }
      }
    }
#pragma unroll
    for (int rt = 0; rt < RT; ++rt) {
      const float l = sum_rows4(lsum[rt]);
      const int r = 16 * (RT * w + rt) + lr;
      if (r >= it.n_row) continue;
#pragma unroll
      for (int dt = 0; dt < DT; ++dt)
        emit8(r, rtok[rt], rhead[rt], dt * 16 + lq * 4, acc[rt][dt][0], acc[rt][dt][1], acc[rt][dt][2], acc[rt][dt][3],
              mrow[rt], l);
    }
    return;
  }

  // ------------------------------------------------------------------ narrow
  constexpr int TILE = 16 * D * 2 * 2;  // bytes of a 16-key tile: keys, then values
  static_assert(4 * 2 * TILE == sizeof(s_kv), "a ring of two per wave");
  char* ring = reinterpret_cast<char*>(s_kv) + w * 2 * TILE;
  const uint32_t ring_lds = lds_addr(ring);
  const int na = tiles_of(ka, 16), nb = tiles_of(kb, 16);
  const int n = (na + nb - w + 3) >> 2;  // this wave's tiles: w, w + 4, ...
  auto issue = [&](int i) __attribute__((always_inline)) {
    const int ti = w + 4 * i;
    const bool own = ti >= na;
    const Keys ks = own ? kb : ka;
    const int p0 = ((ks.lo >> 4) + (own ? ti - na : ti)) * 16;
    issue16(ks, p0, ring_lds + (i & 1) * TILE, ring_lds + (i & 1) * TILE + 16 * D * 2);
  };
  if (n > 0) issue(0);
  uint4 qf[KS];
  int rpos, rtok, rhead;
  load_q(lr, qf, &rpos, &rtok, &rhead);
  float mref = -INFINITY, lsum = 0.f;
  px_f32x4 acc[DT];
#pragma unroll
  for (int dt = 0; dt < DT; ++dt) acc[dt] = px_f32x4{0.f, 0.f, 0.f, 0.f};
#pragma unroll
  for (int s = 0; s < KS; ++s) asm volatile("" ::"v"(__builtin_bit_cast(u32x4_t, qf[s])));  // landed before the next tile
#pragma unroll 1
  for (int i = 0; i < n; ++i) {
    if (i + 1 < n) {
      wait_lds();  // the reads of the buffer's tile before have returned
      issue(i + 1);
      wait_vm<DPT>();
    } else {
      wait_vm<0>();
    }
    const int ti = w + 4 * i;
    const bool own = ti >= na;
    const Keys ks = own ? kb : ka;
    const int p0 = ((ks.lo >> 4) + (own ? ti - na : ti)) * 16;
    const bf16_t* K = reinterpret_cast<const bf16_t*>(ring + (i & 1) * TILE);
    uint4 kf[KS];
#pragma unroll
    for (int s = 0; s < KS; ++s) kf[s] = ld16(&K[(lr * NC + ((s * 4 + lq) ^ (lr % NC))) * 8]);
    uint2 va[DT];
    const int vr = 4 * lq + (lr >> 2), vsw = 2 * (vr % (NC / 2));
#pragma unroll
    for (int dt = 0; dt < DT; ++dt)
      va[dt] = ld_tr8(&K[16 * D + (vr * NC + ((2 * dt + ((lr & 3) >> 1)) ^ vsw)) * 8 + (lr & 1) * 4]);
    px_f32x4 sc = {0.f, 0.f, 0.f, 0.f};
#pragma unroll
    for (int s = 0; s < KS; ++s) sc = mma32(kf[s], qf[s], sc);
    const int lo = ks.lo - p0 - 4 * lq, hi = (own ? min(rpos, ks.hi - 1) : ks.hi - 1) - p0 - 4 * lq;
    float x[4], lmax = -INFINITY;
#pragma unroll
    for (int e = 0; e < 4; ++e) {
      x[e] = e >= lo && e <= hi ? sc[e] * qscale : -INFINITY;
      lmax = fmaxf(lmax, x[e]);
    }
    if (__builtin_amdgcn_ballot_w64(lmax > mref + 8.f)) {
      const float mn = max_rows4(fmaxf(mref, lmax));
      const float f = mref == -INFINITY ? 0.f : __builtin_amdgcn_exp2f(mref - mn);
      lsum *= f;
#pragma unroll
      for (int dt = 0; dt < DT; ++dt) acc[dt] *= f;
      mref = mn;
    }
    const float mr = mref == -INFINITY ? 0.f : mref;
    float p[4];
#pragma unroll
    for (int e = 0; e < 4; ++e) {
      p[e] = __builtin_amdgcn_exp2f(x[e] - mr);
      lsum += p[e];
    }
    const uint2 pb = make_uint2(px_cvt(p[0], p[1]), px_cvt(p[2], p[3]));
    const bool edge = (own && it.n_row > g) || p0 < ks.lo || p0 + 16 > ks.hi;  // masked keys: wave-uniform
    bool bad = false;
    if (edge) {
#pragma unroll
      for (int dt = 0; dt < DT; ++dt) va[dt] = make_uint2(finite2(va[dt].x, &bad), finite2(va[dt].y, &bad));
    }
#pragma unroll
    for (int dt = 0; dt < DT; ++dt) acc[dt] = mma16(va[dt], pb, acc[dt]);
    if (edge && __builtin_amdgcn_ballot_w64(bad)) {
#pragma unroll 1
      for (int q = max(p0, ks.lo); q < min(p0 + 16, ks.hi); ++q) {
        const int kk = q - p0, sw = 2 * (kk % (NC / 2));
#pragma unroll
        for (int dt = 0; dt < DT; ++dt) {
          const uint2 y = *reinterpret_cast<const uint2*>(
              &K[16 * D + (kk * NC + ((2 * dt + (lq >> 1)) ^ sw)) * 8 + (lq & 1) * 4]);
          const float v[4] = {lo_bf16(y.x), hi_bf16(y.x), lo_bf16(y.y), hi_bf16(y.y)};
#pragma unroll
          for (int e = 0; e < 4; ++e) acc[dt][e] += !own || q <= rpos ? not_finite(v[e]) : 0.f;
        }
      }
    }
  }
  // the four waves meet in LDS, each wave's outputs in its own ring
  lsum = sum_rows4(lsum);
  wait_lds();
  static_assert(16 * D * 4 <= 2 * TILE, "a wave's outputs fit its ring");
  {
    float* o = reinterpret_cast<float*>(ring);
#pragma unroll
    for (int dt = 0; dt < DT; ++dt)
      *reinterpret_cast<float4*>(&o[lr * D + dt * 16 + 4 * lq]) =
          make_float4(acc[dt][0], acc[dt][1], acc[dt][2], acc[dt][3]);
    if (lq == 0) {
      s_wm[w][lr] = mref;
      s_wl[w][lr] = lsum;
    }
  }
  __syncthreads();
  for (int idx = t; idx < it.n_row * D / 4; idx += 256) {
    const int r = idx / (D / 4), d = 4 * (idx % (D / 4));
    float M = -INFINITY;
#pragma unroll
    for (int k = 0; k < 4; ++k) M = fmaxf(M, s_wm[k][r]);
    float L = 0.f;
    float4 a = make_float4(0.f, 0.f, 0.f, 0.f);
#pragma unroll
    for (int k = 0; k < 4; ++k) {
      const float m = s_wm[k][r];
      const float f = m == -INFINITY ? 0.f : __builtin_amdgcn_exp2f(m - M);
      const float4 o = *reinterpret_cast<const float4*>(reinterpret_cast<char*>(s_kv) + k * 2 * TILE + (r * D + d) * 4);
      L = fmaf(s_wl[k][r], f, L);
      a.x = fmaf(o.x, f, a.x);
      a.y = fmaf(o.y, f, a.y);
      a.z = fmaf(o.z, f, a.z);
      a.w = fmaf(o.w, f, a.w);
    }
    const int row = it.row0 + r;
    emit8(r, pc.ranks[row / g].tok, hk * g + row % g, d, a.x, a.y, a.z, a.w, M, L);
  }
}

// ------------------------------------------------------------------ fp32

// The same items on fp32 caches with v_mfma_f32_16x16x4_f32 (exact products,
// fp32 sums).  One 64-key tile in LDS; wide items: 16 rows per wave and all 64
// keys; narrow items: the same 16 rows in every wave, 16 of the keys each, merged
// at the end.  The four k indices of a matrix step are dims 16 c + 4 lq + e of
// keys and queries alike, so both are read 16 bytes at a time.
template <int D, bool PAGED>
__global__ void __launch_bounds__(256) prefix_attend_f32_kernel(PrefixCall pc, CacheView cv) {
  constexpr int DT = D / 16;
  constexpr int NC = D / 4;         // 16-byte chunks of a row
  constexpr int RI = 64 / NC;       // rows of one DMA instruction
  constexpr int KI = 16 / RI;
  constexpr int HALF_T = kPfxTile * D;
  __shared__ __align__(16) float s_kv[2 * HALF_T];
  __shared__ float s_wm[4][16], s_wl[4][16];

  const PrefixItem it = pc.items[blockIdx.x];
  const int hk = blockIdx.y;
  const int t = threadIdx.x, lane = t & 63, lr = lane & 15, lq = lane >> 4;
  const int w = __builtin_amdgcn_readfirstlane(t >> 6);
  const int Hkv = cv.n_kv_heads;
  const int g = pc.g;
  const float qscale = 1.4426950408889634f / sqrtf((float)D);
  const bool narrow = it.n_row <= 16;
  const Keys ka{pc.prefix_seq, it.a0, it.a1}, kb{it.seq, it.b0, it.b1};
  auto tiles_of = [&](const Keys& ks) {
    return ks.hi > ks.lo ? (ks.hi - 1) / kPfxTile - ks.lo / kPfxTile + 1 : 0;
  };
  const int na = tiles_of(ka), nt = na + tiles_of(kb);
  float* K = s_kv;
  float* V = s_kv + HALF_T;

  const int r = (narrow ? 0 : 16 * w) + lr;
  const int row = it.row0 + (r < it.n_row ? r : 0);
  const PrefixRank m = pc.ranks[row / g];
  const int rhead = hk * g + row % g;
  px_f32x4 qf[DT];
  {
    const char* src = row_ptr(pc.q, 4, m.tok, rhead);
#pragma unroll
    for (int c = 0; c < DT; ++c) qf[c] = __builtin_bit_cast(px_f32x4, ld16_any(src + (16 * c + 4 * lq) * 4));
  }
  float mref = -INFINITY, lsum = 0.f;
  px_f32x4 acc[DT];
#pragma unroll
  for (int dt = 0; dt < DT; ++dt) acc[dt] = px_f32x4{0.f, 0.f, 0.f, 0.f};
  const bool busy = narrow || 16 * w < it.n_row;
  const int kt0 = narrow ? w : 0, kt1 = narrow ? w + 1 : 4;
#pragma unroll 1
  for (int ti = 0; ti < nt; ++ti) {
    const bool own = ti >= na;
    const Keys ks = own ? kb : ka;
    const int p0 = (ks.lo / kPfxTile + (own ? ti - na : ti)) * kPfxTile;
    {
      const int q0 = min(max(p0 + 16 * w, ks.lo & ~15), (ks.hi - 1) & ~15);
      const Rows16<float, D, PAGED> b = rows16<float, D, PAGED>(cv, pc.layer, ks.seq, hk, q0);
      const int rlo = max(ks.lo - q0, 0), rhi = min(ks.hi - 1 - q0, 15);
      const void *bk = uniform_ptr(b.k), *bv = uniform_ptr(b.v);
#pragma unroll
      for (int j = 0; j < KI; ++j) {
        const int rr = j * RI + lane / NC;
        const uint32_t off = (uint32_t)(min(max(rr, rlo), rhi) * D + ((lane % NC) ^ rr) * 4) * 4;
        dma16s(bk, off, lds_addr(K) + (w * 16 * D) * 4 + j * 1024);
        dma16s(bv, off, lds_addr(V) + (w * 16 * D) * 4 + j * 1024);
      }
    }
    wait_vm<0>();
    __syncthreads();
    if (busy) {
      for (int kt = kt0; kt < kt1; ++kt) {
        px_f32x4 sc = {0.f, 0.f, 0.f, 0.f};
#pragma unroll
        for (int c = 0; c < DT; ++c) {
          const px_f32x4 kf =
              *reinterpret_cast<const px_f32x4*>(&K[((kt * 16 + lr) * NC + ((4 * c + lq) ^ lr)) * 4]);
#pragma unroll
          for (int e = 0; e < 4; ++e) sc = __builtin_amdgcn_mfma_f32_16x16x4f32(kf[e], qf[c][e], sc, 0, 0, 0);
        }
        const int base = p0 + 16 * kt;
        const int lo = ks.lo - base - 4 * lq, hi = (own ? min(m.pos, ks.hi - 1) : ks.hi - 1) - base - 4 * lq;
        float x[4], lmax = -INFINITY;
#pragma unroll
        for (int e = 0; e < 4; ++e) {
          x[e] = e >= lo && e <= hi ? sc[e] * qscale : -INFINITY;
          lmax = fmaxf(lmax, x[e]);
        }
        if (__builtin_amdgcn_ballot_w64(lmax > mref)) {
          const float mn = max_rows4(fmaxf(mref, lmax));
          const float f = mref == -INFINITY ? 0.f : __builtin_amdgcn_exp2f(mref - mn);
          lsum *= f;
#pragma unroll
          for (int dt = 0; dt < DT; ++dt) acc[dt] *= f;
          mref = mn;
        }
        const float mr = mref == -INFINITY ? 0.f : mref;
        float p[4];
#pragma unroll
        for (int e = 0; e < 4; ++e) {
          p[e] = __builtin_amdgcn_exp2f(x[e] - mr);
          lsum += p[e];
        }
        const bool edge = own || base < ks.lo || base + 16 > ks.hi;  // masked keys: wave-uniform
        bool bad = false;
#pragma unroll
        for (int dt = 0; dt < DT; ++dt)
#pragma unroll
          for (int e = 0; e < 4; ++e) {
            const int key = 4 * lq + e;
            float v = V[((kt * 16 + key) * NC + ((4 * dt + (lr >> 2)) ^ key)) * 4 + (lr & 3)];
            if (edge) {
              bad = bad || !(fabsf(v) < INFINITY);
              v = fabsf(v) < INFINITY ? v : 0.f;
            }
            acc[dt] = __builtin_amdgcn_mfma_f32_16x16x4f32(v, p[e], acc[dt], 0, 0, 0);
          }
        if (edge && __builtin_amdgcn_ballot_w64(bad)) {
#pragma unroll 1
          for (int q = max(base, ks.lo); q < min(base + 16, ks.hi); ++q) {
            const int key = q - base;
#pragma unroll
            for (int dt = 0; dt < DT; ++dt) {
              const px_f32x4 v =
                  *reinterpret_cast<const px_f32x4*>(&V[((kt * 16 + key) * NC + ((4 * dt + lq) ^ key)) * 4]);
#pragma unroll
              for (int e = 0; e < 4; ++e) acc[dt][e] += !own || q <= m.pos ? not_finite(v[e]) : 0.f;
            }
          }
        }
      }
    }
    __syncthreads();  // the tile's reads are done before the next one lands
  }
  lsum = sum_rows4(lsum);
  auto emit = [&](int rr, int rtok, int head, int dim, float4 a, float M, float L) __attribute__((always_inline)) {
    if (pc.direct) {
      const float inv = L == 0.f ? 0.f : 1.f / L;
      const float4 y = make_float4(a.x * inv, a.y * inv, a.z * inv, a.w * inv);
      __builtin_memcpy(const_cast<char*>(row_ptr(pc.out, 4, rtok, head)) + dim * 4, &y, 16);
      if (dim == 0 && pc.lse) pc.lse[(int64_t)rtok * (Hkv * g) + head] = L == 0.f ? -INFINITY : (M + log2f(L)) * kLn2;
    } else {
      const int64_t pr = ((int64_t)it.slot * Hkv + hk) * pc.rows + it.row0 + rr;
      *reinterpret_cast<float4*>(reinterpret_cast<float*>(pc.part_o) + pr * D + dim) = a;
      if (dim == 0) {
        pc.part_ml[pr * 2 + 0] = M;
        pc.part_ml[pr * 2 + 1] = L;
      }
    }
  };
  if (!narrow) {
    if (r >= it.n_row) return;
#pragma unroll
    for (int dt = 0; dt < DT; ++dt)
      emit(r, m.tok, rhead, dt * 16 + 4 * lq, make_float4(acc[dt][0], acc[dt][1], acc[dt][2], acc[dt][3]), mref, lsum);
    return;
  }
  static_assert(4 * 16 * D <= 2 * HALF_T, "the waves' outputs fit the tile");
#pragma unroll
  for (int dt = 0; dt < DT; ++dt)
    *reinterpret_cast<px_f32x4*>(&s_kv[(w * 16 + lr) * D + dt * 16 + 4 * lq]) = acc[dt];
  if (lq == 0) {
    s_wm[w][lr] = mref;
    s_wl[w][lr] = lsum;
  }
  __syncthreads();
  for (int idx = t; idx < it.n_row * D / 4; idx += 256) {
    const int rr = idx / (D / 4), d = 4 * (idx % (D / 4));
    float M = -INFINITY;
#pragma unroll
    for (int k = 0; k < 4; ++k) M = fmaxf(M, s_wm[k][rr]);
    float L = 0.f;
    float4 a = make_float4(0.f, 0.f, 0.f, 0.f);
#pragma unroll
    for (int k = 0; k < 4; ++k) {
      const float mk = s_wm[k][rr];
      const float f = mk == -INFINITY ? 0.f : __builtin_amdgcn_exp2f(mk - M);
      const float4 o = *reinterpret_cast<const float4*>(&s_kv[(k * 16 + rr) * D + d]);
      L = fmaf(s_wl[k][rr], f, L);
      a.x = fmaf(o.x, f, a.x);
      a.y = fmaf(o.y, f, a.y);
      a.z = fmaf(o.z, f, a.z);
      a.w = fmaf(o.w, f, a.w);
    }
    const int row2 = it.row0 + rr;
    emit(rr, pc.ranks[row2 / g].tok, hk * g + row2 % g, d, a, M, L);
  }
}

// ------------------------------------------------------------------ merge

// out = sum_s O_s 2^(M_s - M) / sum_s L_s 2^(M_s - M), M = max_s M_s, over the slots
// of a row; 16 bytes of output per lane.  Grid (rank, kv heads' rows / rows a block).
template <typename T, int D>
__global__ void __launch_bounds__(256) prefix_merge_kernel(PrefixCall pc, CacheView cv) {
  constexpr int VEC = Store<T>::VEC;
  constexpr int LPR = D / VEC;  // lanes of a row
  const int Hkv = cv.n_kv_heads, g = pc.g, Hq = Hkv * g;
  const PrefixRank m = pc.ranks[blockIdx.x];
  const int head = blockIdx.y * (256 / LPR) + threadIdx.x / LPR, c = threadIdx.x % LPR;
  if (head >= Hq) return;
  const int hk = head / g;
  const int64_t row = (int64_t)hk * pc.rows + (int64_t)blockIdx.x * g + head % g;
  const int64_t step = (int64_t)Hkv * pc.rows;  // rows from a slot to the next
  const T* po = reinterpret_cast<const T*>(pc.part_o);
  float M = -INFINITY, L = 0.f, acc[VEC];
#pragma unroll
  for (int e = 0; e < VEC; ++e) acc[e] = 0.f;
  constexpr int PF = 4;
  const int n = m.na + m.nb;
  for (int i0 = 0; i0 < n; i0 += PF) {
    uint4 x[PF];
    float2 ml[PF];
#pragma unroll
    for (int p = 0; p < PF; ++p) {
      const int i = min(i0 + p, n - 1);
      const int64_t pr = (int64_t)(i < m.na ? i : m.b0 + i - m.na) * step + row;
      x[p] = ld16(po + pr * D + c * VEC);
      ml[p] = *reinterpret_cast<const float2*>(pc.part_ml + pr * 2);
      if (i0 + p >= n) ml[p] = make_float2(-INFINITY, 0.f);
    }
    float mn = M;
#pragma unroll
    for (int p = 0; p < PF; ++p) mn = fmaxf(mn, ml[p].x);
    const float mr = mn == -INFINITY ? 0.f : mn;
    const float f = __builtin_amdgcn_exp2f(M - mr);
    L *= f;
#pragma unroll
    for (int e = 0; e < VEC; ++e) acc[e] *= f;
#pragma unroll
    for (int p = 0; p < PF; ++p) {
      const float wgt = ml[p].x == -INFINITY ? 0.f : __builtin_amdgcn_exp2f(ml[p].x - mr);
      float y[VEC];
      Store<T>::unpack(x[p], y);
      L = fmaf(ml[p].y, wgt, L);
      if (wgt != 0.f) {
#pragma unroll
        for (int e = 0; e < VEC; ++e) acc[e] = fmaf(y[e], wgt, acc[e]);
      }
    }
    M = mn;
  }
  const float inv = L == 0.f ? 0.f : 1.f / L;
#pragma unroll
  for (int e = 0; e < VEC; ++e) acc[e] *= inv;
  st16_any(const_cast<char*>(row_ptr(pc.out, sizeof(T), m.tok, head)) + c * 16, Store<T>::pack(acc));
  if (c == 0 && pc.lse) pc.lse[(int64_t)m.tok * Hq + head] = L == 0.f ? -INFINITY : (M + log2f(L)) * kLn2;
}

static int check(hipError_t e) { return e == hipSuccess ? 0 : (int)e; }

int launch_prefix_attend(int dtype, const PrefixCall& call, const CacheView& cv, hipStream_t s) {
  if (call.n_items == 0) return 0;
  const dim3 grid(call.n_items, cv.n_kv_heads);
#define PA(KERNEL, DD, PG) hipLaunchKernelGGL((KERNEL<DD, PG>), grid, dim3(256), 0, s, call, cv)
#define PAD(KERNEL, PG) { if (cv.head_dim == 64) PA(KERNEL, 64, PG); else PA(KERNEL, 128, PG); }
#define PAP(KERNEL) { if (cv.page_size) PAD(KERNEL, true) else PAD(KERNEL, false) }
  if (dtype == 0) PAP(prefix_attend_f32_kernel) else PAP(prefix_attend_kernel)
#undef PAP
#undef PAD
#undef PA
  return check(hipGetLastError());
}

int launch_prefix_merge(int dtype, const PrefixCall& call, const CacheView& cv, hipStream_t s) {
  if (call.n_rank == 0) return 0;
  const int lanes = cv.head_dim * (dtype == 0 ? 4 : 2) / 16, per = 256 / lanes;
  const dim3 grid(call.n_rank, (cv.n_kv_heads * call.g + per - 1) / per);
#define PM(T, DD) hipLaunchKernelGGL((prefix_merge_kernel<T, DD>), grid, dim3(256), 0, s, call, cv)
  if (dtype == 0) { if (cv.head_dim == 64) PM(float, 64); else PM(float, 128); }
  else { if (cv.head_dim == 64) PM(bf16_t, 64); else PM(bf16_t, 128); }
#undef PM
  return check(hipGetLastError());
}

}  // namespace fcg

// Attention of a batch over one shared prefix on gfx950 matrix cores: query rows
// of several sequences meet each key tile of the prefix together, so the prefix
// is read once for all of them, and each sequence's rows then meet its own keys.
//
// An item (one block per kv head) attends up to 128 or 256 query rows (fp32: 64)
// over prefix positions [a0, a1) and positions [b0, b1) of one sequence, the latter
// up to each row's own position; what several items leave for a row is merged by
// prefix_merge_kernel (log-sum-exp).  Rows are sorted by (sequence, position),
// row = rank * g + query head of the group, whatever their sequences: the
// prefix part needs no more.
//
//   o = sum_j 2^(s_j - m) v_j / sum_j 2^(s_j - m),  s_j = q k_j log2(e) / sqrt(D),
//
// in one pass over the keys, m and both sums fp32.  The probabilities enter the second
// product rounded to bf16: the matrix instruction takes both operands in one type, fp16
// does not hold the values' range, and a second product with what the rounding leaves
// would add half to the matrix work of the calls that it bounds.  That rounding is as
// large as the result's own, so a result is 1.4 times as far from the definition as
// one rounded once (2.3e-3 of its norm against 1.7e-3).  S^T = K Q^T and O^T += V^T P^T: a lane holds scores and
// outputs of one query row, the probabilities pass from accumulator to operand
// without leaving their lane, and only maxima and final sums cross lanes.  Rows of
// keys arrive by LDS DMA, whole rows, chunks XOR-swizzled against bank conflicts.
//
// Wide items (more than 32 rows): wave w owns rows 32 w .. 32 w + 31 on 32x32x16
// products, two lanes a row, and the waves share 64-key tiles.  Blocks of four waves
// hold two tiles and run two to a compute unit; blocks of eight hold four tiles, and
// their halves run half a tile apart, one multiplying while the other takes the
// softmax.  On 32x32 products, because a wave's vector instructions beside another
// wave's products took 7.1 cycles each there and 9.1 beside 16x16 ones.
// Narrow items (a decode step's own keys): the waves take 16-key tiles in turn
// (16x16 products, four lanes a row), each through an LDS ring of its own, without
// barriers, and merge at the end; two such items may share a block, half of its waves
// each.
//
// What bounds it (bf16, D 128, 8 key heads; times per call, one after the other):
//   32 sequences of 64 tokens, 4 query heads a key head, over 6007 shared keys and up
//   to 300 own ones: 198 to 214 us for 207 GFLOP, 1.0 PFLOP/s, where an 8192^3 library
//   product reaches 1.18.  A tile takes 3170 cycles of its compute unit, 2048 of them
//   matrix cycles; the rest is the softmax that finds no gap between the products.
//   32 sequences of 4 tokens, 8 query heads, over 22011: 116 to 123 us for 94 GFLOP.  Four
//   row blocks of a head cut in 8 splits each are one round of 256 items; their first
//   tiles, the partials and the merge (7 us) are what is added to the product rate.
//   64 sequences of one token, 4 query heads, over 4321: 21.8 us for 57 MB.  Round
//   trips: page entries, first tiles, partials, merge (4 us).
//
// Tiles start on multiples of their length in position, so the 16 keys that one
// wave brings in lie on one page.  Keys of a tile outside the range re-read a key
// inside it and are masked; a position that is not attended is never read.
#include <type_traits>

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
typedef float px_f32x16 __attribute__((ext_vector_type(16)));
__device__ __forceinline__ px_f32x16 mma_wide(const uint4& a, const uint4& b, const px_f32x16& c) {
  return __builtin_amdgcn_mfma_f32_32x32x16_bf16(__builtin_bit_cast(px_bf16x8, a), __builtin_bit_cast(px_bf16x8, b), c,
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

__device__ __forceinline__ int tiles_of(const Keys& ks, int len) {
  return ks.hi > ks.lo ? (ks.hi - 1) / len - ks.lo / len + 1 : 0;
}

// The 16 positions from q0 (a multiple of 16) of a sequence: its page and the
// library token its values are read from, wave-uniform, through the scalar cache.
struct Entry {
  int32_t page, alias;
};
template <bool PAGED>
__device__ __forceinline__ Entry entry_of(const CacheView& cv, int seq, int pos) {
  Entry e{0, -1};
  if (PAGED) {
    typedef const __attribute__((address_space(4))) int32_t* cptr;
    const cptr row = (cptr)(uintptr_t)(cv.page_table + (int64_t)seq * 2 * cv.n_lp);
    e.page = row[pos >> 4];
    if (cv.v_alias) e.alias = row[cv.n_lp + (pos >> 4)];
  }
  return e;
}
// Page entries of a wave's tiles, 64 tiles at a time in the lanes of two registers: one
// round trip for all of them (an entry read beside the tiles was a miss in its way:
// each sequence's pages are their own, and scalar loads are waited for with the LDS
// reads).  at(i, lane_seq, lane_pos): sequence and position of tile i.
template <bool PAGED>
struct Entries {
  int32_t page, alias;
  int batch = -1;
  template <typename F>
  __device__ __forceinline__ Entry get(const CacheView& cv, int i, int n, int lane, F&& at) {
    if (!PAGED) return Entry{0, -1};
    if (i >> 6 != batch) {  // wave-uniform
      batch = i >> 6;
      int seq, pos;
      at(min(batch * 64 + lane, n - 1), &seq, &pos);
      const int32_t* row = cv.page_table + (int64_t)seq * 2 * cv.n_lp + (pos >> 4);
      page = row[0];
      alias = cv.v_alias ? row[cv.n_lp] : -1;
    }
    return Entry{__builtin_amdgcn_readlane(page, i & 63), __builtin_amdgcn_readlane(alias, i & 63)};
  }
};

// Rows of one kv head of the layer: of position q0 (paged: a multiple of 16, its page
// given), wave-uniform.
template <typename T, int D, bool PAGED>
struct HeadRows {
  const T *k, *v, *lib;  // the layer's and head's first row
  int64_t step;          // paged: elements from a page to the next; else from a sequence to the next
  __device__ __forceinline__ HeadRows(const CacheView& cv, int layer, int hk) {
    const int64_t at = (int64_t)layer * cv.layer_stride + (int64_t)hk * (PAGED ? 16 : cv.max_tokens) * D;
    step = (int64_t)cv.n_kv_heads * (PAGED ? 16 : cv.max_tokens) * D;
    k = reinterpret_cast<const T*>(cv.k) + at;
    v = reinterpret_cast<const T*>(cv.v) + at;
    lib = reinterpret_cast<const T*>(cv.lib_v) + ((int64_t)layer * cv.n_kv_heads + hk) * cv.lib_cap * D;
  }
  __device__ __forceinline__ const T* keys(int seq, int q0, const Entry& e) const {
    return (const T*)uniform_ptr(k + (PAGED ? e.page * step : seq * step + (int64_t)q0 * D));
  }
  __device__ __forceinline__ const T* values(int seq, int q0, const Entry& e) const {
    const T* p = v + (PAGED ? e.page * step : seq * step + (int64_t)q0 * D);
    if (PAGED && e.alias >= 0) p = lib + (int64_t)e.alias * D;
    return (const T*)uniform_ptr(p);
  }
};

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
__device__ __forceinline__ float finite_abs(float x) { return fabsf(x) < INFINITY ? fabsf(x) : 0.f; }

// over lanes l and l ^ 32
__device__ __forceinline__ float max_halves(float v) {
  const auto b = __builtin_amdgcn_permlane32_swap(__float_as_uint(v), __float_as_uint(v), false, false);
  return fmaxf(__uint_as_float(b[0]), __uint_as_float(b[1]));
}
__device__ __forceinline__ float sum_halves(float v) {
  const auto b = __builtin_amdgcn_permlane32_swap(__float_as_uint(v), __float_as_uint(v), false, false);
  return __uint_as_float(b[0]) + __uint_as_float(b[1]);
}

// max over each group of N lanes (16 or 32)
template <int N>
__device__ __forceinline__ float max_lanes(float v) {
  if (N == 32) return max_lanes32(v);
  v = fmaxf(v, dpp_f32<kDppXor1>(v));
  v = fmaxf(v, dpp_f32<kDppXor2>(v));
  v = fmaxf(v, dpp_f32<kDppHalfMirror>(v));
  return fmaxf(v, dpp_f32<kDppMirror>(v));
}

// Where a row's result goes: the output, or the slot's partial.  bf16 caches keep
// partial outputs in fp16, scaled per row by the power of two 2^up that brings the
// row's largest to 2^14 .. 2^15 (so eleven significant bits in two bytes; bf16 ones
// would be a third rounding of the size of the result's own, 2.8e-3 off the definition
// instead of 2.3e-3, and fp32 ones move twice the bytes); max, sum and up are
// fp32.  fp32 caches keep fp32 partials, up = 0.
typedef _Float16 px_f16x2 __attribute__((ext_vector_type(2)));
typedef _Float16 px_f16x8 __attribute__((ext_vector_type(8)));
template <typename T, int D>
struct Emit {
  char* dst;
  float* aux;  // lse, or the partial's (max, sum, up, -)
  float scale, a0, a1, a2;
  bool direct;
  __device__ __forceinline__ Emit(const PrefixCall& pc, const PrefixItem& it, int hk, int Hkv, int r, int tok, int head,
                                  float m, float l, float top) {
    direct = pc.direct;
    if (direct) {
      scale = l == 0.f ? 0.f : 1.f / l;
      dst = const_cast<char*>(row_ptr(pc.out, sizeof(T), tok, head));
      a0 = l == 0.f ? -INFINITY : (m + log2f(l)) * kLn2;
      aux = pc.lse ? pc.lse + (int64_t)tok * (Hkv * pc.g) + head : nullptr;
    } else {
      const int up = sizeof(T) == 2 && top > 0.f ? max(-126, min(126, 15 - __builtin_amdgcn_frexp_expf(top))) : 0;
      scale = __builtin_ldexpf(1.f, up);
      const int64_t pr = ((int64_t)it.slot * Hkv + hk) * pc.rows + it.row0 + r;
      dst = reinterpret_cast<char*>(pc.part_o) + pr * (D * (int)sizeof(T));
      aux = pc.part_ml + pr * 4;
      a0 = m;
      a1 = l;
      a2 = (float)up;
    }
  }
  __device__ __forceinline__ void put_aux() const {
    if (!direct) *reinterpret_cast<float4*>(aux) = make_float4(a0, a1, a2, 0.f);
    else if (aux) *aux = a0;
  }
  // four outputs as they are stored (two-byte kinds)
  __device__ __forceinline__ uint2 pack(float x0, float x1, float x2, float x3) const {
    if (direct) return make_uint2(px_cvt(x0 * scale, x1 * scale), px_cvt(x2 * scale, x3 * scale));
    const px_f16x2 a = __builtin_convertvector((px_f32x2){x0 * scale, x1 * scale}, px_f16x2);
    const px_f16x2 b = __builtin_convertvector((px_f32x2){x2 * scale, x3 * scale}, px_f16x2);
    return make_uint2(__builtin_bit_cast(uint32_t, a), __builtin_bit_cast(uint32_t, b));
  }
  __device__ __forceinline__ void put8(int dim, const uint4& y) const {
    if (dim == 0) put_aux();
    st16_any(dst + dim * 2, y);
  }
  __device__ __forceinline__ void put(int dim, float x0, float x1, float x2, float x3) const {
    if (dim == 0) put_aux();
    if (sizeof(T) == 4) {
      const float4 y = make_float4(x0 * scale, x1 * scale, x2 * scale, x3 * scale);
      __builtin_memcpy(dst + dim * 4, &y, 16);
    } else {
      const uint2 y = pack(x0, x1, x2, x3);
      __builtin_memcpy(dst + dim * 2, &y, 8);
    }
  }
};

// The plan of a call: in device memory, or by value.
template <bool VALUE>
struct Plan {};
template <>
struct Plan<false> {
  const PrefixItem* items;
  const PrefixRank* ranks;
  __device__ __forceinline__ bool paired(int) const { return false; }
  __device__ __forceinline__ PrefixItem item(int b, int) const { return items[b]; }
  __device__ __forceinline__ PrefixRank rank(int r) const { return ranks[r]; }
};
template <>
struct Plan<true> {
  PrefixArgs a;
  // block b holds two own items, one of them for each half of its waves
  __device__ __forceinline__ bool paired(int b) const { return a.paired && b >= a.n_pre; }
  // half: of the block's waves, if paired (an item without rows where there is none left)
  __device__ __forceinline__ PrefixItem item(int b, int half) const {
    PrefixItem it{};
    if (b < a.n_pre) {
      const int rb = b / a.pre_slots, s = b - rb * a.pre_slots;
      it.row0 = rb * a.block;
      it.n_row = min(a.block, a.pre_rows - it.row0);
      it.a0 = s * a.per;
      it.a1 = min(a.prefix_len, it.a0 + a.per);
      it.slot = s;
      return it;
    }
    // the group is the last one whose first item is at most b: one group per lane
    static_assert(kPfxGroups == 64, "one group per lane");
    const int lane = threadIdx.x & 63, x = a.paired ? 2 * (b - a.n_pre) + half : b - a.n_pre;
    if (half && x >= a.paired) return it;
    const PrefixGroup mine = a.group[min(lane, a.n_group - 1)];
    const uint64_t below = __builtin_amdgcn_ballot_w64(lane < a.n_group && mine.item0 <= x);
    const int r = 63 - __builtin_clzll(below);
    const int rows = __builtin_amdgcn_readlane(mine.rows, r), end = __builtin_amdgcn_readlane(mine.end, r);
    it.seq = __builtin_amdgcn_readlane(mine.seq, r);
    const int s = x - __builtin_amdgcn_readlane(mine.item0, r);
    it.row0 = rows & 0xFFFF;
    it.n_row = rows >> 16;
    const int cut = a.prefix_len / kPfxTile * kPfxTile + s * a.per;  // splits are cut at multiples of a tile
    it.b0 = max(a.prefix_len, cut);
    it.b1 = min(end, cut + a.per);
    it.slot = a.pre_slots + s;
    return it;
  }
  __device__ __forceinline__ PrefixRank rank(int r) const {
    const PrefixSmall m = a.rank[r];
    return PrefixRank{m.tok, m.pos, (uint16_t)a.pre_slots, (uint16_t)a.pre_slots, m.nb, 0};
  }
};

}  // namespace

// ------------------------------------------------------------------ bf16

// WAVES 4: 128 query rows, two tiles in LDS, two blocks per compute unit.  WAVES
// 8: 256 rows, four tiles, one block.  VALUE: the plan comes by value.
template <int D, bool PAGED, int WAVES, bool VALUE>
__global__ void __launch_bounds__(WAVES * 64, WAVES == 4 ? 2 : 1) prefix_attend_kernel(PrefixCall pc, Plan<VALUE> plan,
                                                                                       CacheView cv) {
  constexpr int NT = WAVES * 64;
  constexpr int NB = WAVES == 4 ? 2 : 4;  // tiles in LDS
  constexpr int KS = D / 32;              // 32-deep steps over the head dimension
  constexpr int DT = D / 16;              // 16-wide output tiles
  constexpr int NC = D / 8;               // 16-byte chunks of a row
  constexpr int RI = 64 / NC;             // rows of one DMA instruction
  constexpr int KI = 16 / RI;             // instructions for 16 rows
  constexpr int HALF_T = kPfxTile * D;    // elements of a tile's keys (values)
  __shared__ __align__(16) bf16_t s_kv[NB][2 * HALF_T];
  __shared__ float s_wm[WAVES][32], s_wl[WAVES][32];
  __shared__ __align__(16) int s_bad[NB][4];  // a tile's value groups that held non-finite elements

  PrefixItem it = plan.item(blockIdx.y, 0);
  const int hk = blockIdx.x;  // fastest: workgroups go to the eight XCDs in turn, so a head's blocks share an L2
  const int t = threadIdx.x, lane = t & 63, lr = lane & 15, lq = lane >> 4;
  const int w = __builtin_amdgcn_readfirstlane(t >> 6);
  const int Hkv = cv.n_kv_heads;
  const int g = pc.g;
  const float qscale = 1.4426950408889634f / sqrtf((float)D);
  const Keys ka{pc.prefix_seq, it.a0, it.a1};
  Keys kb{it.seq, it.b0, it.b1};

  // DMA instruction j of 16 rows fills rows RI j .. RI j + RI - 1: lane l the chunk
  // position l % NC of row RI j + l / NC.  The chunk that belongs there is the position
  // XOR the row's swizzle (keys: row % NC; values: 2 (row % (NC / 2))), so the lane's byte
  // offset in the 16 rows is the same for every group of 16.
  uint32_t koff[KI], voff[KI];
#pragma unroll
  for (int j = 0; j < KI; ++j) {
    const int r = j * RI + lane / NC;
    koff[j] = (uint32_t)(r * D + ((lane % NC) ^ (r % NC)) * 8) * 2;
    voff[j] = (uint32_t)(r * D + ((lane % NC) ^ (2 * (r % (NC / 2)))) * 8) * 2;
  }
  // 16 rows from position q0 of range ks into LDS, instruction j of KI; rows outside the
  // range re-read one inside it
  auto issue_one = [&](const Keys& ks, int q0, const void* base, uint32_t lds, const uint32_t* off, int j)
                       __attribute__((always_inline)) {
    if (q0 >= ks.lo && q0 + 16 <= ks.hi) {  // wave-uniform
      dma16s(base, off[j], lds + j * 1024);
    } else {
      const int rlo = max(ks.lo - q0, 0), rhi = min(ks.hi - 1 - q0, 15), r = j * RI + lane / NC;
      dma16s(base, off[j] + (uint32_t)((min(max(r, rlo), rhi) - r) * (D * 2)), lds + j * 1024);
    }
  };
  auto issue16 = [&](const Keys& ks, int q0, const void* base, uint32_t lds, const uint32_t* off)
                     __attribute__((always_inline)) {
#pragma unroll
    for (int j = 0; j < KI; ++j) issue_one(ks, q0, base, lds, off, j);
  };
  const HeadRows<bf16_t, D, PAGED> head(cv, pc.layer, hk);
  // a group of 16 positions with none inside the range stands for the nearest one that has
  auto group_of = [&](const Keys& ks, int p0) __attribute__((always_inline)) {
    return min(max(p0, ks.lo & ~15), (ks.hi - 1) & ~15);
  };
  // non-finite elements of 16 value rows in LDS to zeros; true if there were some
  auto clean16 = [&](bf16_t* v) __attribute__((always_inline)) -> bool {
    bool bad = false;
#pragma unroll
    for (int j = 0; j < KI; ++j) {
      uint4* p = reinterpret_cast<uint4*>(v) + j * 64 + lane;
      uint4 x = *p;
      bool b = false;
      x = make_uint4(finite2(x.x, &b), finite2(x.y, &b), finite2(x.z, &b), finite2(x.w, &b));
      if (b) *p = x;
      bad = bad || b;
    }
    return __builtin_amdgcn_ballot_w64(bad) != 0;
  };

  if (it.n_row > 32) {
    // ---------------------------------------------------------------- wide
    constexpr int KS = D / 16;           // 16-deep steps over the head dimension
    constexpr int DT = D / 32;           // 32-wide output tiles
    const int lc = lane & 31, lh = lane >> 5;
    constexpr int DPT = 8 * KI / WAVES;  // DMA instructions of this wave for a tile
    const int ta0 = ka.lo / kPfxTile, tb0 = kb.lo / kPfxTile;
    const int na = tiles_of(ka, kPfxTile), nt = na + tiles_of(kb, kPfxTile);
    const int grp = w & 3;               // the 16 keys this wave brings in
    auto first_of = [&](int ti) __attribute__((always_inline)) {
      return (ti >= na ? tb0 + ti - na : ta0 + ti) * kPfxTile;
    };
    // this lane's query row, column lc of the 32-row matrix operands (rows past the item's
    // repeat its first one and are not written)
    const int r = 32 * w + lc;
    const int row = it.row0 + (r < it.n_row ? r : 0);
    const PrefixRank m = plan.rank(row / g);
    const int pmin = plan.rank(it.row0 / g).pos;
    Entries<PAGED> entries;
    auto entry = [&](int ti) __attribute__((always_inline)) -> Entry {  // the page of this wave's rows of tile ti
      return entries.get(cv, ti, nt, lane, [&](int i, int* seq, int* pos) __attribute__((always_inline)) {
        const bool own = i >= na;
        *seq = own ? kb.seq : ka.seq;
        const int lo = own ? kb.lo : ka.lo, hi = own ? kb.hi : ka.hi;
        *pos = min(max(first_of(i) + 16 * grp, lo & ~15), (hi - 1) & ~15);
      });
    };
    auto issue = [&](int ti) __attribute__((always_inline)) {
      const Keys ks = ti >= na ? kb : ka;
      const int q0 = group_of(ks, first_of(ti) + 16 * grp);
      bf16_t* buf = s_kv[ti & (NB - 1)];
      const uint32_t lds = lds_addr(buf) + grp * (16 * D * 2);
      const Entry ent = entry(ti);
      if (WAVES == 4 || w < 4) issue16(ks, q0, head.keys(ks.seq, q0, ent), lds, koff);
      if (WAVES == 4 || w >= 4) issue16(ks, q0, head.values(ks.seq, q0, ent), lds + HALF_T * 2, voff);
    };
    if (nt) issue(0);
    const int rpos = m.pos, rhead = hk * g + row % g;
    uint4 qf[KS];
    {
      const char* src = row_ptr(pc.q, 2, m.tok, rhead);
#pragma unroll
      for (int ks = 0; ks < KS; ++ks) qf[ks] = ld16_any(src + (ks * 16 + lh * 8) * 2);
    }
    // the compiler cannot see the tile loads: its wait for these must not fall into the loop
#pragma unroll
    for (int s = 0; s < KS; ++s) asm volatile("" ::"v"(__builtin_bit_cast(u32x4_t, qf[s])));
    asm volatile("" ::"v"(rpos), "v"(m.tok));
    float mrow = -INFINITY, lsum = 0.f;
    px_f32x16 acc[DT];
#pragma unroll
    for (int dt = 0; dt < DT; ++dt)
#pragma unroll
      for (int e = 0; e < 16; ++e) acc[dt][e] = 0.f;
    const bool busy = 32 * w < it.n_row;  // some row of this wave

    px_f32x16 st[2];  // scores of the tile at hand: element 4 q + e of st[kt] is key 32 kt + 8 q + 4 lh + e
    uint4 pb[4];      // its probabilities, bf16: of keys 16 s + 4 lh .. + 3 and 16 s + 8 + 4 lh .. + 3
    // A tile with keys that some row of the block does not see (block-uniform).  Own keys
    // belong to items of one sequence, whose first row has the smallest position.
    auto is_edge = [&](int ti) __attribute__((always_inline)) -> bool {
      const int p0 = first_of(ti);
      return ti >= na ? p0 < kb.lo || p0 + kPfxTile > min(kb.hi, pmin + 1) : p0 < ka.lo || p0 + kPfxTile > ka.hi;
    };
    // key fragment i: keys 32 (i % 2) + lc, dims 16 (i / 2) + 8 lh ..
    auto kfrag = [&](const bf16_t* K, int i) __attribute__((always_inline)) -> uint4 {
      return ld16(&K[((i % 2 * 32 + lc) * NC + ((i / 2 * 2 + lh) ^ (lc % NC))) * 8]);
    };
    // value fragment i, dt = i % DT, s = i / DT: lane (lc, lh) needs V[key][32 dt + lc] of the
    // eight keys of pb[s]; in the transpose read lane lr of a 16-lane group addresses the
    // group's row lr / 4, dims 4 (lr % 4) .. + 3 of its 16
    const int vr = 4 * lh + (lr >> 2), vsw = 2 * (vr % (NC / 2));
    auto vfrag = [&](const bf16_t* V, int i) __attribute__((always_inline)) -> uint4 {
      const int vc = (4 * (i % DT) + 2 * ((lane >> 4) & 1) + ((lr & 3) >> 1)) ^ vsw;
      const bf16_t* row = &V[((16 * (i / DT) + vr) * NC + vc) * 8 + (lr & 1) * 4];
      const uint2 lo2 = ld_tr8(row), hi2 = ld_tr8(row + 8 * D);
      return make_uint4(lo2.x, lo2.y, hi2.x, hi2.y);
    };
    // S^T = K Q^T of one tile and O^T += V^T P^T of another (or one of the two), their
    // fragments read ahead in turn; both take 2 KS = 4 DT fragments
    // Fragments are read AH steps ahead of their products (a step's products take 64 matrix
    // cycles, an LDS read returns after more than that); loaded: the first AH already are.
    constexpr int AH = 3;
    uint4 kf[AH], vf[AH];
    auto products = [&](const bf16_t* K, const bf16_t* V, auto with_k, auto with_v, auto loaded, auto&& beside)
                        __attribute__((always_inline)) {
      constexpr bool KK = decltype(with_k)::value, VV = decltype(with_v)::value;
      static_assert(2 * KS == 4 * DT, "as many fragments of both");
      constexpr int N = 2 * KS;
      if constexpr (!decltype(loaded)::value) {
#pragma unroll
        for (int i = 0; i < AH; ++i) {
          if (KK) kf[i] = kfrag(K, i);
          if (VV) vf[i] = vfrag(V, i);
        }
      }
#pragma unroll
      for (int i = 0; i < N; ++i) {
        const uint4 kc = kf[i % AH], vc = vf[i % AH];
        if constexpr (KK) st[i % 2] = mma_wide(kc, qf[i / 2], i < 2 ? px_f32x16{} : st[i % 2]);
        if constexpr (VV) acc[i % DT] = mma_wide(vc, pb[i / DT], acc[i % DT]);
        if (i + AH < N) {
          if (KK) kf[i % AH] = kfrag(K, i + AH);
          if (VV) vf[i % AH] = vfrag(V, i + AH);
        }
        beside(i);
        // no further ahead: the scheduler hoisted all reads and ran out of registers
        if constexpr (KK && VV) __builtin_amdgcn_sched_barrier(0);
      }
    };
    // mask and softmax of tile ti: scores -> probabilities, running max and sum, outputs rescaled
    auto softmax = [&](int ti, auto masked) __attribute__((always_inline)) {
      if (decltype(masked)::value && is_edge(ti)) {
        const bool own = ti >= na;
        const int lo = own ? kb.lo : ka.lo, hi = own ? kb.hi : ka.hi, p0 = first_of(ti);
        // key p0 + 32 kt + 8 q + 4 lh + e is visible iff a <= 32 kt + 8 q + e <= b
        const int b = (own ? min(rpos, hi - 1) : hi - 1) - p0 - 4 * lh;
#pragma unroll
        for (int kt = 0; kt < 2; ++kt)
#pragma unroll
          for (int i = 0; i < 16; ++i) st[kt][i] = 32 * kt + 8 * (i / 4) + i % 4 <= b ? st[kt][i] : -INFINITY;
        if (p0 < lo) {
          const int a = lo - p0 - 4 * lh;
#pragma unroll
          for (int kt = 0; kt < 2; ++kt)
#pragma unroll
            for (int i = 0; i < 16; ++i) st[kt][i] = 32 * kt + 8 * (i / 4) + i % 4 >= a ? st[kt][i] : -INFINITY;
        }
      }
      float top[4];  // a wave's dependent instructions are what this costs: four chains
#pragma unroll
      for (int c = 0; c < 4; ++c) {
        top[c] = st[c / 2][c % 2 * 8];
#pragma unroll
        for (int i = 1; i < 8; ++i) top[c] = fmaxf(top[c], st[c / 2][c % 2 * 8 + i]);
      }
      const float tmax = max_halves(fmaxf(fmaxf(top[0], top[1]), fmaxf(top[2], top[3]))) * qscale;
      // the reference moves only when a row's max grows by more than 2^8: the
      // probabilities stay below 2^8, harmless in fp32 and bf16
      if (__builtin_amdgcn_ballot_w64(tmax > mrow + 8.f)) {
        const float mnew = fmaxf(mrow, tmax);
        const float alpha = mrow == -INFINITY ? 0.f : __builtin_amdgcn_exp2f(mrow - mnew);
        mrow = mnew;
        lsum *= alpha;
#pragma unroll
        for (int dt = 0; dt < DT; ++dt) acc[dt] *= alpha;
      }
      const float mref = mrow == -INFINITY ? 0.f : mrow;
      float pv[2][16];
#pragma unroll
      for (int kt = 0; kt < 2; ++kt)
#pragma unroll
        for (int i = 0; i < 16; ++i) pv[kt][i] = __builtin_amdgcn_exp2f(fmaf(st[kt][i], qscale, -mref));
      float ps[8];
#pragma unroll
      for (int c = 0; c < 8; ++c)
        ps[c] = (pv[c / 4][c % 4 * 4] + pv[c / 4][c % 4 * 4 + 1]) + (pv[c / 4][c % 4 * 4 + 2] + pv[c / 4][c % 4 * 4 + 3]);
      lsum += ((ps[0] + ps[1]) + (ps[2] + ps[3])) + ((ps[4] + ps[5]) + (ps[6] + ps[7]));
#pragma unroll
      for (int s = 0; s < 4; ++s) {
        const float* p = &pv[s / 2][s % 2 * 8];
        pb[s] = make_uint4(px_cvt(p[0], p[1]), px_cvt(p[2], p[3]), px_cvt(p[4], p[5]), px_cvt(p[6], p[7]));
      }
      // computed here, not where the products want them (past the barrier that ends the half)
      if constexpr (WAVES == 8)
        asm volatile("" ::"v"(__builtin_bit_cast(u32x4_t, pb[0])), "v"(__builtin_bit_cast(u32x4_t, pb[1])),
                     "v"(__builtin_bit_cast(u32x4_t, pb[2])), "v"(__builtin_bit_cast(u32x4_t, pb[3])), "v"(lsum));
    };
    auto cleaned = [&](int ti) __attribute__((always_inline)) -> bool {
      const int* sb = s_bad[ti & (NB - 1)];
      return __builtin_amdgcn_readfirstlane(sb[0] | sb[1] | sb[2] | sb[3]) != 0;
    };
    // values of tile ti that were cleaned out of its buffer, to the rows that see them
    auto restore = [&](int ti) __attribute__((always_inline)) {
      const bool own = ti >= na;
      const int lo = own ? kb.lo : ka.lo, hi = own ? kb.hi : ka.hi, p0 = first_of(ti), seq = own ? kb.seq : ka.seq;
#pragma unroll 1
      for (int p = max(p0, lo); p < min(p0 + kPfxTile, hi); ++p) {
        const bf16_t* row = head.values(seq, p & ~15, entry_of<PAGED>(cv, seq, p)) + (p & 15) * D + lh * 4;
#pragma unroll
        for (int dt = 0; dt < DT; ++dt)
#pragma unroll
          for (int q = 0; q < 4; ++q) {
            const uint2 x = *reinterpret_cast<const uint2*>(row + dt * 32 + q * 8);
            const float v[4] = {lo_bf16(x.x), hi_bf16(x.x), lo_bf16(x.y), hi_bf16(x.y)};
#pragma unroll
            for (int e = 0; e < 4; ++e) acc[dt][4 * q + e] += !own || p <= rpos ? not_finite(v[e]) : 0.f;
          }
      }
    };
    // this wave's value rows of an edge tile, landed: non-finite elements out
    auto clean = [&](int ti) __attribute__((always_inline)) {
      const bool bad = clean16(s_kv[ti & (NB - 1)] + HALF_T + grp * 16 * D);
      if (lane == 0) s_bad[ti & (NB - 1)][grp] = bad;
    };
    using Yes = std::true_type;
    using No = std::false_type;
    auto nothing = [](int) {};

    if constexpr (WAVES == 4) {
      // Two blocks per compute unit: one block's softmax beside the other's products.
      auto step = [&](int ti, auto buf) __attribute__((always_inline)) {
        const bf16_t* K = s_kv[buf];
        wait_vm<0>();  // this wave's loads of the tile have landed ...
        if (is_edge(ti)) clean(ti);
        lds_barrier();  // ... and every wave's; every wave is done with the tile before
        if (ti + 1 < nt) issue(ti + 1);
        if (!busy) return;
        products(K, K, Yes{}, No{}, No{}, nothing);
        softmax(ti, Yes{});
        products(K, K + HALF_T, No{}, Yes{}, No{}, nothing);
        if (is_edge(ti) && cleaned(ti)) restore(ti);
      };
      // unrolled by the ring, so that every LDS address is a constant past a lane's base
      for (int ti = 0; ti < nt; ti += 2) {
        step(ti, std::integral_constant<int, 0>{});
        if (ti + 1 < nt) step(ti + 1, std::integral_constant<int, 1>{});
      }
    } else if (nt) {
      // One block per compute unit, two waves per SIMD, half a tile apart: while waves
      // 0-3 feed the matrix cores (scores of tile t, outputs of tile t - 1), waves 4-7
      // do the softmax of tile t - 1, and the other way round; a barrier after each
      // half.  (In step, both waves of a SIMD wanted the matrix cores at once and then
      // both the vector unit: 37% of the matrix rate.)  Waves 0-3 bring in keys, 4-7
      // values.  Counting halves so that waves 0-3 multiply tile t in half 2 t and waves
      // 4-7 in 2 t + 1: tile u is requested in halves 2 u - 4 (keys) and 2 u - 3 (values),
      // after the last reads of tile u - 4 in its buffer (keys half 2 u - 7, values half
      // 2 u - 5), and has landed by the end of half 2 u - 1, before its first reads in
      // half 2 u.
      const bool late = w >= 4;
      uint32_t off[KI];
#pragma unroll
      for (int j = 0; j < KI; ++j) off[j] = late ? voff[j] : koff[j];
      if (1 < nt) {
        issue(1);
        wait_vm<DPT>();
      } else {
        wait_vm<0>();
      }
      if (late && is_edge(0)) clean(0);
      lds_barrier();
      if (late) lds_barrier();
      // (waves without rows go along on a repeated one: branches around the products
      // cost every wave registers)
      // What a half needs besides its products and its softmax is done in the softmax
      // half before it: a wave's scalar and branch instructions do not overlap its own
      // products.
      const uint32_t lds0 = lds_addr(s_kv[0]) + grp * (16 * D * 2) + (late ? HALF_T * 2 : 0);
      const void* base;    // this wave's rows of the tile to request next
      uint32_t offx[KI];   // and the lane's offsets in them
      bool bad = false;    // values of the tile before were cleaned
      auto request = [&](int ti, const uint32_t* o) {  // tile ti + 2, an instruction at a time between the products
        return [=](int i) __attribute__((always_inline)) {
          constexpr int EVERY = 2 * KS / KI;
          if (i % EVERY == EVERY - 1)
            dma16s(base, o[i / EVERY], lds0 + ((ti + 2) & (NB - 1)) * (2 * HALF_T * 2) + i / EVERY * 1024);
        };
      };
      // the rows of tile t; past the last tile its rows again, into a buffer that nothing reads
      auto prepare = [&](int t0) __attribute__((always_inline)) {
        const int t = min(t0, nt - 1);
        const Keys ks = t >= na ? kb : ka;
        const int q0 = group_of(ks, first_of(t) + 16 * grp);
        const Entry ent = entry(t);
        base = late ? head.values(ks.seq, q0, ent) : head.keys(ks.seq, q0, ent);
        const int rlo = max(ks.lo - q0, 0), rhi = min(ks.hi - 1 - q0, 15);
#pragma unroll
        for (int j = 0; j < KI; ++j) {
          const int rr = j * RI + lane / NC;
          offx[j] = off[j] + (uint32_t)((min(max(rr, rlo), rhi) - rr) * (D * 2));
        }
      };
      // the first fragments of tile t's products: its keys have landed a half ago
      auto preload = [&](int t) __attribute__((always_inline)) {
#pragma unroll
        for (int i = 0; i < AH; ++i) {
          kf[i] = kfrag(s_kv[t & (NB - 1)], i);
          vf[i] = vfrag(s_kv[(t - 1) & (NB - 1)] + HALF_T, i);
        }
      };
      auto half_m = [&](int ti, auto first) __attribute__((always_inline)) {
        const bf16_t* K = s_kv[ti & (NB - 1)];
        __builtin_amdgcn_s_setprio(1);  // the other wave's softmax fills the gaps between products, not the reverse
        if constexpr (decltype(first)::value)
          products(K, K, Yes{}, No{}, No{}, request(ti, offx));
        else
          products(K, s_kv[(ti - 1) & (NB - 1)] + HALF_T, Yes{}, Yes{}, Yes{}, request(ti, offx));
        __builtin_amdgcn_s_setprio(0);
        if (bad) restore(ti - 1);
        wait_vm<DPT>();  // this wave's loads of tile ti + 1
        if (late && ti + 1 < nt && is_edge(ti + 1)) clean(ti + 1);
        lds_barrier();
        __builtin_amdgcn_sched_barrier(0);  // the softmax stays in its half
      };
      auto half_s = [&](int ti) __attribute__((always_inline)) {
        softmax(ti, Yes{});
        prepare(ti + 3);
        preload(ti + 1);
        bad = is_edge(ti) && cleaned(ti);
        __builtin_amdgcn_sched_barrier(0);
        lds_barrier();
      };
      prepare(2);
      half_m(0, Yes{});
      half_s(0);
      int ti = 1;
      // Whole tiles of the prefix, up to the last few: the loop that long prefixes spend
      // their time in, with no mask and the least scalar work.
      const int whole = ka.lo % kPfxTile ? 0 : ka.hi / kPfxTile - ta0;
      if (ti + 3 < whole) {  // (tile 0 is whole too: nothing of it was cleaned)
        const bf16_t* pool = late ? head.v : head.k;
        const bf16_t* lib = late ? head.lib : head.k;
        const bf16_t* row = PAGED ? nullptr : pool + ka.seq * head.step + (int64_t)(ta0 * kPfxTile + 16 * grp) * D;
#pragma unroll 1
        for (; ti + 3 < whole; ++ti) {
          __builtin_amdgcn_s_setprio(1);
          products(s_kv[ti & (NB - 1)], s_kv[(ti - 1) & (NB - 1)] + HALF_T, Yes{}, Yes{}, Yes{}, request(ti, off));
          __builtin_amdgcn_s_setprio(0);
          wait_vm<DPT>();
          lds_barrier();
          __builtin_amdgcn_sched_barrier(0);
          softmax(ti, No{});
          const Entry ent = entry(ti + 3);
          base = uniform_ptr(!PAGED ? row + (int64_t)(ti + 3) * (kPfxTile * D)
                             : late && ent.alias >= 0 ? lib + (int64_t)ent.alias * D : pool + ent.page * head.step);
          preload(ti + 1);
          __builtin_amdgcn_sched_barrier(0);
          lds_barrier();
        }
        prepare(ti + 2);  // (the same rows; offsets for the halves that clamp)
      }
#pragma unroll 1
      for (; ti < nt; ++ti) {
        half_m(ti, No{});
        half_s(ti);
      }
      if (!late) lds_barrier();
      const bf16_t* K = s_kv[(nt - 1) & (NB - 1)];
      products(K, K + HALF_T, No{}, Yes{}, No{}, nothing);
      if (bad) restore(nt - 1);
      wait_vm<0>();  // no load may land in LDS after the block
    }
    const float l = sum_halves(lsum);
    float top = 0.f;
#pragma unroll
    for (int dt = 0; dt < DT; ++dt)
#pragma unroll
      for (int e = 0; e < 16; ++e) top = fmaxf(top, finite_abs(acc[dt][e]));
    const Emit<bf16_t, D> em(pc, it, hk, Hkv, r, m.tok, rhead, mrow, l, max_halves(top));
#pragma unroll
    for (int dt = 0; dt < DT; ++dt)
#pragma unroll
      for (int q = 0; q < 4; q += 2) {
        // lanes l and l + 32 hold dims 8 q + 0 .. 3 and + 4 .. 7 of q and q + 1: exchanged, the
        // first has all of q's eight and the other all of q + 1's
        const uint2 x = em.pack(acc[dt][4 * q], acc[dt][4 * q + 1], acc[dt][4 * q + 2], acc[dt][4 * q + 3]);
        const uint2 y = em.pack(acc[dt][4 * q + 4], acc[dt][4 * q + 5], acc[dt][4 * q + 6], acc[dt][4 * q + 7]);
        const auto s0 = __builtin_amdgcn_permlane32_swap(x.x, y.x, false, false);
        const auto s1 = __builtin_amdgcn_permlane32_swap(x.y, y.y, false, false);
        if (r < it.n_row) em.put8(dt * 32 + (q + lh) * 8, make_uint4(s0[0], s1[0], s0[1], s1[1]));
      }
    return;
  }

  // ------------------------------------------------------------------ narrow
  constexpr int TILE = 16 * D * 2 * 2;  // bytes of a 16-key tile: keys, then values
  constexpr int DPT = 2 * KI;
  static_assert(WAVES * 2 * TILE == sizeof(s_kv) || WAVES == 8, "a ring of two per wave");
  static_assert(WAVES * 2 * TILE <= sizeof(s_kv) && 32 * D * 4 <= 2 * TILE, "rings and results fit");
  char* ring = reinterpret_cast<char*>(s_kv) + w * 2 * TILE;
  // this item's waves: w0 .. w0 + nw - 1
  const int nw = plan.paired(blockIdx.y) ? WAVES / 2 : WAVES, w0 = w & ~(nw - 1), wi = w - w0;
  if (w0) {
    it = plan.item(blockIdx.y, 1);
    kb = Keys{it.seq, it.b0, it.b1};
  }
  auto narrow = [&](auto row_tiles) __attribute__((always_inline)) {
    constexpr int RT = decltype(row_tiles)::value;
    const uint32_t ring_lds = lds_addr(ring);
    const int na = tiles_of(ka, 16), nb = tiles_of(kb, 16);
    const int n = (na + nb - wi + nw - 1) / nw;  // this wave's tiles: wi, wi + nw, ...
    auto first_of = [&](int i) __attribute__((always_inline)) {
      const int ti = wi + nw * i;
      return (ti >= na ? (kb.lo >> 4) + ti - na : (ka.lo >> 4) + ti) * 16;
    };
    auto own_of = [&](int i) __attribute__((always_inline)) { return wi + nw * i >= na; };
    Entries<PAGED> entries;
    auto entry = [&](int i) __attribute__((always_inline)) -> Entry {
      return entries.get(cv, i, n, lane, [&](int j, int* seq, int* pos) __attribute__((always_inline)) {
        *seq = own_of(j) ? kb.seq : ka.seq;
        *pos = first_of(j);
      });
    };
    auto issue = [&](int i) __attribute__((always_inline)) {
      const Keys ks = own_of(i) ? kb : ka;
      const int q0 = first_of(i);
      const Entry ent = entry(i);
      issue16(ks, q0, head.keys(ks.seq, q0, ent), ring_lds + (i & 1) * TILE, koff);
      issue16(ks, q0, head.values(ks.seq, q0, ent), ring_lds + (i & 1) * TILE + 16 * D * 2, voff);
    };
    if (n > 0) issue(0);
    uint4 qf[RT][KS];
    int rpos[RT];
#pragma unroll
    for (int rt = 0; rt < RT; ++rt) {
      const int r = 16 * rt + lr;
      const int row = it.row0 + (r < it.n_row ? r : 0);
      const PrefixRank m = plan.rank(row / g);
      rpos[rt] = m.pos;
      const char* src = row_ptr(pc.q, 2, m.tok, hk * g + row % g);
#pragma unroll
      for (int ks = 0; ks < KS; ++ks) qf[rt][ks] = ld16_any(src + (ks * 32 + lq * 8) * 2);
    }
    float mref[RT], lsum[RT];
    px_f32x4 acc[RT][DT];
#pragma unroll
    for (int rt = 0; rt < RT; ++rt) {
      mref[rt] = -INFINITY;
      lsum[rt] = 0.f;
#pragma unroll
      for (int dt = 0; dt < DT; ++dt) acc[rt][dt] = px_f32x4{0.f, 0.f, 0.f, 0.f};
#pragma unroll
      for (int s = 0; s < KS; ++s) asm volatile("" ::"v"(__builtin_bit_cast(u32x4_t, qf[rt][s])));
      asm volatile("" ::"v"(rpos[rt]));
    }
#pragma unroll 1
    for (int i = 0; i < n; ++i) {
      if (i + 1 < n) {
        wait_lds();  // the reads of the buffer's tile before have returned
        issue(i + 1);
        wait_vm<DPT>();
      } else {
        wait_vm<0>();
      }
      const bool own = own_of(i);
      const int lo = own ? kb.lo : ka.lo, hi = own ? kb.hi : ka.hi;
      const int p0 = first_of(i);
      bf16_t* K = reinterpret_cast<bf16_t*>(ring + (i & 1) * TILE);
      const bool edge = (own && it.n_row > g) || p0 < lo || p0 + 16 > hi;  // masked keys: wave-uniform
      const bool bad = edge && clean16(K + 16 * D);
      uint4 kf[KS];
#pragma unroll
      for (int s = 0; s < KS; ++s) kf[s] = ld16(&K[(lr * NC + ((s * 4 + lq) ^ (lr % NC))) * 8]);
      uint2 va[DT];
      const int vr = 4 * lq + (lr >> 2), vsw = 2 * (vr % (NC / 2));
#pragma unroll
      for (int dt = 0; dt < DT; ++dt)
        va[dt] = ld_tr8(&K[16 * D + (vr * NC + ((2 * dt + ((lr & 3) >> 1)) ^ vsw)) * 8 + (lr & 1) * 4]);
#pragma unroll
      for (int rt = 0; rt < RT; ++rt) {
        px_f32x4 sc = {0.f, 0.f, 0.f, 0.f};
#pragma unroll
        for (int s = 0; s < KS; ++s) sc = mma32(kf[s], qf[rt][s], sc);
        const int a = lo - p0 - 4 * lq, b = (own ? min(rpos[rt], hi - 1) : hi - 1) - p0 - 4 * lq;
        float x[4], lmax = -INFINITY;
#pragma unroll
        for (int e = 0; e < 4; ++e) {
          x[e] = e >= a && e <= b ? sc[e] * qscale : -INFINITY;
          lmax = fmaxf(lmax, x[e]);
        }
        if (__builtin_amdgcn_ballot_w64(lmax > mref[rt] + 8.f)) {
          const float mn = max_rows4(fmaxf(mref[rt], lmax));
          const float f = mref[rt] == -INFINITY ? 0.f : __builtin_amdgcn_exp2f(mref[rt] - mn);
          lsum[rt] *= f;
#pragma unroll
          for (int dt = 0; dt < DT; ++dt) acc[rt][dt] *= f;
          mref[rt] = mn;
        }
        const float mr = mref[rt] == -INFINITY ? 0.f : mref[rt];
        float p[4];
#pragma unroll
        for (int e = 0; e < 4; ++e) {
          p[e] = __builtin_amdgcn_exp2f(x[e] - mr);
          lsum[rt] += p[e];
        }
        const uint2 pb = make_uint2(px_cvt(p[0], p[1]), px_cvt(p[2], p[3]));
#pragma unroll
        for (int dt = 0; dt < DT; ++dt) acc[rt][dt] = mma16(va[dt], pb, acc[rt][dt]);
      }
      if (bad) {
        const int seq = own ? kb.seq : ka.seq;
        const bf16_t* rows = head.values(seq, p0, entry_of<PAGED>(cv, seq, p0));
#pragma unroll 1
        for (int p = max(p0, lo); p < min(p0 + 16, hi); ++p)
#pragma unroll
          for (int dt = 0; dt < DT; ++dt) {
            const uint2 y = *reinterpret_cast<const uint2*>(rows + (p - p0) * D + dt * 16 + lq * 4);
            const float v[4] = {lo_bf16(y.x), hi_bf16(y.x), lo_bf16(y.y), hi_bf16(y.y)};
#pragma unroll
            for (int rt = 0; rt < RT; ++rt)
#pragma unroll
              for (int e = 0; e < 4; ++e) acc[rt][dt][e] += !own || p <= rpos[rt] ? not_finite(v[e]) : 0.f;
          }
      }
    }
    // the waves meet in LDS, each wave's outputs in its own ring
    wait_lds();
    float* o = reinterpret_cast<float*>(ring);
#pragma unroll
    for (int rt = 0; rt < RT; ++rt) {
      const float l = sum_rows4(lsum[rt]);
#pragma unroll
      for (int dt = 0; dt < DT; ++dt)
        *reinterpret_cast<float4*>(&o[(16 * rt + lr) * D + dt * 16 + 4 * lq]) =
            make_float4(acc[rt][dt][0], acc[rt][dt][1], acc[rt][dt][2], acc[rt][dt][3]);
      if (lq == 0) {
        s_wm[w][16 * rt + lr] = mref[rt];
        s_wl[w][16 * rt + lr] = l;
      }
    }
  };
  if (it.n_row > 16) narrow(std::integral_constant<int, 2>{});
  else narrow(std::integral_constant<int, 1>{});
  __syncthreads();
  constexpr int LPR = D / 4;  // lanes of a row
  for (int idx = t - w0 * 64; idx < it.n_row * LPR; idx += nw * 64) {
    const int r = idx / LPR, d = 4 * (idx % LPR);
    float M = -INFINITY;
#pragma unroll
    for (int k = 0; k < WAVES; ++k)
      if (k < nw) M = fmaxf(M, s_wm[w0 + k][r]);
    float L = 0.f;
    float4 a = make_float4(0.f, 0.f, 0.f, 0.f);
#pragma unroll
    for (int k = 0; k < WAVES; ++k) {
      if (k >= nw) break;
      const float m = s_wm[w0 + k][r];
      const float f = m == -INFINITY ? 0.f : __builtin_amdgcn_exp2f(m - M);
      const float4 o =
          *reinterpret_cast<const float4*>(reinterpret_cast<char*>(s_kv) + (w0 + k) * 2 * TILE + (r * D + d) * 4);
      L = fmaf(s_wl[w0 + k][r], f, L);
      a.x = fmaf(o.x, f, a.x);
      a.y = fmaf(o.y, f, a.y);
      a.z = fmaf(o.z, f, a.z);
      a.w = fmaf(o.w, f, a.w);
    }
    const int row = it.row0 + r;
    const float top = fmaxf(fmaxf(finite_abs(a.x), finite_abs(a.y)), fmaxf(finite_abs(a.z), finite_abs(a.w)));
    const Emit<bf16_t, D> em(pc, it, hk, Hkv, r, plan.rank(row / g).tok, hk * g + row % g, M, L, max_lanes<LPR>(top));
    em.put(d, a.x, a.y, a.z, a.w);
  }
}

// ------------------------------------------------------------------ fp32

// The same items on fp32 caches with v_mfma_f32_16x16x4_f32 (exact products,
// fp32 sums).  One 64-key tile in LDS, two blocks per compute unit; wide items: 16
// rows per wave and all 64 keys; narrow items: the same 16 rows in every wave, 16 of
// the keys each, merged at the end.  The four k indices of a matrix step are dims
// 16 c + 4 lq + e of keys and queries alike, so both are read 16 bytes at a time.
// The next tile's keys are requested when every wave is done with this one's, and
// arrive beside the products with its values; values likewise.
template <int D, bool PAGED, bool VALUE>
__global__ void __launch_bounds__(256, 2) prefix_attend_f32_kernel(PrefixCall pc, Plan<VALUE> plan, CacheView cv) {
  constexpr int DT = D / 16;
  constexpr int NC = D / 4;         // 16-byte chunks of a row
  constexpr int RI = 64 / NC;       // rows of one DMA instruction
  constexpr int KI = 16 / RI;
  constexpr int HALF_T = kPfxTile * D;
  __shared__ __align__(16) float s_kv[2 * HALF_T];
  __shared__ float s_wm[4][16], s_wl[4][16];

  const PrefixItem it = plan.item(blockIdx.y, 0);
  const int hk = blockIdx.x;
  const int t = threadIdx.x, lane = t & 63, lr = lane & 15, lq = lane >> 4;
  const int w = __builtin_amdgcn_readfirstlane(t >> 6);
  const int Hkv = cv.n_kv_heads;
  const int g = pc.g;
  const float qscale = 1.4426950408889634f / sqrtf((float)D);
  const bool narrow = it.n_row <= 16;
  const Keys ka{pc.prefix_seq, it.a0, it.a1}, kb{it.seq, it.b0, it.b1};
  const int na = tiles_of(ka, kPfxTile), nt = na + tiles_of(kb, kPfxTile);
  const HeadRows<float, D, PAGED> head(cv, pc.layer, hk);
  float* K = s_kv;
  float* V = s_kv + HALF_T;

  const int r = (narrow ? 0 : 16 * w) + lr;
  const int row = it.row0 + (r < it.n_row ? r : 0);
  const PrefixRank m = plan.rank(row / g);
  const int rhead = hk * g + row % g;
  px_f32x4 qf[DT];
  {
    const char* src = row_ptr(pc.q, 4, m.tok, rhead);
#pragma unroll
    for (int c = 0; c < DT; ++c) qf[c] = __builtin_bit_cast(px_f32x4, ld16_any(src + (16 * c + 4 * lq) * 4));
  }
  // the compiler cannot see the tile loads: its wait for these must not fall into the loop
#pragma unroll
  for (int c = 0; c < DT; ++c) asm volatile("" ::"v"(qf[c]));
  asm volatile("" ::"v"(m.pos), "v"(m.tok));
  float mref = -INFINITY, lsum = 0.f;
  px_f32x4 acc[DT];
#pragma unroll
  for (int dt = 0; dt < DT; ++dt) acc[dt] = px_f32x4{0.f, 0.f, 0.f, 0.f};
  const bool busy = narrow || 16 * w < it.n_row;
  const int pmin = __builtin_amdgcn_readfirstlane(plan.rank(it.row0 / g).pos);
  auto first_of = [&](int ti) __attribute__((always_inline)) {
    return ((ti >= na ? kb.lo : ka.lo) / kPfxTile + (ti >= na ? ti - na : ti)) * kPfxTile;
  };
  // keys or values of tile ti, 16 rows by each wave
  auto issue = [&](int ti, auto values) __attribute__((always_inline)) {
    const Keys ks = ti >= na ? kb : ka;
    const int q0 = min(max(first_of(ti) + 16 * w, ks.lo & ~15), (ks.hi - 1) & ~15);
    const Entry e = entry_of<PAGED>(cv, ks.seq, q0);
    const int rlo = max(ks.lo - q0, 0), rhi = min(ks.hi - 1 - q0, 15);
    constexpr bool VV = decltype(values)::value;
    const void* base = VV ? head.values(ks.seq, q0, e) : head.keys(ks.seq, q0, e);
#pragma unroll
    for (int j = 0; j < KI; ++j) {
      const int rr = j * RI + lane / NC;
      dma16s(base, (uint32_t)(min(max(rr, rlo), rhi) * D + ((lane % NC) ^ rr) * 4) * 4,
             lds_addr(VV ? V : K) + (w * 16 * D) * 4 + j * 1024);
    }
  };
  // LDS offsets (floats).  Chunk x of row r lies at x ^ (r % 16), so chunk 4 c + lq of key lr at
  // 4 (c ^ lr / 4) + (lq ^ lr % 4), and element 16 dt + lr of key 4 lq + e at chunk
  // 4 (dt ^ lq) + (lr / 4 ^ e): four offsets each for the low two bits of c, dt and e
  int kat[4], vat[4][4];
#pragma unroll
  for (int c = 0; c < 4; ++c) {
    kat[c] = lr * D + 16 * (c ^ (lr >> 2)) + 4 * (lq ^ (lr & 3));
#pragma unroll
    for (int e = 0; e < 4; ++e) vat[c][e] = (4 * lq + e) * D + 16 * (c ^ lq) + 4 * ((lr >> 2) ^ e) + (lr & 3);
  }
  // tile ti of the products: NK groups of 16 keys, from group k0 on
  auto tile = [&](int ti, int k0, auto groups) __attribute__((always_inline)) {
    constexpr int NK = decltype(groups)::value;
    const bool own = ti >= na;
    const int lo = own ? kb.lo : ka.lo, hi = own ? kb.hi : ka.hi, p0 = first_of(ti) + 16 * k0;
    const bool last = ti + 1 == nt;
    px_f32x4 st[NK];
    wait_vm<KI>();  // this wave's keys of the tile have landed ...
    lds_barrier();  // ... and every wave's
    if (busy) {
      const float* Kt = K + k0 * 16 * D;
#pragma unroll
      for (int kt = 0; kt < NK; ++kt) st[kt] = px_f32x4{0.f, 0.f, 0.f, 0.f};
#pragma unroll
      for (int c = 0; c < DT; ++c)
#pragma unroll
        for (int kt = 0; kt < NK; ++kt) {
          const px_f32x4 kf = *reinterpret_cast<const px_f32x4*>(&Kt[kat[c & 3] + (c >> 2) * 64 + kt * 16 * D]);
#pragma unroll
          for (int e = 0; e < 4; ++e) st[kt] = __builtin_amdgcn_mfma_f32_16x16x4f32(kf[e], qf[c][e], st[kt], 0, 0, 0);
        }
    }
    lds_barrier();
    if (!last) issue(ti + 1, std::false_type{});
    float p[NK][4];
    // some row of the item does not see some key (wave-uniform); own keys belong to items of
    // one sequence, whose first row has the smallest position
    const bool edge = p0 < lo || p0 + 16 * NK > (own ? min(hi, pmin + 1) : hi);
    if (busy) {
      if (edge) {
        const int a = lo - p0 - 4 * lq, b = (own ? min(m.pos, hi - 1) : hi - 1) - p0 - 4 * lq;
#pragma unroll
        for (int kt = 0; kt < NK; ++kt)
#pragma unroll
          for (int e = 0; e < 4; ++e) st[kt][e] = 16 * kt + e >= a && 16 * kt + e <= b ? st[kt][e] : -INFINITY;
      }
      float lmax = -INFINITY;
#pragma unroll
      for (int kt = 0; kt < NK; ++kt)
#pragma unroll
        for (int e = 0; e < 4; ++e) lmax = fmaxf(lmax, st[kt][e]);
      lmax *= qscale;
      // as above: the reference moves when a row's max grows by more than 2^8
      if (__builtin_amdgcn_ballot_w64(lmax > mref + 8.f)) {
        const float mn = max_rows4(fmaxf(mref, lmax));
        const float f = mref == -INFINITY ? 0.f : __builtin_amdgcn_exp2f(mref - mn);
        lsum *= f;
#pragma unroll
        for (int dt = 0; dt < DT; ++dt) acc[dt] *= f;
        mref = mn;
      }
      const float mr = mref == -INFINITY ? 0.f : mref;
#pragma unroll
      for (int kt = 0; kt < NK; ++kt)
#pragma unroll
        for (int e = 0; e < 4; ++e) {
          p[kt][e] = __builtin_amdgcn_exp2f(fmaf(st[kt][e], qscale, -mr));
          lsum += p[kt][e];
        }
    }
    if (!last) wait_vm<KI>();  // the tile's values
    else wait_vm<0>();
    lds_barrier();
    if (busy) {
      const float* Vt = V + k0 * 16 * D;
      bool bad = false;
      auto output = [&](auto clean) __attribute__((always_inline)) {
#pragma unroll
        for (int kt = 0; kt < NK; ++kt)
#pragma unroll
          for (int e = 0; e < 4; ++e)
#pragma unroll
            for (int dt = 0; dt < DT; ++dt) {
              float v = Vt[vat[dt & 3][e] + (dt >> 2) * 64 + kt * 16 * D];
              if constexpr (decltype(clean)::value) {
                bad = bad || !(fabsf(v) < INFINITY);
                v = fabsf(v) < INFINITY ? v : 0.f;
              }
              acc[dt] = __builtin_amdgcn_mfma_f32_16x16x4f32(v, p[kt][e], acc[dt], 0, 0, 0);
            }
      };
      if (edge) output(std::true_type{});
      else output(std::false_type{});
      if (edge && __builtin_amdgcn_ballot_w64(bad)) {
#pragma unroll 1
        for (int q = max(p0, lo); q < min(p0 + 16 * NK, hi); ++q) {
          const int key = q - p0;
#pragma unroll
          for (int dt = 0; dt < DT; ++dt) {
            const px_f32x4 v =
                *reinterpret_cast<const px_f32x4*>(&Vt[(key * NC + ((4 * dt + lq) ^ (key & 15))) * 4]);
#pragma unroll
            for (int e = 0; e < 4; ++e) acc[dt][e] += !own || q <= m.pos ? not_finite(v[e]) : 0.f;
          }
        }
      }
    }
    lds_barrier();
    if (!last) issue(ti + 1, std::true_type{});
  };
  if (nt) {
    issue(0, std::false_type{});
    issue(0, std::true_type{});
  }
  if (narrow) {
#pragma unroll 1
    for (int ti = 0; ti < nt; ++ti) tile(ti, w, std::integral_constant<int, 1>{});
  } else {
#pragma unroll 1
    for (int ti = 0; ti < nt; ++ti) tile(ti, 0, std::integral_constant<int, 4>{});
  }
  lsum = sum_rows4(lsum);
  if (!narrow) {
    if (r >= it.n_row) return;
    const Emit<float, D> em(pc, it, hk, Hkv, r, m.tok, rhead, mref, lsum, 0.f);
#pragma unroll
    for (int dt = 0; dt < DT; ++dt) em.put(dt * 16 + 4 * lq, acc[dt][0], acc[dt][1], acc[dt][2], acc[dt][3]);
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
    const Emit<float, D> em(pc, it, hk, Hkv, rr, plan.rank(row2 / g).tok, hk * g + row2 % g, M, L, 0.f);
    em.put(d, a.x, a.y, a.z, a.w);
  }
}

// ------------------------------------------------------------------ merge

// out = sum_s O_s 2^(M_s - M) / sum_s L_s 2^(M_s - M), M = max_s M_s, over the slots
// of a row (O_s kept times 2^up_s).  A row is shared by LPR lanes of 16 bytes each in
// SG groups, group k folding slots k, k + SG, ..., so that the slots arrive in few
// round trips however few rows there are; the groups meet in LDS.
template <typename T, int D, bool VALUE>
__global__ void __launch_bounds__(256) prefix_merge_kernel(PrefixCall pc, Plan<VALUE> plan, int Hq) {
  constexpr int VEC = 16 / (int)sizeof(T);  // elements of a lane: bf16 caches keep fp16 partials
  constexpr int LPR = D / VEC;
  constexpr int SG = 4, RPB = 256 / (LPR * SG);
  __shared__ float s_o[SG][RPB][D];
  __shared__ float s_m[SG][RPB], s_l[SG][RPB];
  const int g = pc.g, Hkv = Hq / g;
  const PrefixRank m = plan.rank(blockIdx.x);
  const int c = threadIdx.x % LPR, k = threadIdx.x / LPR % SG, rb = threadIdx.x / (LPR * SG);
  const int head = blockIdx.y * RPB + rb;
  const int hk = min(head, Hq - 1) / g;
  const int64_t row = (int64_t)hk * pc.rows + (int64_t)blockIdx.x * g + min(head, Hq - 1) % g;
  const int64_t step = (int64_t)Hkv * pc.rows;  // rows from a slot to the next
  const T* po = reinterpret_cast<const T*>(pc.part_o);
  float M = -INFINITY, L = 0.f, acc[VEC];
#pragma unroll
  for (int e = 0; e < VEC; ++e) acc[e] = 0.f;
  constexpr int PF = 4;
  const int n = m.na + m.nb;
  for (int i0 = k; i0 < n; i0 += SG * PF) {
    uint4 x[PF];
    float4 ml[PF];
#pragma unroll
    for (int p = 0; p < PF; ++p) {
      const int i = min(i0 + p * SG, n - 1);
      const int64_t pr = (int64_t)(i < m.na ? i : m.b0 + i - m.na) * step + row;
      x[p] = ld16(po + pr * D + c * VEC);
      ml[p] = *reinterpret_cast<const float4*>(pc.part_ml + pr * 4);
      if (i0 + p * SG >= n) ml[p] = make_float4(-INFINITY, 0.f, 0.f, 0.f);
    }
    float mn = M;
#pragma unroll
    for (int p = 0; p < PF; ++p) mn = fmaxf(mn, ml[p].x);
    const float mr = mn == -INFINITY ? 0.f : mn;
    const float f = M == -INFINITY ? 0.f : __builtin_amdgcn_exp2f(M - mr);
    L *= f;
#pragma unroll
    for (int e = 0; e < VEC; ++e) acc[e] *= f;
#pragma unroll
    for (int p = 0; p < PF; ++p) {
      // a slot without a visible key: no weight (its sum is 0, or NaN where its scores were)
      const bool none = ml[p].x == -INFINITY;
      const float part = none ? 0.f : __builtin_amdgcn_exp2f(ml[p].x - mr);
      L = fmaf(ml[p].y, part, L);
      // the two powers apart: of one sum of exponents, small values' (up 126) came out as 0
      // and others lost bits of the first to the size of the second
      const float wgt = part * __builtin_amdgcn_exp2f(-ml[p].z);
      float y[VEC];
      if constexpr (sizeof(T) == 2) {
        const px_f16x8 h = __builtin_bit_cast(px_f16x8, x[p]);
#pragma unroll
        for (int e = 0; e < VEC; ++e) y[e] = (float)h[e];
      } else {
        Store<float>::unpack(x[p], y);
      }
      if (!none) {
#pragma unroll
        for (int e = 0; e < VEC; ++e) acc[e] = fmaf(y[e], wgt, acc[e]);
      }
    }
    M = mn;
  }
#pragma unroll
  for (int e = 0; e < VEC; e += 4)
    *reinterpret_cast<float4*>(&s_o[k][rb][c * VEC + e]) = make_float4(acc[e], acc[e + 1], acc[e + 2], acc[e + 3]);
  if (c == 0) {
    s_m[k][rb] = M;
    s_l[k][rb] = L;
  }
  __syncthreads();
  // 256 lanes over RPB rows of D: D RPB / 256 elements each
  constexpr int EPL = D * RPB / 256;
  const int r2 = threadIdx.x / (D / EPL), d = threadIdx.x % (D / EPL) * EPL;
  const int head2 = blockIdx.y * RPB + r2;
  if (head2 >= Hq) return;
  float M2 = -INFINITY, L2 = 0.f, y[EPL];
#pragma unroll
  for (int q = 0; q < SG; ++q) M2 = fmaxf(M2, s_m[q][r2]);
#pragma unroll
  for (int e = 0; e < EPL; ++e) y[e] = 0.f;
#pragma unroll
  for (int q = 0; q < SG; ++q) {
    const float f = s_m[q][r2] == -INFINITY ? 0.f : __builtin_amdgcn_exp2f(s_m[q][r2] - M2);
    L2 = fmaf(s_l[q][r2], f, L2);
#pragma unroll
    for (int e = 0; e < EPL; ++e) y[e] = fmaf(s_o[q][r2][d + e], f, y[e]);
  }
  const float inv = L2 == 0.f ? 0.f : 1.f / L2;
  T* dst = reinterpret_cast<T*>(const_cast<char*>(row_ptr(pc.out, sizeof(T), m.tok, head2))) + d;
#pragma unroll
  for (int e = 0; e < EPL; ++e) y[e] *= inv;
  if constexpr (sizeof(T) == 2) {
    uint32_t o[EPL / 2];
#pragma unroll
    for (int e = 0; e < EPL / 2; ++e) o[e] = px_cvt(y[2 * e], y[2 * e + 1]);
    __builtin_memcpy(dst, o, EPL * 2);
  } else {
    __builtin_memcpy(dst, y, EPL * 4);
  }
  if (d == 0 && pc.lse) pc.lse[(int64_t)m.tok * Hq + head2] = L2 == 0.f ? -INFINITY : (M2 + log2f(L2)) * kLn2;
}

static int check(hipError_t e) { return e == hipSuccess ? 0 : (int)e; }

int launch_prefix_attend(int dtype, const PrefixCall& call, const PrefixArgs* args, const PrefixItem* items,
                         const PrefixRank* ranks, int n_items, int waves, const CacheView& cv, hipStream_t s) {
  if (n_items == 0) return 0;
  if (n_items > 65535) return (int)hipErrorInvalidValue;
  const dim3 grid(cv.n_kv_heads, n_items);
  const Plan<false> lst{items, ranks};
#define PA(...) hipLaunchKernelGGL((__VA_ARGS__)
#define PB(DD, PG)                                                                                                  \
  {                                                                                                                 \
    if (waves == 8 && args)                                                                                         \
      PA(prefix_attend_kernel<DD, PG, 8, true>), grid, dim3(512), 0, s, call, Plan<true>{*args}, cv);               \
    else if (waves == 8) PA(prefix_attend_kernel<DD, PG, 8, false>), grid, dim3(512), 0, s, call, lst, cv);         \
    else if (args) PA(prefix_attend_kernel<DD, PG, 4, true>), grid, dim3(256), 0, s, call, Plan<true>{*args}, cv);  \
    else PA(prefix_attend_kernel<DD, PG, 4, false>), grid, dim3(256), 0, s, call, lst, cv);                         \
  }
#define PF(DD, PG)                                                                                                  \
  {                                                                                                                 \
    if (args) PA(prefix_attend_f32_kernel<DD, PG, true>), grid, dim3(256), 0, s, call, Plan<true>{*args}, cv);      \
    else PA(prefix_attend_f32_kernel<DD, PG, false>), grid, dim3(256), 0, s, call, lst, cv);                        \
  }
  const bool paged = cv.page_size != 0, small = cv.head_dim == 64;
  if (dtype == 0) {
    if (paged) { if (small) PF(64, true) else PF(128, true) }
    else { if (small) PF(64, false) else PF(128, false) }
  } else {
    if (paged) { if (small) PB(64, true) else PB(128, true) }
    else { if (small) PB(64, false) else PB(128, false) }
  }
#undef PF
#undef PB
#undef PA
  return check(hipGetLastError());
}

int launch_prefix_merge(int dtype, const PrefixCall& call, const PrefixArgs* args, const PrefixRank* ranks, int n_rank,
                        int Hq, int D, hipStream_t s) {
  if (n_rank == 0) return 0;
  const int rpb = 256 / (D * (dtype == 0 ? 4 : 2) / 16 * 4);
  const dim3 grid(n_rank, (Hq + rpb - 1) / rpb);
  const Plan<false> lst{nullptr, ranks};
#define PM(T, DD)                                                                                             \
  {                                                                                                           \
    if (args) hipLaunchKernelGGL((prefix_merge_kernel<T, DD, true>), grid, dim3(256), 0, s, call, Plan<true>{*args}, Hq); \
    else hipLaunchKernelGGL((prefix_merge_kernel<T, DD, false>), grid, dim3(256), 0, s, call, lst, Hq);       \
  }
  if (dtype == 0) { if (D == 64) PM(float, 64) else PM(float, 128) }
  else { if (D == 64) PM(bf16_t, 64) else PM(bf16_t, 128) }
#undef PM
  return check(hipGetLastError());
}

}  // namespace fcg

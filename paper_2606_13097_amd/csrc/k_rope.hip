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
#include "rope_rows.hpp"

namespace fcg {

template <typename T, int D, bool PAIRS, int MODE, bool PAGED>
__global__ void __launch_bounds__(256) rope_rows_kernel(Where<MODE> where, RopeRows rows, CacheView cv, int layer0,
                                                        RopeArgs ra, const float2* __restrict__ tab) {
  rope_rows<T, D, PAIRS, MODE, PAGED, false>(where, rows, cv, layer0, ra, tab, NormArgs<false>{});
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

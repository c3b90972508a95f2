// Entry points of norms with a rotary turn (include/fcg.h): apply, its gradient, append.
#include <cfloat>
#include <cmath>

#include "objects.hpp"
#include "ops.hpp"

using namespace fcg;

namespace {

fcg_status check_norm(const fcg_norm* n, const char* what) {
  if (!n) return FCG_OK;
  if (n->layer < 0 || n->head < 0) return fail(FCG_EINVAL, std::string(what) + ": negative stride of the norm's weights");
  if (!(n->eps >= (double)FLT_MIN && n->eps <= (double)FLT_MAX))
    return fail(FCG_EINVAL, std::string(what) + ": eps must be > 0, in the range of normal fp32 numbers");
  if (!(std::fabs(n->offset) <= (double)FLT_MAX)) return fail(FCG_EINVAL, std::string(what) + ": offset is not finite");
  return FCG_OK;
}

NormView view_of(const fcg_norm* n) {
  if (!n) return NormView{nullptr, 0, 0, 1.f, 1.f, 0};
  return NormView{n->weight, n->layer, n->head, (float)n->eps, n->weight ? (float)n->offset : 1.f, 1};
}

fcg_status check_shape(const fcg_rope* rope, int32_t dtype, int32_t head_dim, int32_t n_layers, int32_t n_tok) {
  if (!rope) return fail(FCG_EINVAL, "null rope");
  if (dtype != FCG_F32 && dtype != FCG_BF16) return fail(FCG_EINVAL, "unknown dtype");
  if (head_dim != 64 && head_dim != 128) return fail(FCG_EINVAL, "head_dim must be 64 or 128");
  if (rope->rot > head_dim) return fail(FCG_EINVAL, "rotary_dim exceeds head_dim");
  if (n_layers < 0 || n_layers > 65535 || n_tok < 0) return fail(FCG_EINVAL, "a count is negative, or more than 65535 layers");
  if (n_tok > 1 << 30) return fail(FCG_EINVAL, "more than 2^30 tokens");
  return FCG_OK;
}

fcg_status check_heads(int32_t heads) {
  if (heads < 0 || heads > 4096) return fail(FCG_EINVAL, "heads must be in [0, 4096]");
  return FCG_OK;
}

// How a side of the backward pass is cut: ranges of heads, and `spread` blocks that share
// the chunks of tokens of each.  Four blocks for each of 256 compute units, over all layers
// and both sides, with as many heads each as leave that many (a chunk's angles are computed by
// every block that has it); each leaves a partial of the weights' gradient.  (4.4K tokens of
// 16 + 4 fp32 heads, for 512, 1024, 2048 and 4096 blocks: 40, 37, 40, 43 us.)
struct SideCut {
  int32_t heads_per, head_blocks, spread;
};
SideCut cut_side(int32_t dtype, int32_t head_dim, int32_t n_layers, int32_t n_tok, int32_t heads, int32_t all_heads) {
  constexpr int64_t kBlocks = 1024;
  const int32_t tokens = norm_tokens(head_dim, esize(dtype));
  const int64_t chunks = std::max<int64_t>(1, (n_tok + tokens - 1) / tokens);
  SideCut c;
  c.heads_per = (int32_t)std::min<int64_t>({heads, kNormHeads, std::max<int64_t>(1, n_layers * chunks * all_heads / kBlocks)});
  c.head_blocks = (heads + c.heads_per - 1) / c.heads_per;
  c.heads_per = (heads + c.head_blocks - 1) / c.head_blocks;  // ranges of like size
  const int64_t total = (int64_t)n_layers * ((all_heads + c.heads_per - 1) / c.heads_per);
  c.spread = (int32_t)std::max<int64_t>(1, std::min(chunks, (kBlocks + total - 1) / total));
  return c;
}

}  // namespace

// ----------------------------------------------------------------------- apply

fcg_status fcg_norm_rope_apply(const fcg_rope* rope, int32_t dtype, int32_t head_dim, int32_t n_layers, int32_t n_tok,
                               const int32_t* pos, int32_t n_q_heads, const fcg_norm* q_norm, const fcg_tensor* q,
                               const fcg_tensor* q_out, int32_t n_k_heads, const fcg_norm* k_norm,
                               const fcg_tensor* k, const fcg_tensor* k_out, void* stream) {
  if (fcg_status st = check_shape(rope, dtype, head_dim, n_layers, n_tok)) return st;
  struct {
    const fcg_tensor *in, *out;
    int32_t heads;
    const fcg_norm* norm;
    const char* name;
  } both[2] = {{q, q_out, n_q_heads, q_norm, "q"}, {k, k_out, n_k_heads, k_norm, "k"}};
  bool has[2], work = false;
  for (int i = 0; i < 2; ++i) {
    const auto& b = both[i];
    if (fcg_status st = check_heads(b.heads)) return st;
    has[i] = b.in && b.heads;
    work = work || (has[i] && n_layers > 0 && n_tok > 0);
    if (has[i] && !b.out) return fail(FCG_EINVAL, "an input without its output");
    if (fcg_status st = check_norm(b.norm, b.name)) return st;
  }
  if (work && !pos) return fail(FCG_EINVAL, "null positions");
  for (int i = 0; i < 2; ++i) {
    if (!has[i]) continue;
    const auto& b = both[i];
    if (work && (!b.in->data || !b.out->data)) return fail(FCG_EINVAL, std::string(b.name) + ": null tensor");
    if (fcg_status st = check_strides(b.in, b.name)) return st;
    if (fcg_status st = check_strides(b.out, b.name)) return st;
    if (fcg_status st = check_output(b.out, n_layers, n_tok, b.heads, head_dim, b.name)) return st;
    if (work)
      if (fcg_status st = check_alias(b.in, b.out, b.name)) return st;
  }
  if (!work) return FCG_OK;
  RopeRows rows{};
  if (has[0]) {
    rows.q = fcg::view_of(q);
    rows.q_out = fcg::view_of(q_out);
    rows.Hq = n_q_heads;
  }
  if (has[1]) {
    rows.k = fcg::view_of(k);
    rows.k_out = fcg::view_of(k_out);
    rows.Hk = n_k_heads;
  }
  rows.n_layers = n_layers;
  rows.sign = 1.f;
  cut_rows(&rows, n_tok, n_layers, rows.Hq + rows.Hk, head_dim * (int)esize(dtype) / 32);
  const RopeArgs args = rope->args();
  const NormArgs<true> norm{::view_of(q_norm), ::view_of(k_norm)};
  const int64_t per = (int64_t)kGridX * rows.tb;  // tokens of a launch
  for (int64_t t0 = 0; t0 < n_tok; t0 += per) {
    RopeRows part = rows;
    for (RowView* v : {&part.q, &part.q_out, &part.k, &part.k_out})
      if (v->p) v->p = (const char*)v->p + t0 * v->token * (int64_t)esize(dtype);
    part.n_tok = (int32_t)std::min<int64_t>(per, n_tok - t0);
    if (int rc = launch_norm_rope(dtype, head_dim, rope->pairs(), part, pos + t0, args, norm, (hipStream_t)stream))
      return hip_fail((hipError_t)rc, "norm launch");
  }
  return FCG_OK;
}

// -------------------------------------------------------------------- gradient

fcg_status fcg_norm_rope_workspace(int32_t head_dim, int32_t n_layers, int32_t n_tok, int32_t n_q_heads,
                                   int32_t n_k_heads, int64_t* bytes) {
  if (!bytes) return fail(FCG_EINVAL, "null output");
  if (head_dim != 64 && head_dim != 128) return fail(FCG_EINVAL, "head_dim must be 64 or 128");
  if (n_layers < 0 || n_layers > 65535 || n_tok < 0 || n_tok > 1 << 30) return fail(FCG_EINVAL, "a count is out of range");
  int64_t rows = 0;
  for (int32_t heads : {n_q_heads, n_k_heads}) {
    if (fcg_status st = check_heads(heads)) return st;
    if (!heads || !n_layers) continue;
    int64_t most = 0;
    for (int32_t dtype : {FCG_F32, FCG_BF16})
      most = std::max<int64_t>(most, cut_side(dtype, head_dim, n_layers, n_tok, heads, n_q_heads + n_k_heads).spread);
    rows += (int64_t)n_layers * most * heads;  // (shared weights take ranges of heads in place of heads)
  }
  *bytes = rows * head_dim * 4;
  return FCG_OK;
}

fcg_status fcg_norm_rope_backward(const fcg_rope* rope, int32_t dtype, int32_t head_dim, int32_t n_layers,
                                  int32_t n_tok, const int32_t* pos, const fcg_norm_side* q, const fcg_norm_side* k,
                                  void* workspace, int64_t workspace_bytes, void* stream) {
  if (fcg_status st = check_shape(rope, dtype, head_dim, n_layers, n_tok)) return st;
  const fcg_norm_side* side[2] = {q && q->heads ? q : nullptr, k && k->heads ? k : nullptr};
  const char* name[2] = {"q", "k"};
  for (const fcg_norm_side* s : {q, k})
    if (s)
      if (fcg_status st = check_heads(s->heads)) return st;
  const bool rows = n_layers > 0 && n_tok > 0;
  int32_t all_heads = 0;
  bool any = false, dweight = false;
  for (int i = 0; i < 2; ++i) {
    const fcg_norm_side* s = side[i];
    if (!s) continue;
    any = true;
    all_heads += s->heads;
    if (fcg_status st = check_norm(s->norm, name[i])) return st;
    if (s->dweight && (!s->norm || !s->norm->weight))
      return fail(FCG_EINVAL, std::string(name[i]) + ": a gradient of weights that are not given");
    dweight = dweight || s->dweight;
    if (rows && (!s->grad.data || !s->dx.data || (s->norm && !s->x.data)))
      return fail(FCG_EINVAL, std::string(name[i]) + ": null tensor");
    for (const fcg_tensor* t : {&s->x, &s->grad, &s->dx})
      if (fcg_status st = check_strides(t, name[i])) return st;
    if (fcg_status st = check_output(&s->dx, n_layers, n_tok, s->heads, head_dim, name[i])) return st;
    if (!rows) continue;
    if (s->norm)
      if (fcg_status st = check_alias(&s->x, &s->dx, name[i])) return st;
    if (fcg_status st = check_alias(&s->grad, &s->dx, name[i])) return st;
  }
  if (!any || !n_layers) return FCG_OK;
  if (rows && !pos) return fail(FCG_EINVAL, "null positions");
  if (!rows && !dweight) return FCG_OK;
  NormGradArgs a{};
  a.pos = pos;
  a.part = (float*)workspace;
  a.n_tok = n_tok;
  a.n_layers = n_layers;
  int64_t part = 0;
  for (int i = 0; i < 2; ++i) {
    const fcg_norm_side* s = side[i];
    if (!s) continue;
    NormSide& d = a.side[i];
    // (rows that are turned only: any readable rows in place of x)
    d.x = fcg::view_of(s->norm ? &s->x : &s->grad);
    d.gy = fcg::view_of(&s->grad);
    d.dx = fcg::view_of(&s->dx);
    d.norm = ::view_of(s->norm);
    d.dw = s->dweight;
    d.part0 = part;
    d.heads = s->heads;
    d.w_heads = s->norm && s->norm->head ? s->heads : 1;
    const SideCut c = cut_side(dtype, head_dim, n_layers, n_tok, s->heads, all_heads);
    d.heads_per = c.heads_per;
    d.head_blocks = c.head_blocks;
    d.spread = c.spread;
    d.parts = n_tok ? d.w_heads > 1 ? c.spread : c.spread * c.head_blocks : 0;
    if (s->dweight) part += (int64_t)n_layers * d.w_heads * d.parts * head_dim;
    if (i == 0) a.blocks_q = c.head_blocks * c.spread;
  }
  if (part) {
    if (!workspace || (uintptr_t)workspace % 16) return fail(FCG_EINVAL, "workspace: null or not 16-byte aligned");
    if (workspace_bytes < part * 4) return fail(FCG_EINVAL, "the workspace is too small");
  }
  if (int rc = launch_norm_rope_grad(dtype, head_dim, rope->pairs(), a, rope->args(), (hipStream_t)stream))
    return hip_fail((hipError_t)rc, "norm gradient launch");
  return FCG_OK;
}

// ---------------------------------------------------------------------- append

fcg_status fcg_append_norm(fcg_cache* c, int32_t layer, int32_t n_layers, int32_t n_tok, const int32_t* seq,
                           const int32_t* pos, const fcg_rope* rope, const fcg_norm* q_norm, const fcg_norm* k_norm,
                           const fcg_tensor* q, const fcg_tensor* q_out, const fcg_tensor* k, const fcg_tensor* v,
                           uint32_t flags, void* stream) {
  if (fcg_status st = check_norm(q_norm, "q")) return st;
  if (fcg_status st = check_norm(k_norm, "k")) return st;
  const bool rows = n_layers > 0 && n_tok > 0;  // (tensors of none may have no address)
  if (rows && ((q_norm && !(q && q->data)) || (k_norm && !(k && k->data))))
    return fail(FCG_EINVAL, "a norm without its rows");
  const NormArgs<true> norm{::view_of(q_norm), ::view_of(k_norm)};
  auto launch = [](const void* context, int dtype, bool pairs, const RopeRows& rows, const AppendArgs& args, int n_runs,
                   const AppendGroup* groups, int n_groups, const CacheView& cv, int layer0, const RopeArgs& ra,
                   const float2* tab, hipStream_t s) {
    return launch_append_norm(dtype, pairs, rows, args, n_runs, groups, n_groups, cv, layer0, ra, tab,
                              *(const NormArgs<true>*)context, s);
  };
  return append_tokens(c, layer, n_layers, n_tok, seq, pos, rope, q, q_out, k, v, flags, stream, AppendLaunch{launch, &norm});
}

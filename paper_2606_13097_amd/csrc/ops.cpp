// Entry points around the cache that take a rotary handle or a shared prefix
// (include/fcg.h): rotary handles, rope apply, append, prefix attention.
#include <algorithm>
#include <cfloat>
#include <cmath>

#include "objects.hpp"

using namespace fcg;

namespace {

fcg_status fail(fcg_status s, const std::string& msg) { return report(s, msg); }

bool capturing(hipStream_t s) {
  hipStreamCaptureStatus st = hipStreamCaptureStatusNone;
  if (hipStreamIsCapturing(s, &st) == hipSuccess) return st != hipStreamCaptureStatusNone;
  (void)hipGetLastError();  // not this call's error
  return false;
}

RowView view_of(const fcg_tensor* t) {
  return t ? RowView{t->data, t->layer, t->token, t->head} : RowView{nullptr, 0, 0, 0};
}

// strides of a tensor [layers][tokens][heads][D]
fcg_status check_strides(const fcg_tensor* t, const char* what) {
  if (t && (t->layer < 0 || t->token < 0 || t->head < 0))
    return fail(FCG_EINVAL, std::string(what) + ": negative stride");
  return FCG_OK;
}

// Rows of an output must not meet: sorted by stride, each dimension steps over
// what the smaller ones cover.
fcg_status check_output(const fcg_tensor* t, int64_t layers, int64_t tokens, int64_t heads, int64_t D, const char* what) {
  std::pair<int64_t, int64_t> dim[3] = {{t->layer, layers}, {t->token, tokens}, {t->head, heads}};  // stride, size
  std::sort(dim, dim + 3);
  int64_t extent = D;
  for (auto& d : dim) {
    if (d.second <= 1) continue;
    if (d.first < extent) return fail(FCG_EINVAL, std::string(what) + ": rows of an output overlap");
    extent = d.first * (d.second - 1) + extent;
  }
  return FCG_OK;
}

bool same_view(const fcg_tensor* a, const fcg_tensor* b) {
  return a->data == b->data && a->layer == b->layer && a->token == b->token && a->head == b->head;
}

// an output that starts where its input does is that input in place, or an error
fcg_status check_alias(const fcg_tensor* in, const fcg_tensor* out, const char* what) {
  if (in->data == out->data && !same_view(in, out))
    return fail(FCG_EINVAL, std::string(what) + ": an output in its input's place needs its strides");
  return FCG_OK;
}

}  // namespace

// ---------------------------------------------------------------- rotary forms

fcg_status fcg_rope_create(const fcg_rope_desc* d, fcg_rope** out) {
  if (!d || !out) return fail(FCG_EINVAL, "null rope descriptor or output");
  if (d->rotary_dim < 16 || d->rotary_dim > 2 * kRopePairs || d->rotary_dim % 16)
    return fail(FCG_EINVAL, "rotary_dim must be a multiple of 16 in [16, 128]");
  if (d->layout != FCG_ROPE_HALF && d->layout != FCG_ROPE_PAIRS) return fail(FCG_EINVAL, "unknown rope layout");
  if (d->scaling < FCG_ROPE_PLAIN || d->scaling > FCG_ROPE_GIVEN) return fail(FCG_EINVAL, "unknown rope scaling");
  // (the kernels take it in fp32)
  if (!(d->attn_factor >= (double)FLT_MIN && d->attn_factor <= (double)FLT_MAX))
    return fail(FCG_EINVAL, "attn_factor must be > 0, in the range of normal fp32 numbers");
  const bool given = d->scaling == FCG_ROPE_GIVEN, scaled = d->scaling != FCG_ROPE_PLAIN && !given;
  if (!given && (!(d->theta > 1.0) || !std::isfinite(d->theta))) return fail(FCG_EINVAL, "theta must be > 1");
  if (scaled && (!(d->factor >= 1.0) || !std::isfinite(d->factor))) return fail(FCG_EINVAL, "factor must be >= 1");
  if (d->scaling == FCG_ROPE_PARTS) {
    if (!(d->orig_tokens > 0.0) || !std::isfinite(d->orig_tokens)) return fail(FCG_EINVAL, "orig_tokens must be > 0");
    if (!(d->low_turns >= 0.0) || !(d->high_turns > d->low_turns) || !std::isfinite(d->high_turns))
      return fail(FCG_EINVAL, "0 <= low_turns < high_turns is needed");
  }
  const int n = d->rotary_dim / 2;
  if (given) {
    if (!d->freqs) return fail(FCG_EINVAL, "null frequencies");
    for (int i = 0; i < n; ++i)
      if (!std::isfinite(d->freqs[i] * 2147483648.0))
        return fail(FCG_EINVAL, "a frequency, or its angle at position 2^31, is not finite");
  }
  return guarded([&]() -> fcg_status {
    std::vector<double> w(n);
    const double R = d->rotary_dim;
    const double theta = d->scaling == FCG_ROPE_NTK ? d->theta * std::pow(d->factor, R / (R - 2.0)) : d->theta;
    for (int i = 0; i < n; ++i) {
      w[i] = given ? d->freqs[i] : std::pow(theta, -2.0 * i / R);
      if (d->scaling == FCG_ROPE_LINEAR) w[i] /= d->factor;
      if (d->scaling == FCG_ROPE_PARTS) {
        const double r = d->orig_tokens * w[i] / 6.283185307179586477;
        const double keep = std::min(1.0, std::max(0.0, (r - d->low_turns) / (d->high_turns - d->low_turns)));
        w[i] *= (1.0 - keep) / d->factor + keep;
      }
    }
    fcg_rope* r = new fcg_rope();
    r->rot = d->rotary_dim;
    r->layout = d->layout;
    r->attn_factor = d->attn_factor;
    r->freqs = std::move(w);
    *out = r;
    return FCG_OK;
  });
}

fcg_status fcg_rope_frequencies(const fcg_rope* rope, double* freqs) {
  if (!rope || !freqs) return fail(FCG_EINVAL, "null rope or output");
  std::copy(rope->freqs.begin(), rope->freqs.end(), freqs);
  return FCG_OK;
}

fcg_status fcg_rope_destroy(fcg_rope* rope) {
  delete rope;
  return FCG_OK;
}

namespace {

// How the tokens' rows are cut into blocks.  A block moves slice_rows rows of a group of
// tb tokens, kRopePass pairs of vectors (nch of each row).  Groups as large as fill their
// slices best, while there are a few blocks for each compute unit: the (cos, sin) of a token
// are computed by each block that has rows of it.  Where up to four layers a block bring
// the grid down to what is resident at once (eight blocks for each of 256 compute units),
// they do (32 layers of 713 tokens of 8 heads, one layer a block 18.2 us, two 17.3, three
// 16.2, four 16.7); larger calls keep one (8 layers of 11K tokens into pages, one 417 us,
// two 429, three 436).
void cut_rows(RopeRows* rows, int64_t n_tok, int64_t n_layers, int H, int nch) {
  constexpr int64_t kResident = 2048;
  const int slice = kRopePass / nch;
  rows->tb = 1;
  double best = 0.0;
  for (int tb = 1; tb <= kAppMaxTb; ++tb) {
    const int64_t slices = ((int64_t)tb * H + slice - 1) / slice;
    if (tb > 1 && (n_tok + tb - 1) / tb * slices * n_layers < kResident) break;
    const double used = (double)tb * H / (double)(slices * slice);
    if (used > best + 0.02) {
      best = used;
      rows->tb = tb;
    }
  }
  rows->slice_rows = std::min(slice, rows->tb * H);
  rows->h_magic = H > 1 ? (uint32_t)((((uint64_t)1 << 32) + H - 1) / H) : 0;
  const int64_t blocks = (n_tok + rows->tb - 1) / rows->tb * (((int64_t)rows->tb * H + slice - 1) / slice) * n_layers;
  const int64_t each = (blocks + kResident - 1) / kResident;
  rows->grid_layers = (int32_t)(each <= 4 ? (n_layers + each - 1) / each : n_layers);
  // More than the last-level cache holds (256 MB): nothing of it will be there when it is read
  // (2.2 GB in all, plain 414 us, written past the caches 401, read so too 385).  Less may lie
  // there (96 MB in all 17.2 us, read past the caches 21.4).
  rows->stream = n_tok * n_layers * H * nch * 32 > (int64_t)256 << 20;
}

}  // namespace

fcg_status fcg_rope_apply(const fcg_rope* rope, int32_t dtype, int32_t head_dim, int32_t n_layers, int32_t n_tok,
                          const int32_t* pos, int32_t n_q_heads, const fcg_tensor* q, const fcg_tensor* q_out,
                          int32_t n_k_heads, const fcg_tensor* k, const fcg_tensor* k_out, uint32_t flags,
                          void* stream) {
  if (!rope) return fail(FCG_EINVAL, "null rope");
  if (dtype != FCG_F32 && dtype != FCG_BF16) return fail(FCG_EINVAL, "unknown dtype");
  if (head_dim != 64 && head_dim != 128) return fail(FCG_EINVAL, "head_dim must be 64 or 128");
  if (rope->rot > head_dim) return fail(FCG_EINVAL, "rotary_dim exceeds head_dim");
  if (n_layers < 0 || n_layers > 65535 || n_tok < 0 || n_q_heads < 0 || n_k_heads < 0)
    return fail(FCG_EINVAL, "a count is negative, or more than 65535 layers");
  if (n_tok > 1 << 30) return fail(FCG_EINVAL, "more than 2^30 tokens");
  if (n_q_heads > 4096 || n_k_heads > 4096) return fail(FCG_EINVAL, "more than 4096 heads");
  if (flags & ~FCG_ROPE_BACKWARD) return fail(FCG_EINVAL, "unknown flags");
  const bool has_q = q && n_q_heads, has_k = k && n_k_heads;
  if ((has_q && !q_out) || (has_k && !k_out)) return fail(FCG_EINVAL, "an input without its output");
  struct {
    const fcg_tensor *in, *out;
    int32_t heads;
    const char* name;
  } both[2] = {{q, q_out, n_q_heads, "q"}, {k, k_out, n_k_heads, "k"}};
  const bool work = n_layers > 0 && n_tok > 0 && (has_q || has_k);
  if (work && !pos) return fail(FCG_EINVAL, "null positions");
  for (int i = 0; i < 2; ++i) {
    if (!(i ? has_k : has_q)) continue;
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
  if (has_q) {
    rows.q = view_of(q);
    rows.q_out = view_of(q_out);
    rows.Hq = n_q_heads;
  }
  if (has_k) {
    rows.k = view_of(k);
    rows.k_out = view_of(k_out);
    rows.Hk = n_k_heads;
  }
  rows.n_tok = n_tok;
  rows.n_layers = n_layers;
  rows.sign = flags & FCG_ROPE_BACKWARD ? -1.f : 1.f;
  cut_rows(&rows, n_tok, n_layers, rows.Hq + rows.Hk, head_dim * (int)esize(dtype) / 32);
  const RopeArgs args = rope->args();
  const int64_t per = (int64_t)kGridX * rows.tb;  // tokens of a launch
  for (int64_t t0 = 0; t0 < n_tok; t0 += per) {
    RopeRows part = rows;
    for (RowView* v : {&part.q, &part.q_out, &part.k, &part.k_out})
      if (v->p) v->p = (const char*)v->p + t0 * v->token * (int64_t)esize(dtype);
    part.n_tok = (int32_t)std::min<int64_t>(per, n_tok - t0);
    if (int rc = launch_rope_apply(dtype, head_dim, rope->pairs(), part, pos + t0, args, (hipStream_t)stream))
      return hip_fail((hipError_t)rc, "rope launch");
  }
  return FCG_OK;
}

// ---------------------------------------------------------------------- append

fcg_status fcg_append(fcg_cache* c, int32_t layer, int32_t n_layers, int32_t n_tok, const int32_t* seq,
                      const int32_t* pos, const fcg_rope* rope, const fcg_tensor* q, const fcg_tensor* q_out,
                      const fcg_tensor* k, const fcg_tensor* v, uint32_t flags, void* stream) {
  if (!c) return fail(FCG_EINVAL, "null cache");
  if (n_layers < 0 || n_tok < 0) return fail(FCG_EINVAL, "negative count");
  if (n_tok > 0 && (!seq || !pos)) return fail(FCG_EINVAL, "null token array");
  if (flags & ~FCG_REPLACE) return fail(FCG_EINVAL, "unknown flags");
  const fcg_model_desc& d = c->desc;
  if (rope && rope->rot > d.head_dim) return fail(FCG_EINVAL, "rotary_dim exceeds head_dim");
  const bool has_k = k && k->data, has_v = v && v->data, has_q = q && q->data;
  if (has_k != has_v) return fail(FCG_EINVAL, "k and v must both be given or both be null");
  if (has_q && (!q_out || !q_out->data)) return fail(FCG_EINVAL, "q without q_out");
  if (has_q && !has_k) return fail(FCG_EINVAL, "q without k and v");
  if (has_k && c->layout_only()) return fail(FCG_EINVAL, "a layout-only cache takes no data");
  for (const fcg_tensor* t : {has_k ? k : nullptr, has_v ? v : nullptr, has_q ? q : nullptr, has_q ? q_out : nullptr})
    if (fcg_status st = check_strides(t, "append")) return st;
  if (has_q) {
    if (fcg_status st = check_output(q_out, n_layers, n_tok, d.n_q_heads, d.head_dim, "q_out")) return st;
    if (fcg_status st = check_alias(q, q_out, "q")) return st;
  }
  return guarded([&]() -> fcg_status {
    std::vector<std::pair<int32_t, int32_t>> new_pages;
    std::vector<int32_t> order;
    std::vector<Span> runs_of;  // runs of consecutive positions
    std::string msg;
    if (fcg_status st = c->plan.check_place(layer, n_layers, n_tok, seq, pos, (flags & FCG_REPLACE) != 0, &order,
                                            &runs_of, &new_pages, &msg))
      return fail(st, msg);
    if (n_tok == 0 || n_layers == 0) return FCG_OK;
    Staged staged(c, new_pages);
    auto commit = [&]() {
      staged.keep();
      for (const Span& x : runs_of)
        for (int32_t l = layer; l < layer + n_layers; ++l) c->plan.mark_range(x.seq, l, x.dst, x.len);
      return FCG_OK;
    };
    if (c->layout_only()) {
      staged.map();
      return commit();
    }
    if (!has_k && new_pages.empty()) return commit();  // nothing for the device to do
    OnDevice dev(c->device);
    HIP_TRY(dev.err, "hipSetDevice");
    hipStream_t s = (hipStream_t)stream;
    RopeRows rows{};
    rows.n_tok = n_tok;
    rows.n_layers = n_layers;
    rows.sign = 1.f;
    if (has_q) {
      rows.q = view_of(q);
      rows.q_out = view_of(q_out);
      rows.Hq = d.n_q_heads;
    }
    if (has_k) {
      rows.k = view_of(k);
      rows.v = view_of(v);
      rows.Hk = rows.Hv = d.n_kv_heads;
    }
    const int H = rows.Hq + rows.Hk + rows.Hv;
    cut_rows(&rows, n_tok, n_layers, std::max(H, 1), d.head_dim * (int)esize(d.dtype) / 32);
    // runs: consecutive positions of one sequence at consecutive indices
    std::vector<AppendRun> runs;
    for (int32_t i = 0; i < n_tok;) {
      const int32_t t0 = order[i];
      int32_t j = i + 1;
      while (j < n_tok && order[j] == t0 + (j - i) && seq[order[j]] == seq[t0] && pos[order[j]] == pos[t0] + (j - i)) ++j;
      runs.push_back(AppendRun{t0, seq[t0], pos[t0], j - i, 0, 0});
      i = j;
    }
    int64_t n_page = 0;
    int32_t n_groups = 0;
    for (auto& r : runs) {
      r.grp0 = n_groups;
      n_groups += (r.n + rows.tb - 1) / rows.tb;
      if (c->page_size) {
        r.page0 = (int32_t)n_page;
        n_page += (r.pos0 + r.n - 1) / 16 - r.pos0 / 16 + 1;
      }
    }
    const bool by_value = (int)runs.size() <= kAppRuns && n_page <= kAppPages && has_k && n_groups <= kGridX;
    // what needs an upload cannot be captured: its staging memory is used again
    if ((!by_value || !new_pages.empty()) && capturing(s))
      return fail(FCG_ESTATE, "this append maps pages or has too many runs to be captured into a graph");
    const RopeArgs ra = rope ? rope->args() : [&] {
      RopeArgs a{};
      a.rot = d.head_dim;
      return a;
    }();
    const bool pairs = rope && rope->pairs();
    const float2* tab = rope ? nullptr : c->d_rope;
    staged.map();
    if (by_value) {
      AppendArgs args;
      size_t np = 0;  // new_pages is sorted by (sequence, logical page)
      for (size_t i = 0; i < runs.size(); ++i) {
        AppendRun& r = runs[i];
        if (c->page_size) {
          const int32_t lp0 = r.pos0 / 16, lp1 = (r.pos0 + r.n - 1) / 16;
          std::copy(c->plan.page_row(r.seq) + lp0, c->plan.page_row(r.seq) + lp1 + 1, args.page + r.page0);
          while (np < new_pages.size() && new_pages[np] < std::pair<int32_t, int32_t>(r.seq, lp0)) ++np;
          if (np < new_pages.size() && new_pages[np] <= std::pair<int32_t, int32_t>(r.seq, lp1)) r.page0 |= INT32_MIN;
        }
        args.run[i] = r;
      }
      const int rc = launch_append(d.dtype, pairs, rows, args, (int)runs.size(), nullptr, n_groups, c->view(), layer, ra,
                                   tab, s);
      if (rc) return hip_fail((hipError_t)rc, "append launch");
      return commit();
    }
    Blob blob;
    std::vector<std::pair<int32_t, size_t>> page_rows;
    stage_pages(c, new_pages, &blob, &page_rows);
    std::vector<AppendGroup> groups;
    if (has_k)
      for (const auto& r : runs)
        for (int32_t j = 0; j < r.n; j += rows.tb) {
          AppendGroup g{r.tok0 + j, r.seq, r.pos0 + j, std::min(rows.tb, r.n - j), 0, 0, 0, 0};
          if (c->page_size) {
            g.page_a = c->plan.page_of(r.seq, g.pos0);
            g.page_b = c->plan.page_of(r.seq, g.pos0 + g.n - 1);
          }
          groups.push_back(g);
        }
    const size_t o_groups = blob.add(groups.data(), groups.size() * sizeof(AppendGroup));
    char* dplan = nullptr;
    if (fcg_status st = upload(c, blob, page_rows, s, &dplan, &staged)) return st;
    for (size_t i = 0; i < groups.size(); i += kGridX)
      if (int rc = launch_append(d.dtype, pairs, rows, AppendArgs{}, 0, (const AppendGroup*)(dplan + o_groups) + i,
                                 (int)std::min<size_t>(kGridX, groups.size() - i), c->view(), layer, ra, tab, s))
        return hip_fail((hipError_t)rc, "append launch");
    if (fcg_status st = c->ring.retire(s)) return st;
    return commit();
  });
}

// ------------------------------------------------------------ prefix attention

namespace {

struct PrefixPlan {
  std::vector<PrefixItem> items;
  std::vector<PrefixRank> ranks;
  PrefixArgs args;
  int n_items = 0, slots = 0, waves = 4;
  bool direct = false, by_value = false;
};

int64_t tiles_of(int64_t lo, int64_t hi) { return hi > lo ? (hi - 1) / kPfxTile - lo / kPfxTile + 1 : 0; }

// Consecutive tokens (in order of position) of one sequence.  Fused: they fill a
// row block by themselves, which goes over prefix and own keys in one item, so
// that nothing is merged between the two.  The others share the prefix items and
// have own items per sequence.
struct PrefixTokens {
  int32_t first, n, seq, end;  // of the sorted tokens; end: one past the last attended position
  bool fused;
};

// A block shape of the kernel: rows, blocks at once on the chip, the most rows of a
// narrow item, and what items were measured to take: us per tile with a compute unit to
// itself and beside a second block, and to begin and end; per tile of a narrow item.
struct PrefixShape {
  int rows, at_once, narrow;
  double tile_us, tile2_us, item_us, ntile_us;
};
constexpr PrefixShape kShape4{kPfxRows, 512, 32, 1.5, 2.65, 6.0, 0.45}, kShape8{2 * kPfxRows, 256, 32, 2.0, 2.0, 12.0, 0.3};
constexpr PrefixShape kShapeF32{kPfxRowsF32, 512, 16, 5.0, 9.5, 6.0, 1.0};

// Choose the split length (in tiles) of a call cut into row blocks of a shape, and
// return the estimated time (us) that the choice of shape goes by: rounds of wide items,
// the narrow ones (5 us and their tiles, no faster than 5.3 TB/s), and the merge (a round
// trip per four slots, and the partials at 4 TB/s).  Against measured times (us):
//   64 tokens over 4.3K shared keys, two row blocks of 128, per 5, 6, 8, 12, 17 tiles: 29,
//   28, 28, 32, 39 (blocks of 256 rows: 38 at best);
//   128 tokens, 8 query heads a kv head, over 22K: 140 (128-row blocks), 135 (256-row);
//   one token over 8K, per 1, 2, 4, 8, 16: 24, 17, 16, 18, 22;
//   four tokens over 8K, per 1, 2, 4, 6, 8, 16: 30, 23, 19, 17, 18, 23;
//   8 tokens over own keys of up to 4K, per 1, 3, 6, 12, 24: 35, 25, 22, 21, 27.
double cut_prefix(const fcg_model_desc& d, int32_t P, const std::vector<PrefixTokens>& toks, int n_tok,
                  const PrefixShape& shape, int64_t* per_out) {
  const int g = d.n_q_heads / d.n_kv_heads;
  const int64_t ta = tiles_of(0, P);
  // row blocks: those with keys of their own by their tiles, the shared ones and the narrow
  // items by their number (a decode step plans in a few us: no loop over its sequences per
  // candidate)
  std::vector<int32_t> wide;
  int32_t small_rows = 0, longest = 1, own_longest = 0, n_narrow = 0;
  int64_t narrow_tiles = 0;
  auto add = [&](int32_t rows, int32_t t) {
    longest = std::max(longest, t);
    if (rows > shape.narrow) {
      wide.push_back(t);
    } else if (t) {
      ++n_narrow;
      narrow_tiles += t;
    }
  };
  for (const PrefixTokens& x : toks) {
    const int32_t own = (int32_t)tiles_of(P, x.end);
    if (!x.fused) {
      small_rows += x.n * g;
      own_longest = std::max(own_longest, own);
    }
    add(x.n * g, own + (x.fused ? (int32_t)ta : 0));
  }
  int32_t n_shared = 0;
  if (small_rows > shape.narrow && ta) {
    n_shared = (small_rows + shape.rows - 1) / shape.rows;
    longest = std::max(longest, (int32_t)ta);
  } else if (small_rows) {
    add(small_rows, (int32_t)ta);
  }
  const double es = d.dtype == FCG_F32 ? 4.0 : 2.0;
  const double slot_us = (double)n_tok * d.n_q_heads * d.head_dim * es * 2.0 / 4e6;
  const double read_us = (double)narrow_tiles * kPfxTile * d.n_kv_heads * d.head_dim * es * 2.0 / 5.3e6;
  double best = 1e30;
  // at most 64 splits: slots are counted in 16 bits, and the merge reads them all
  for (int32_t ns : {1, 2, 3, 4, 5, 6, 8, 10, 12, 14, 16, 20, 24, 32, 40, 48, 64}) {
    if (ns > longest) break;
    const int32_t per = (longest + ns - 1) / ns;
    int64_t blocks = (int64_t)n_shared * ((ta + per - 1) / per);
    for (int32_t t : wide) blocks += (t + per - 1) / per;
    blocks *= d.n_kv_heads;
    const double nblocks = d.n_kv_heads * std::max((double)n_narrow, (double)narrow_tiles / per + 0.5 * n_narrow);
    double us = std::ceil((double)blocks / shape.at_once) *
                (per * (blocks <= 256 ? shape.tile_us : shape.tile2_us) + shape.item_us);
    if (n_narrow) {
      const double rounds = blocks ? nblocks / shape.at_once : std::ceil(nblocks / shape.at_once);
      us += std::max(rounds * (5.0 + shape.ntile_us * std::min<double>(per, (double)narrow_tiles / n_narrow)), read_us);
    }
    const int64_t slots = small_rows ? (ta + per - 1) / per + (own_longest + per - 1) / per : (longest + per - 1) / per;
    if (slots > 1) us += 3.0 + slots * (0.1 + slot_us);
    if (us < best) {
      best = us;
      *per_out = per;
    }
  }
  return best;
}

std::vector<PrefixTokens> group_tokens(int g, int32_t n, const std::vector<int32_t>& order, const int32_t* seq,
                                       const int32_t* pos, int block) {
  std::vector<PrefixTokens> out, fused;
  const int32_t per = block / g;  // tokens of a full row block
  for (int32_t i = 0; i < n;) {
    int32_t j = i;
    while (j < n && seq[order[j]] == seq[order[i]]) ++j;
    while (i < j) {
      const bool full = j - i >= per || (int64_t)(j - i) * g * 4 >= 3 * block;
      const int32_t m = full ? std::min(per, j - i) : j - i;
      (full ? fused : out).push_back(PrefixTokens{i, m, seq[order[i]], pos[order[i + m - 1]] + 1, full});
      i += m;
    }
  }
  // own items that start last should be the short ones: longest first
  std::stable_sort(out.begin(), out.end(), [](const PrefixTokens& a, const PrefixTokens& b) { return a.end > b.end; });
  out.insert(out.end(), fused.begin(), fused.end());  // ranks of the shared row blocks come first
  return out;
}

void plan_prefix(const fcg_model_desc& d, int32_t P, int32_t n, const int32_t* seq, const int32_t* pos, PrefixPlan* p) {
  const int g = d.n_q_heads / d.n_kv_heads;
  std::vector<int32_t> order(n);
  for (int32_t t = 0; t < n; ++t) order[t] = t;
  auto less = [&](int32_t a, int32_t b) { return seq[a] != seq[b] ? seq[a] < seq[b] : pos[a] < pos[b]; };
  if (!std::is_sorted(order.begin(), order.end(), less)) std::stable_sort(order.begin(), order.end(), less);
  const PrefixShape& small_shape = d.dtype == FCG_F32 ? kShapeF32 : kShape4;
  int block = small_shape.rows;
  std::vector<PrefixTokens> toks = group_tokens(g, n, order, seq, pos, block);
  int64_t per = 1;
  const double us = cut_prefix(d, P, toks, n, small_shape, &per);
  if (d.dtype == FCG_BF16 && (int64_t)n * g > kPfxRows) {
    std::vector<PrefixTokens> toks8 = group_tokens(g, n, order, seq, pos, kShape8.rows);
    int64_t per8 = 1;
    if (cut_prefix(d, P, toks8, n, kShape8, &per8) < us) {
      p->waves = 8;
      block = kShape8.rows;
      toks = std::move(toks8);
      per = per8;
    }
  }
  const int64_t ta = tiles_of(0, P), t0 = P / kPfxTile;
  p->ranks.reserve(n);
  int32_t small_rows = 0, n_small = 0, n_own = 0;
  std::vector<int32_t> rank0;
  for (const PrefixTokens& x : toks) {
    rank0.push_back((int32_t)p->ranks.size());
    for (int32_t i = 0; i < x.n; ++i)
      p->ranks.push_back(PrefixRank{order[x.first + i], pos[order[x.first + i]], 0, 0, 0, 0});
    if (!x.fused) {
      small_rows += x.n * g;
      ++n_small;
    }
  }
  const int pre_slots = small_rows && P ? (int)((ta + per - 1) / per) : 0;
  const int n_pre = (small_rows + block - 1) / block * pre_slots;
  p->slots = pre_slots;
  auto own_splits = [&](const PrefixTokens& x) { return (int)((tiles_of(P, x.end) + per - 1) / per); };
  p->by_value = n_small == (int)toks.size() && n_small <= kPfxGroups && n <= kPfxRanks;
  if (p->by_value) {
    PrefixArgs& a = p->args;
    a.n_pre = n_pre;
    a.pre_slots = pre_slots;
    a.pre_rows = small_rows;
    a.block = block;
    a.per = (int32_t)(per * kPfxTile);
    a.prefix_len = P;
    a.n_group = n_small;
  }
  for (size_t gi = 0; gi < toks.size(); ++gi) {
    const PrefixTokens& x = toks[gi];
    if (x.fused) break;
    const int ns = own_splits(x);
    for (int32_t i = 0; i < x.n; ++i) {
      PrefixRank& r = p->ranks[rank0[gi] + i];
      r.na = (uint16_t)pre_slots;
      r.b0 = (uint16_t)pre_slots;
      r.nb = (uint16_t)ns;
      if (p->by_value) p->args.rank[rank0[gi] + i] = PrefixSmall{r.pos, (uint16_t)r.tok, (uint16_t)ns};
    }
    if (p->by_value) p->args.group[gi] = PrefixGroup{x.seq, x.end, rank0[gi] * g | x.n * g << 16, n_own};
    n_own += ns;
    p->slots = std::max(p->slots, pre_slots + ns);
  }
  p->n_items = n_pre + n_own;
  if (p->by_value) {
    // Two own items a block, if they are narrow and the blocks then take fewer rounds: an
    // item's time is mostly its chain of round trips (page entries, first tile, partials),
    // which two in a block share (64 tokens over 4.3K, 224 prefix blocks and 544 own items on
    // 512 places: 24.5 us, paired 22.7).
    const PrefixShape& shape = d.dtype == FCG_F32 ? kShapeF32 : p->waves == 8 ? kShape8 : kShape4;
    bool pair = d.dtype == FCG_BF16;
    for (const PrefixTokens& x : toks) pair = pair && x.n * g <= shape.narrow;
    const int halved = n_pre + (n_own + 1) / 2;
    auto rounds = [&](int items) { return (items * d.n_kv_heads + shape.at_once - 1) / shape.at_once; };
    pair = pair && rounds(halved) < rounds(p->n_items);
    p->args.paired = pair ? n_own : 0;
    if (pair) p->n_items = halved;
  }
  if (!p->by_value) {
    for (int32_t r0 = 0; r0 < small_rows && pre_slots; r0 += block)
      for (int s = 0; s < pre_slots; ++s)
        p->items.push_back(PrefixItem{r0, std::min(block, small_rows - r0), 0, (int32_t)(s * per * kPfxTile),
                                      (int32_t)std::min<int64_t>(P, (s + 1) * per * kPfxTile), 0, 0, s});
    for (size_t gi = 0; gi < toks.size(); ++gi) {
      const PrefixTokens& x = toks[gi];
      const int32_t row0 = rank0[gi] * g, rows = x.n * g;
      if (!x.fused) {
        const int ns = own_splits(x);
        for (int s = 0; s < ns; ++s) {  // own positions, cut at multiples of a tile
          const int64_t cut = (t0 + s * per) * kPfxTile;
          p->items.push_back(PrefixItem{row0, rows, x.seq, 0, 0, (int32_t)std::max<int64_t>(P, cut),
                                        (int32_t)std::min<int64_t>(x.end, cut + per * kPfxTile), pre_slots + s});
        }
        continue;
      }
      // prefix tiles, then own tiles: one run of tiles, cut every `per`
      const int64_t tb = tiles_of(P, x.end);
      const int ns = (int)((ta + tb + per - 1) / per);
      for (int s = 0; s < ns; ++s) {
        const int64_t a = s * per, b = std::min(ta + tb, (s + 1) * per);
        PrefixItem it{row0, rows, x.seq, 0, 0, 0, 0, s};
        if (a < ta) {
          it.a0 = (int32_t)(a * kPfxTile);
          it.a1 = (int32_t)std::min<int64_t>(P, std::min(b, ta) * kPfxTile);
        }
        if (b > ta) {
          it.b0 = (int32_t)std::max<int64_t>(P, (t0 + std::max<int64_t>(a - ta, 0)) * kPfxTile);
          it.b1 = (int32_t)std::min<int64_t>(x.end, (t0 + b - ta) * kPfxTile);
        }
        p->items.push_back(it);
      }
      for (int32_t i = 0; i < x.n; ++i) p->ranks[rank0[gi] + i].na = (uint16_t)ns;
      p->slots = std::max(p->slots, ns);
    }
    p->n_items = (int)p->items.size();
  }
  p->direct = n > 0;
  for (const PrefixRank& r : p->ranks) p->direct = p->direct && r.na + r.nb == 1;
}

// The workspace of prefix partials.  One that a captured graph uses is kept until
// the cache is destroyed when a larger one takes its place.
fcg_status prefix_workspace(fcg_cache* c, size_t bytes, bool cap) {
  if (bytes > c->xpart_bytes) {
    if (cap) return fail(FCG_ESTATE, "fcg_prefix_attend needs a larger workspace: run a call of this size before the capture");
    if (c->xpart_captured) {
      c->xkept.push_back(c->xpart);
      c->xpart = nullptr;
      c->xpart_bytes = 0;
      c->xpart_captured = false;
    }
    if (fcg_status st = grow(&c->xpart, &c->xpart_bytes, bytes, "prefix partials")) return st;
  }
  if (cap) c->xpart_captured = true;
  return FCG_OK;
}

}  // namespace

fcg_status fcg_prefix_attend(fcg_cache* c, int32_t layer, int32_t prefix_seq, int32_t prefix_len, int32_t n_tok,
                             const int32_t* seq, const int32_t* pos, const fcg_tensor* q, const fcg_tensor* out,
                             float* lse, void* stream) {
  if (!c) return fail(FCG_EINVAL, "null cache");
  if (n_tok < 0) return fail(FCG_EINVAL, "negative token count");
  if (n_tok > 0 && (!seq || !pos)) return fail(FCG_EINVAL, "null token array");
  const fcg_model_desc& d = c->desc;
  if (n_tok > 0 && !c->layout_only()) {
    if (!q || !out || !q->data || !out->data) return fail(FCG_EINVAL, "null tensor");
    if (fcg_status st = check_strides(q, "q")) return st;
    if (fcg_status st = check_strides(out, "out")) return st;
    if (fcg_status st = check_output(out, 1, n_tok, d.n_q_heads, d.head_dim, "out")) return st;
    fcg_tensor a = *q, b = *out;
    a.layer = b.layer = 0;
    if (fcg_status st = check_alias(&a, &b, "out")) return st;
  }
  if (n_tok > kGridX) return fail(FCG_EINVAL, "more than 2^24 - 1 tokens");
  if ((int64_t)n_tok * d.n_q_heads > 1 << 30) return fail(FCG_EINVAL, "more than 2^30 query rows");
  return guarded([&]() -> fcg_status {
    std::string msg;
    if (fcg_status st = c->plan.check_attend(layer, prefix_seq, prefix_len, n_tok, seq, pos, &msg)) return fail(st, msg);
    if (n_tok == 0 || c->layout_only()) return FCG_OK;
    OnDevice dev(c->device);
    HIP_TRY(dev.err, "hipSetDevice");
    hipStream_t s = (hipStream_t)stream;
    PrefixPlan p;
    plan_prefix(d, prefix_len, n_tok, seq, pos, &p);
    const int g = d.n_q_heads / d.n_kv_heads;
    const size_t prow = (size_t)p.slots * d.n_kv_heads * n_tok * g;
    const size_t o_bytes = (prow * d.head_dim * esize(d.dtype) + 255) & ~size_t(255);
    const bool merge = !p.direct, work = merge && p.slots;
    const bool cap = (work || !p.by_value) && capturing(s);
    // what needs an upload cannot be captured: its staging memory is used again
    if (cap && !p.by_value) return fail(FCG_ESTATE, "this prefix attention has too many tokens to be captured into a graph");
    if (work)
      if (fcg_status st = prefix_workspace(c, o_bytes + prow * 16, cap)) return st;
    PrefixCall pc{};
    pc.q = view_of(q);
    pc.out = view_of(out);
    pc.lse = lse;
    pc.part_o = c->xpart;
    pc.part_ml = (float*)((char*)c->xpart + o_bytes);
    pc.rows = n_tok * g;
    pc.g = g;
    pc.prefix_seq = prefix_seq;
    pc.layer = layer;
    pc.direct = p.direct;
    const PrefixItem* items = nullptr;
    const PrefixRank* ranks = nullptr;
    if (!p.by_value) {
      Blob blob;
      const size_t o_items = blob.add(p.items.data(), p.items.size() * sizeof(PrefixItem));
      const size_t o_ranks = blob.add(p.ranks.data(), p.ranks.size() * sizeof(PrefixRank));
      char* dplan = nullptr;
      if (fcg_status st = upload(c, blob, {}, s, &dplan, nullptr)) return st;
      items = (const PrefixItem*)(dplan + o_items);
      ranks = (const PrefixRank*)(dplan + o_ranks);
    }
    const PrefixArgs* args = p.by_value ? &p.args : nullptr;
    constexpr int kGridY = 65535;
    for (int i0 = 0; i0 < p.n_items; i0 += kGridY)  // more only from plans in memory
      if (int rc = launch_prefix_attend(d.dtype, pc, args, items + (args ? 0 : i0), ranks, std::min(kGridY, p.n_items - i0),
                                        p.waves, c->view(), s))
        return hip_fail((hipError_t)rc, "prefix attention launch");
    if (merge)
      if (int rc = launch_prefix_merge(d.dtype, pc, args, ranks, n_tok, d.n_q_heads, d.head_dim, s))
        return hip_fail((hipError_t)rc, "prefix merge launch");
    return p.by_value ? FCG_OK : c->ring.retire(s);
  });
}

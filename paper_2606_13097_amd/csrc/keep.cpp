// Entry points of what a cache keeps of its positions (include/fcg.h): the attention
// weight they receive, and eviction by it.
#include <algorithm>

#include "objects.hpp"
#include "ops.hpp"

using namespace fcg;

// ------------------------------------------------- attention weight per position

namespace {

constexpr int kGridY = 65535;

struct WeightPlan {
  std::vector<WeightItem> items;
  std::vector<WeightRank> ranks;
  WeightArgs args;
  int n_items = 0, n_kb = 0, splits = 1, block = 128;
  bool by_value = false;
};

// Blocks of 256 keys (the rows are read half as often from LDS) where the work is enough
// for four times the blocks that are resident at once, else of 128.  The rows of a block
// of keys are cut into splits where that makes twice the resident blocks of like work, of
// 4 tiles of 64 rows at least: a split costs a partial, and a call with any a second launch.
// (us a call: 32 sequences of 64 tokens past a prefix of 6007, 256 keys 139, 128 keys 152; one
// token each of 64 sequences, prefix 4321, 128 keys 12.0, 256 keys 13.9.)
constexpr int64_t kResident = 512;
void plan_weights(const fcg_model_desc& d, int32_t prefix_seq, int32_t P, int32_t n, const int32_t* seq,
                  const int32_t* pos, WeightPlan* p) {
  const int g = d.n_q_heads / d.n_kv_heads;
  std::vector<int32_t> order(n);
  for (int32_t t = 0; t < n; ++t) order[t] = t;
  auto less = [&](int32_t a, int32_t b) { return seq[a] != seq[b] ? seq[a] < seq[b] : pos[a] < pos[b]; };
  if (!std::is_sorted(order.begin(), order.end(), less)) std::stable_sort(order.begin(), order.end(), less);
  p->ranks.reserve(n);
  std::vector<WeightGroup> groups;
  if (P && n) groups.push_back(WeightGroup{prefix_seq, 0, P, 0, n * g, 0, 0});
  for (int32_t i = 0; i < n;) {
    int32_t j = i;
    for (; j < n && seq[order[j]] == seq[order[i]]; ++j) p->ranks.push_back(WeightRank{order[j], pos[order[j]]});
    const int32_t end = pos[order[j - 1]] + 1;
    if (end > P) groups.push_back(WeightGroup{seq[order[i]], P, end, i * g, (j - i) * g, 0, 0});
    i = j;
  }
  // tiles of 64 rows past a block of keys, over all kv heads
  auto work = [&](int64_t len) {
    int64_t tiles = 0;
    for (const WeightGroup& x : groups) tiles += (x.hi - x.lo + len - 1) / len * ((x.rows + 63) / 64);
    return tiles * d.n_kv_heads;
  };
  p->block = weights_most_keys(esize(d.dtype), d.head_dim);
  if (work(p->block) < 8 * kResident) p->block = 128;
  // (at most the 2^30 rows that a call has)
  const int64_t split_tiles = std::max<int64_t>(4, (work(p->block) + 2 * kResident - 1) / (2 * kResident));
  const int32_t split_rows = (int32_t)std::min<int64_t>(split_tiles, 1 << 24) * 64;
  const int pre = P && n ? 1 : 0;  // the first group is the prefix
  int64_t all = 0;
  for (const WeightGroup& x : groups)
    all += (int64_t)((x.hi - x.lo + p->block - 1) / p->block) * ((x.rows + split_rows - 1) / split_rows);
  p->by_value = (int)groups.size() - pre <= kWgtGroups && n <= kWgtRanks && all <= kGridY;
  WeightArgs& a = p->args;
  if (p->by_value) {
    a.n_group = (int)groups.size() - pre;
    a.block = p->block;
    a.split_rows = split_rows;
    a.n_pre = 0;
    std::copy(p->ranks.begin(), p->ranks.end(), a.rank);
  }
  for (size_t i = 0; i < groups.size(); ++i) {
    WeightGroup& x = groups[i];
    const int32_t nkb = (x.hi - x.lo + p->block - 1) / p->block;
    x.kb0 = p->n_kb;
    x.item0 = p->n_items;
    p->n_kb += nkb;
    if (p->by_value) {
      const int32_t ns = (x.rows + split_rows - 1) / split_rows;
      p->n_items += nkb * ns;
      p->splits = std::max(p->splits, ns);
      if ((int)i < pre) {
        a.pre = x;
        a.n_pre = p->n_items;
      } else {
        a.group[i - pre] = x;
      }
      continue;
    }
    int32_t r = x.row0 / g;
    const int32_t r1 = r + x.rows / g;
    for (int32_t kb = 0; kb < nkb; ++kb) {
      WeightItem it{x.seq, x.lo + kb * p->block, 0, 0, 0, x.kb0 + kb, 0, 0};
      it.k1 = std::min(x.hi, it.k0 + p->block);
      // own keys: from the first row that sees one of them (rows of several sequences,
      // before the shared prefix, all see all)
      if (x.lo >= P)
        while (r < r1 && p->ranks[r].pos < it.k0) ++r;
      const int32_t left = (r1 - r) * g;
      it.n_split = (left + split_rows - 1) / split_rows;
      p->splits = std::max(p->splits, it.n_split);
      for (; it.split < it.n_split; ++it.split) {
        it.row0 = r * g + it.split * split_rows;
        it.n_row = std::min(split_rows, left - it.split * split_rows);
        p->items.push_back(it);
      }
    }
  }
  if (!p->by_value) p->n_items = (int)p->items.size();
}

}  // namespace

fcg_status fcg_attend_weights(fcg_cache* c, int32_t layer, int32_t prefix_seq, int32_t prefix_len, int32_t n_tok,
                              const int32_t* seq, const int32_t* pos, const fcg_tensor* q, const float* lse,
                              float* weights, uint32_t flags, void* stream) {
  if (!c) return fail(FCG_EINVAL, "null cache");
  if (n_tok < 0) return fail(FCG_EINVAL, "negative token count");
  if (n_tok > 0 && (!seq || !pos)) return fail(FCG_EINVAL, "null token array");
  if (flags & ~FCG_ADD) return fail(FCG_EINVAL, "unknown flags");
  const fcg_model_desc& d = c->desc;
  if (n_tok > 0 && !c->layout_only()) {
    if (!q || !q->data || !lse || !weights) return fail(FCG_EINVAL, "null tensor");
    if (fcg_status st = check_strides(q, "q")) return st;
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
    WeightPlan p;
    plan_weights(d, prefix_seq, prefix_len, n_tok, seq, pos, &p);
    if (!p.n_items) return FCG_OK;  // no token has a key
    const bool split = p.splits > 1;
    const bool cap = (split || !p.by_value) && capturing(s);
    // what needs an upload cannot be captured: its staging memory is used again
    if (cap && !p.by_value) return fail(FCG_ESTATE, "this call has too many tokens or sequences to be captured into a graph");
    if (split)
      if (fcg_status st = prefix_workspace(c, (size_t)p.splits * p.n_kb * d.n_kv_heads * p.block * 4, cap, "fcg_attend_weights"))
        return st;
    WeightCall wc{};
    wc.q = view_of(q);
    wc.lse = lse;
    wc.weights = weights;
    wc.part = split ? (float*)c->xpart : nullptr;
    wc.n_q_heads = d.n_q_heads;
    while ((d.n_kv_heads << wc.g_shift) < d.n_q_heads) ++wc.g_shift;
    wc.layer = layer;
    wc.n_kb = p.n_kb;
    wc.add = (flags & FCG_ADD) != 0;
    const WeightItem* items = nullptr;
    const WeightRank* ranks = nullptr;
    if (!p.by_value) {
      Blob blob;
      const size_t o_items = blob.add(p.items.data(), p.items.size() * sizeof(WeightItem));
      const size_t o_ranks = blob.add(p.ranks.data(), p.ranks.size() * sizeof(WeightRank));
      char* dplan = nullptr;
      if (fcg_status st = upload(c, blob, {}, s, &dplan, nullptr)) return st;
      items = (const WeightItem*)(dplan + o_items);
      ranks = (const WeightRank*)(dplan + o_ranks);
    }
    for (int i0 = 0; i0 < p.n_items;) {
      int i1 = std::min(kGridY, p.n_items - i0) + i0;
      // each launch adds up the splits of its blocks of keys: it ends between two blocks
      // (which have at most 2 kResident splits; a plan by value is one launch)
      if (i1 < p.n_items)
        while (p.items[i1].split) --i1;
      if (int rc = launch_attend_weights(d.dtype, wc, p.by_value ? &p.args : nullptr, items ? items + i0 : nullptr, ranks,
                                         i1 - i0, p.block, c->view(), s))
        return hip_fail((hipError_t)rc, "attention weights launch");
      i0 = i1;
    }
    return p.by_value ? FCG_OK : c->ring.retire(s);
  });
}

// -------------------------------------------------------------------- eviction

fcg_status fcg_evict(fcg_cache* c, int32_t n_items, const int32_t* src, const int32_t* dst, const int32_t* keep,
                     int32_t n_first, int32_t n_recent, const fcg_rope* rope, float* weights, int32_t* kept, void* stream) {
  if (!c) return fail(FCG_EINVAL, "null cache");
  if (n_items < 0 || n_first < 0 || n_recent < 0) return fail(FCG_EINVAL, "negative count");
  if (n_items > 0 && (!src || !dst || !keep)) return fail(FCG_EINVAL, "null item array");
  const fcg_model_desc& d = c->desc;
  if (rope && rope->rot > d.head_dim) return fail(FCG_EINVAL, "rotary_dim exceeds head_dim");
  if (n_items > 0 && !c->layout_only() && !weights) return fail(FCG_EINVAL, "null weights");
  // (a selection block for each layer and kv head of an item, of at most 1024 threads)
  if ((int64_t)d.n_kv_heads * 2 > kGridY || (int64_t)d.n_kv_heads * d.n_layers > 1 << 20)
    return fail(FCG_EINVAL, "too many layers or kv heads");
  return guarded([&]() -> fcg_status {
    std::string msg;
    std::vector<int32_t> len;
    std::vector<std::pair<int32_t, int32_t>> new_pages;
    if (fcg_status st = c->plan.check_evict(n_items, src, dst, keep, &len, &new_pages, &msg)) return fail(st, msg);
    if (n_items == 0) return FCG_OK;
    auto stays = [&](int32_t i) { return std::min(keep[i], len[i]); };
    auto cut = [&](int32_t i0, int32_t i1) {  // in place
      for (int32_t i = i0; i < i1; ++i)
        if (src[i] == dst[i]) c->plan.truncate(dst[i], stays(i));
    };
    auto fill_targets = [&]() {
      for (int32_t i = 0; i < n_items; ++i)
        if (src[i] != dst[i]) c->plan.mark_all_layers(dst[i], 0, stays(i));
      return FCG_OK;
    };
    auto empty_targets = [&]() {
      for (int32_t i = 0; i < n_items; ++i)
        if (src[i] != dst[i]) (void)fcg_cache_reset(c, dst[i]);
    };
    if (c->layout_only()) {
      empty_targets();
      c->plan.map_pages(new_pages);
      cut(0, n_items);
      return fill_targets();
    }
    OnDevice dev(c->device);
    HIP_TRY(dev.err, "hipSetDevice");
    hipStream_t s = (hipStream_t)stream;
    int32_t most = 0, far = 0;  // positions kept, the furthest that a row moves
    for (int32_t i = 0; i < n_items; ++i) {
      most = std::max(most, keep[i]);
      far = std::max(far, len[i] - stays(i));
    }
    RopeArgs ra{};
    if (rope) ra = rope->args();
    else ra.rot = d.head_dim;
    const int half = ra.rot / 2;
    const size_t kept_bytes = kept ? 0 : ((size_t)d.n_layers * n_items * d.n_kv_heads * most * 4 + 255) & ~size_t(255);
    const size_t turn_bytes = rope ? ((size_t)far + 1) * half * sizeof(float2) : 0;
    const bool cap = capturing(s);
    // what needs an upload cannot be captured: its staging memory is used again
    if (cap && !new_pages.empty()) return fail(FCG_ESTATE, "this eviction maps pages: it cannot be captured into a graph");
    if (kept_bytes + turn_bytes)
      if (fcg_status st = prefix_workspace(c, kept_bytes + turn_bytes, cap, "fcg_evict")) return st;
    EvictCall ec{};
    ec.weights = weights;
    ec.kept = kept ? kept : (int32_t*)c->xpart;
    ec.turns = rope ? (float2*)((char*)c->xpart + kept_bytes) : c->d_rope;
    ec.kept_stride = most;
    ec.n_items = n_items;
    ec.first = n_first;
    ec.recent = n_recent;
    // What takes much memory comes before the targets are emptied: room for their page rows,
    // which are filled in once the pages are mapped.
    Blob blob;
    std::vector<std::pair<int32_t, size_t>> rows;
    const size_t row_bytes = 2 * sizeof(int32_t) * c->plan.n_logical_pages();
    for (const auto& page : new_pages)  // (in order of the targets)
      if (rows.empty() || rows.back().first != page.first)
        rows.push_back({page.first, rows.size() * ((row_bytes + 255) & ~size_t(255))});
    if (!rows.empty()) {
      blob.bytes.resize(rows.back().second + row_bytes);
      if (fcg_status st = c->ring.reserve(blob.bytes.size() + 512)) return st;
    }
    empty_targets();
    c->plan.map_pages(new_pages);
    auto undo = [&](fcg_status st) {
      empty_targets();
      return st;
    };
    if (!rows.empty()) {
      for (const auto& r : rows) {
        std::memcpy(blob.bytes.data() + r.second, c->plan.page_row(r.first), row_bytes / 2);
        std::memcpy(blob.bytes.data() + r.second + row_bytes / 2, c->plan.alias_row(r.first), row_bytes / 2);
      }
      char* at = nullptr;
      fcg_status st;
      try {
        st = upload(c, blob, rows, s, &at, nullptr);
        if (!st) st = c->ring.retire(s);
      } catch (...) {  // (the list of staged regions grows)
        empty_targets();
        throw;
      }
      if (st) return undo(st);
    }
    // launches of up to kEvictItems items, those into other sequences and those in place
    bool table = rope != nullptr;
    for (int in_place = 0; in_place < 2; ++in_place)
      for (int32_t i = 0; i < n_items;) {
        EvictArgs args;
        args.n = 0;
        int64_t chunks = 0, rows_of = 0;
        ec.item0 = i;
        for (; i < n_items && args.n < kEvictItems; ++i) {
          // items of one launch are neighbours in the call: `kept` counts them on
          if ((src[i] == dst[i]) != (in_place == 1)) {
            if (args.n) break;
            ec.item0 = i + 1;
            continue;
          }
          const int64_t more = (stays(i) + kEvictRows - 1) / kEvictRows;
          rows_of += (int64_t)d.n_kv_heads * d.n_layers;
          if (args.n && (chunks + more > kGridX || rows_of > 1 << 20)) break;
          args.item[args.n++] = EvictItem{src[i], dst[i], len[i], stays(i), (int32_t)chunks};
          chunks += more;
        }
        if (!args.n) break;
        if (int rc = launch_evict_select(ec, args, ra, d.n_layers, c->n_seqs, d.n_kv_heads, c->max_tokens,
                                         table ? far + 1 : 0, s))
          return undo(hip_fail((hipError_t)rc, "eviction launch"));
        table = false;
        if (chunks)
          if (int rc = launch_evict_move(d.dtype, rope && rope->pairs(), in_place == 1, ec, args, (int)chunks, c->view(),
                                         half, d.n_layers, s))
            return undo(hip_fail((hipError_t)rc, "eviction launch"));
        // (at once: should a later launch fail, the length goes with the rows)
        if (in_place) cut(ec.item0, ec.item0 + args.n);
      }
    return fill_targets();
  });
}

// Calls that map pages, with every allocation and every HIP call of theirs made to
// fail in turn: a failed call leaves the layout as it was, the same call succeeds
// afterwards, and the device page table then holds every page the host has mapped.
#include "host_runtime.hpp"

#include <functional>
#include <numeric>

namespace {

int failures = 0;
#define CHECK(cond, ...)                                   \
  do {                                                     \
    if (!(cond)) {                                         \
      std::printf("FAILED %s:%d: ", __FILE__, __LINE__);   \
      std::printf(__VA_ARGS__);                            \
      std::printf(" (%s)\n", #cond);                       \
      ++failures;                                          \
    }                                                      \
  } while (0)

constexpr int L = 2, HQ = 4, HKV = 2, D = 64, SEQS = 70, TOKENS = 160;

fcg_model_desc desc(int32_t dtype) { return fcg_model_desc{L, HQ, HKV, D, 1e4, dtype, 0}; }

struct World {
  fcg_lib* lib = nullptr;
  fcg_cache* cache = nullptr;
  std::vector<float> data = std::vector<float>((size_t)L * SEQS * TOKENS * HQ * D / 8);
  World(int32_t dtype, int page, uint32_t flags) {
    const fcg_model_desc d = desc(dtype);
    if (fcg_lib_create(&d, 400, 4, 0, &lib) || fcg_cache_create(&d, SEQS, TOKENS, page, 500, flags, &cache)) std::abort();
    int32_t id;
    for (int len : {100, 40, 16}) fcg_lib_add_segment(lib, len, 0, data.data(), data.data(), nullptr, &id);
  }
  ~World() {
    fcg_cache_destroy(cache);
    fcg_lib_destroy(lib);
  }
  fcg_tensor rows(int heads) { return fcg_tensor{data.data(), (int64_t)SEQS * heads * D, heads * D, D}; }
};

struct Layout {
  std::vector<int32_t> pages, alias, lens;
  std::vector<uint8_t> written;
  std::vector<int32_t> pins;
  bool operator==(const Layout& o) const {
    return pages == o.pages && alias == o.alias && lens == o.lens && written == o.written && pins == o.pins;
  }
};

Layout layout_of(const World& w) {
  Layout a;
  const int nlp = w.cache->plan.n_logical_pages();
  for (int s = 0; s < SEQS; ++s)
    for (int l = 0; l < L; ++l) {
      std::vector<int32_t> p(std::max(nlp, 1)), v(std::max(nlp, 1));
      std::vector<uint8_t> wr(TOKENS);
      int32_t n;
      fcg_cache_export_layout(w.cache, s, l, p.data(), &n, wr.data());
      fcg_cache_export_v_alias(w.cache, s, v.data());
      a.pages.insert(a.pages.end(), p.begin(), p.end());
      a.alias.insert(a.alias.end(), v.begin(), v.end());
      a.lens.push_back(n);
      a.written.insert(a.written.end(), wr.begin(), wr.end());
    }
  for (const Segment& s : w.lib->segs) a.pins.push_back(s.pins);
  return a;
}

// every page the host has mapped is in the device table, with the same place for its values
bool table_agrees(const World& w) {
  const fcg_cache* c = w.cache;
  const int nlp = c->plan.n_logical_pages();
  for (int s = 0; s < SEQS; ++s)
    for (int p = 0; p < nlp; ++p) {
      const int32_t* row = c->d_page_table + (int64_t)s * 2 * nlp;
      if (c->plan.page_row(s)[p] < 0) continue;
      if (row[p] != c->plan.page_row(s)[p] || row[nlp + p] != c->plan.alias_row(s)[p]) {
        std::printf("  sequence %d page %d: device %d / %d, host %d / %d\n", s, p, row[p], row[nlp + p],
                    c->plan.page_row(s)[p], c->plan.alias_row(s)[p]);
        return false;
      }
    }
  return true;
}

using Call = std::function<fcg_status(World&)>;

void every_failure(const char* name, int32_t dtype, int page, uint32_t flags, const Call& before, const Call& call,
                   const Call& after = nullptr) {
  for (bool hip : {false, true}) {
    int n = 0;
    for (;; ++n) {
      World w(dtype, page, flags);
      if (before) CHECK(before(w) == FCG_OK, "%s: the calls before", name);
      const Layout was = layout_of(w);
      const fcg_lib* bound = w.cache->alias_lib;
      (hip ? host::fail_hip : host::fail_alloc) = n;
      const fcg_status st = call(w);
      const bool reached = (hip ? host::fail_hip : host::fail_alloc) < 0;
      host::fail_hip = host::fail_alloc = -1;
      const char* kind = hip ? "HIP call" : "allocation";
      if (!reached) {
        CHECK(st == FCG_OK, "%s: status %d although nothing failed", name, st);
        break;
      }
      if (st != FCG_OK) {
        CHECK(hip ? st == FCG_EHIP || st == FCG_ENOMEM : st == FCG_ENOMEM, "%s, %s %d: status %d", name, kind, n, st);
        // a failure of the runtime may give back pages that hold nothing; nothing else may change
        Layout now = layout_of(w);
        if (hip)
          for (size_t i = 0; i < now.pages.size(); ++i)
            if (now.pages[i] < 0) now.pages[i] = was.pages[i];
        CHECK(now == was, "%s, %s %d: the layout changed", name, kind, n);
        CHECK(w.cache->alias_lib == bound, "%s, %s %d: bound to a library", name, kind, n);
        CHECK(call(w) == FCG_OK, "%s, %s %d: the call again: %s", name, kind, n, fcg_last_error());
      }
      CHECK(table_agrees(w), "%s, %s %d: the device page table", name, kind, n);
      if (after) {
        CHECK(after(w) == FCG_OK, "%s, %s %d: the call after: %s", name, kind, n, fcg_last_error());
        CHECK(table_agrees(w), "%s, %s %d: the device page table after", name, kind, n);
      }
      if (failures > 20) return;
    }
    CHECK(n > 0, "%s: nothing could fail", name);
    std::printf("%s: %d %s\n", name, n, hip ? "HIP calls" : "allocations");
  }
}

std::vector<int32_t> iota(int n, int from = 0, int step = 1) {
  std::vector<int32_t> v(n);
  for (int i = 0; i < n; ++i) v[i] = from + i * step;
  return v;
}

Call append(std::vector<int32_t> seq, std::vector<int32_t> pos, bool data, uint32_t flags = 0) {
  return [=](World& w) {
    const fcg_tensor q = w.rows(HQ), kv = w.rows(HKV);
    return fcg_append(w.cache, 0, L, (int)seq.size(), seq.data(), pos.data(), nullptr, data ? &q : nullptr,
                      data ? &q : nullptr, data ? &kv : nullptr, data ? &kv : nullptr, flags, nullptr);
  };
}

Call graft(std::vector<int32_t> seq, std::vector<int32_t> seg, std::vector<int32_t> dst) {
  return [=](World& w) {
    return fcg_graft(w.cache, w.lib, (int)seq.size(), seq.data(), seg.data(), dst.data(), nullptr);
  };
}

Call prefill(std::vector<int32_t> seq, std::vector<int32_t> pos) {
  return [=](World& w) {
    return fcg_patch_prefill(w.cache, 0, (int)seq.size(), seq.data(), pos.data(), w.data.data(), w.data.data(),
                             w.data.data(), w.data.data(), nullptr);
  };
}

Call decode(std::vector<int32_t> seq, bool noalloc) {
  return [=](World& w) {
    float* x = w.data.data();
    return (noalloc ? fcg_decode_noalloc : fcg_decode)(w.cache, 0, (int)seq.size(), seq.data(), x, x, x, x, nullptr, nullptr);
  };
}

// calls without a layout to compare: a failed allocation is a status, not an exception
void entry_points_return_a_status() {
  const fcg_model_desc d = desc(FCG_BF16);
  auto each = [](const char* name, const std::function<fcg_status()>& call) {
    for (int n = 0; n < 1000; ++n) {
      host::fail_alloc = n;
      const fcg_status st = call();
      const bool reached = host::fail_alloc < 0;
      host::fail_alloc = -1;
      // (a sort does without the room it would like)
      CHECK(st == FCG_OK || (reached && st == FCG_ENOMEM), "%s, allocation %d: status %d", name, n, st);
      if (!reached) return;
    }
    CHECK(false, "%s: never got through", name);
  };
  each("cache", [&] {
    fcg_cache* c = nullptr;
    const fcg_status st = fcg_cache_create(&d, 3, 100, 16, 40, 0, &c);
    const long left = host::fail_alloc;
    fcg_cache_destroy(c);
    host::fail_alloc = left;
    return st;
  });
  World w(FCG_BF16, 16, 0);
  int32_t id = 0;
  if (fcg_lib_host_reserve(w.lib, 400) != FCG_OK) std::abort();
  each("segment", [&] { return fcg_lib_add_segment(w.lib, 16, 0, nullptr, nullptr, nullptr, &id); });
  const int64_t used = w.lib->used;
  for (int i = 0; i < 3; ++i) {
    each("offload", [&] { return w.lib->segs[i].tok_off < 0 ? FCG_OK : fcg_lib_offload(w.lib, i, nullptr); });
    each("reload", [&] { return w.lib->segs[i].tok_off >= 0 ? FCG_OK : fcg_lib_reload(w.lib, i, nullptr); });
  }
  CHECK(w.lib->used == used, "offload and reload: %lld tokens used", (long long)w.lib->used);
  fcg_locality* loc = nullptr;
  each("scorer", [&] {
    fcg_locality_destroy(loc);
    loc = nullptr;
    return fcg_locality_create(4, 3, 0.4, 0.3, 0.3, &loc);
  });
  const std::vector<int32_t> trace = {0, 1, 2, 3};
  std::vector<double> score(4);
  std::vector<int64_t> cost(4, 1);
  std::vector<uint8_t> keep(4);
  each("record", [&] { return fcg_locality_record(loc, 4, trace.data()); });
  each("scores", [&] { return fcg_locality_scores(loc, score.data()); });
  each("residency", [&] { return fcg_locality_residency(loc, 2, cost.data(), keep.data()); });
  each("update", [&] { return fcg_lib_update_residency(w.lib, loc, (int64_t)1 << 30, 0.0, nullptr, nullptr, nullptr); });
  fcg_locality_destroy(loc);
}

}  // namespace

int main() {
  std::setvbuf(stdout, nullptr, _IOLBF, 0);
  const std::vector<int32_t> zero40(40, 0), two(2, 1), all = iota(SEQS);
  const Call full_page = append(all, std::vector<int32_t>(SEQS, 0), true);
  const Call next_page = append(all, std::vector<int32_t>(SEQS, 16), true);
  // the plan by value, from memory (70 runs), and a reservation
  every_failure("append by value", FCG_BF16, 16, 0, nullptr, append(zero40, iota(40, 3), true),
                append({0, 0}, {1, 50}, true));
  every_failure("append list", FCG_BF16, 16, 0, full_page, next_page, append({0}, {17}, true));
  every_failure("reserve", FCG_BF16, 16, 0, nullptr, append(all, iota(SEQS), false), append({0, 9}, {1, 10}, true));
  every_failure("append contiguous", FCG_F32, 0, 0, nullptr, append(all, iota(SEQS), true));
  // grafts by value and from memory; values copied, and read from the library
  std::vector<int32_t> seg40(40, 1);
  for (uint32_t flags : {0u, (uint32_t)FCG_ALIAS_V}) {
    const char* name[2][2] = {{"graft by value", "graft list"}, {"graft by value, values in the library", "graft list, values in the library"}};
    every_failure(name[flags != 0][0], FCG_BF16, 16, flags, nullptr, graft({0, 0, 3}, {0, 1, 2}, {0, 100, 5}),
                  append({0, 3}, {140, 30}, true));
    every_failure(name[flags != 0][1], FCG_BF16, 16, flags, nullptr, graft(iota(40), seg40, std::vector<int32_t>(40, 7)),
                  append({0, 39}, {47, 50}, true));
  }
  // A cut inside a page whose positions before it were never written leaves the page mapped and
  // empty; a graft that covers it puts its values into the library, a failed one must not: the
  // tokens placed there next have their own.
  const Call emptied = [&](World& w) {
    if (fcg_status st = append({0}, {40}, true)(w)) return st;
    return fcg_cache_truncate(w.cache, 0, 36, nullptr);
  };
  every_failure("graft over an empty page, values in the library", FCG_BF16, 16, FCG_ALIAS_V, emptied,
                graft({0}, {0}, {20}), append({0}, {140}, true));
  {
    // the failed graft, then tokens of the page without the graft
    for (int n = 0; n < 64; ++n) {
      World w(FCG_BF16, 16, FCG_ALIAS_V);
      CHECK(emptied(w) == FCG_OK, "empty page");
      host::fail_hip = n;
      const fcg_status st = graft({0}, {0}, {20})(w);
      const bool reached = host::fail_hip < 0;
      host::fail_hip = -1;
      if (!reached) break;
      if (st == FCG_OK) continue;
      CHECK(append({0, 0}, {33, 34}, true)(w) == FCG_OK, "append after a failed graft, HIP call %d", n);
      CHECK(table_agrees(w), "append after a failed graft, HIP call %d", n);
    }
  }
  // the calls with attention
  every_failure("prefill", FCG_BF16, 16, 0, nullptr, prefill(zero40, iota(40)), decode({0}, false));
  std::vector<int32_t> back = iota(40, 39, -1);
  every_failure("prefill, tokens backwards", FCG_BF16, 16, 0, nullptr, prefill(zero40, back), decode({0}, true));
  every_failure("prefill fp32", FCG_F32, 16, 0, nullptr, prefill(zero40, iota(40)), decode({0}, false));
  const Call sixteen = [](World& w) {
    std::vector<int32_t> seq, pos;
    for (int s = 0; s < SEQS; ++s)
      for (int p = 0; p < 16; ++p) seq.push_back(s), pos.push_back(p);
    return fcg_append(w.cache, 0, L, (int)seq.size(), seq.data(), pos.data(), nullptr, nullptr, nullptr, nullptr, nullptr,
                      0, nullptr);
  };
  every_failure("decode", FCG_BF16, 16, 0, sixteen, decode(all, false), decode(all, false));
  every_failure("decode without allocation", FCG_BF16, 16, 0, sixteen, decode(all, true), decode(all, true));
  // a cut inside a page whose values are read from the library
  every_failure("cut", FCG_BF16, 16, FCG_ALIAS_V, graft({0}, {0}, {0}),
                [](World& w) { return fcg_cache_truncate(w.cache, 0, 40, nullptr); }, append({0, 0}, {40, 41}, true));
  entry_points_return_a_status();
  if (!failures) std::printf("ok\n");
  return failures ? 1 : 0;
}

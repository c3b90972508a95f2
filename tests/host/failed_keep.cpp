// What a cache takes in with norms and what it keeps, with every allocation and every HIP call
// of the calls made to fail in turn: a failed append or sum of weights leaves the layout as it
// was; a failed eviction too, but that it may leave its targets empty.
// The same call succeeds afterwards, and the device page table holds every mapped page.
#include "host_runtime.hpp"

#include <functional>
#include <numeric>

namespace fcg {
// the launches that host_runtime.hpp does not have
int launch_norm_rope(int, int, bool, const RopeRows&, const int32_t*, const RopeArgs&, const NormArgs<true>&, hipStream_t) {
  return host::launch();
}
int launch_append_norm(int dtype, bool pairs, const RopeRows& rows, const AppendArgs& args, int n_runs,
                       const AppendGroup* groups, int n_groups, const CacheView& cv, int layer0, const RopeArgs& ra,
                       const float2* tab, const NormArgs<true>&, hipStream_t s) {
  return launch_append(dtype, pairs, rows, args, n_runs, groups, n_groups, cv, layer0, ra, tab, s);
}
int launch_norm_rope_grad(int, int, bool, const NormGradArgs&, const RopeArgs&, hipStream_t) { return host::launch(); }
int launch_attend_weights(int, const WeightCall&, const WeightArgs*, const WeightItem*, const WeightRank*, int, int,
                          const CacheView&, hipStream_t) {
  return host::launch();
}
int launch_evict_select(const EvictCall&, const EvictArgs&, const RopeArgs&, int, int, int, int, int, hipStream_t) {
  return host::launch();
}
int launch_evict_move(int, bool, bool, const EvictCall&, const EvictArgs&, int, const CacheView&, int, int, hipStream_t) {
  return host::launch();
}
int launch_logprobs(int, const LogpArgs&, hipStream_t) { return host::launch(); }
int launch_logprobs_grad(int, const LogpGradArgs&, hipStream_t) { return host::launch(); }
}  // namespace fcg

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

constexpr int L = 2, HQ = 4, HKV = 2, D = 64, SEQS = 70, TOKENS = 160, PAGE = 16;

struct World {
  fcg_cache* cache = nullptr;
  std::vector<float> data = std::vector<float>((size_t)L * SEQS * TOKENS * HQ * D / 8);
  std::vector<float> w = std::vector<float>((size_t)L * SEQS * HKV * TOKENS);
  fcg_norm norm{};
  World() {
    const fcg_model_desc d{L, HQ, HKV, D, 1e4, FCG_BF16, 0};
    if (fcg_cache_create(&d, SEQS, TOKENS, PAGE, 400, 0, &cache)) std::abort();
    norm.eps = 1e-6f;
  }
  ~World() { fcg_cache_destroy(cache); }
  fcg_tensor rows(int heads) { return fcg_tensor{data.data(), (int64_t)SEQS * heads * D, heads * D, D}; }
};

typedef std::vector<std::vector<int32_t>> Layout;  // of each sequence: lengths of the layers, mapped pages
Layout layout_of(const World& w) {
  Layout a;
  for (int s = 0; s < SEQS; ++s) {
    std::vector<int32_t> x;
    for (int l = 0; l < L; ++l) x.push_back(w.cache->plan.seq_len(s, l));
    for (int p = 0; p < w.cache->plan.n_logical_pages(); ++p) x.push_back(w.cache->plan.page_row(s)[p]);
    a.push_back(x);
  }
  return a;
}
bool table_agrees(const World& w) {
  const int nlp = w.cache->plan.n_logical_pages();
  for (int s = 0; s < SEQS; ++s)
    for (int p = 0; p < nlp; ++p) {
      const int32_t at = w.cache->plan.page_row(s)[p];
      if (at >= 0 && w.cache->d_page_table[(int64_t)s * 2 * nlp + p] != at) return false;
    }
  return true;
}

typedef std::function<fcg_status(World&)> Call;

// may_empty: sequences that a failure may leave empty
void every_failure(const char* name, const Call& before, const Call& call, const std::vector<int>& may_empty = {}) {
  for (bool hip : {false, true}) {
    int n = 0;
    for (;; ++n) {
      World w;
      if (before) CHECK(before(w) == FCG_OK, "%s: the calls before: %s", name, fcg_last_error());
      const Layout was = layout_of(w);
      (hip ? host::fail_hip : host::fail_alloc) = n;
      const fcg_status st = call(w);
      const bool reached = (hip ? host::fail_hip : host::fail_alloc) < 0;
      host::fail_hip = host::fail_alloc = -1;
      const char* kind = hip ? "HIP call" : "allocation";
      if (!reached) {
        CHECK(st == FCG_OK, "%s: status %d although nothing failed: %s", name, st, fcg_last_error());
        break;
      }
      if (st != FCG_OK) {
        CHECK(hip ? st == FCG_EHIP || st == FCG_ENOMEM : st == FCG_ENOMEM, "%s, %s %d: status %d", name, kind, n, st);
        const Layout now = layout_of(w);
        for (int s = 0; s < SEQS; ++s) {
          bool same = now[s] == was[s];
          const bool target = std::count(may_empty.begin(), may_empty.end(), s);
          if (!same && (hip || target)) {
            // empty, or only pages that hold nothing given back
            bool empty = target, less = true;
            for (size_t i = 0; i < now[s].size(); ++i) {
              empty = empty && now[s][i] == (i < L ? 0 : -1);
              less = less && hip && (now[s][i] == was[s][i] || (i >= L && now[s][i] < 0));
            }
            same = empty || less;
          }
          CHECK(same, "%s, %s %d: the layout of sequence %d changed", name, kind, n, s);
        }
        CHECK(table_agrees(w), "%s, %s %d: the device page table", name, kind, n);
        CHECK(call(w) == FCG_OK, "%s, %s %d: the call again: %s", name, kind, n, fcg_last_error());
      }
      CHECK(table_agrees(w), "%s, %s %d: the device page table after", name, kind, n);
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

Call append(std::vector<int32_t> seq, std::vector<int32_t> pos) {
  return [=](World& w) {
    const fcg_tensor q = w.rows(HQ), kv = w.rows(HKV);
    return fcg_append_norm(w.cache, 0, L, (int)seq.size(), seq.data(), pos.data(), nullptr, &w.norm, &w.norm, &q, &q, &kv,
                           &kv, 0, nullptr);
  };
}
// n positions of sequences 0 .. 3 and of sequence `more`
Call filled(int n, int more) {
  return [=](World& w) {
    for (int s : {0, 1, 2, 3, more}) {
      const std::vector<int32_t> seq(n, s), pos = iota(n);
      if (fcg_status st = fcg_append(w.cache, 0, L, n, seq.data(), pos.data(), nullptr, nullptr, nullptr, nullptr, nullptr, 0,
                                     nullptr))
        return st;
    }
    return FCG_OK;
  };
}
Call weights(std::vector<int32_t> seq, std::vector<int32_t> pos) {
  return [=](World& w) {
    const fcg_tensor q = w.rows(HQ);
    return fcg_attend_weights(w.cache, 1, -1, 0, (int)seq.size(), seq.data(), pos.data(), &q, w.data.data(), w.w.data(), 0,
                              nullptr);
  };
}
Call evict(std::vector<int32_t> src, std::vector<int32_t> dst, std::vector<int32_t> keep) {
  return [=](World& w) {
    return fcg_evict(w.cache, (int)src.size(), src.data(), dst.data(), keep.data(), 1, 2, nullptr, w.w.data(), nullptr,
                     nullptr);
  };
}

}  // namespace

int main() {
  std::setvbuf(stdout, nullptr, _IOLBF, 0);
  every_failure("append by value", nullptr, append(std::vector<int32_t>(40, 0), iota(40, 3)));
  every_failure("append list", nullptr, append(iota(SEQS), std::vector<int32_t>(SEQS, 0)));
  const Call full = filled(100, 60);
  every_failure("weights by value", full, weights({0, 0, 1, 60}, {97, 99, 5, 40}));
  std::vector<int32_t> seq(200);
  for (int i = 0; i < 200; ++i) seq[i] = i & 3;
  every_failure("weights list", full, weights(seq, std::vector<int32_t>(200, 90)));
  // several splits of the rows: partials in the workspace
  every_failure("weights, split", full, weights(std::vector<int32_t>(1000, 2), iota(1000, 0, 0)));
  every_failure("eviction in place", full, evict({0, 3}, {0, 3}, {10, 200 - 60}));
  every_failure("eviction into others", full, evict({0, 0, 2}, {5, 60, 7}, {30, 100, 0}), {5, 60, 7});
  every_failure("eviction, both", full, evict({0, 1, 2}, {5, 1, 60}, {33, 17, 1}), {5, 60});
  if (!failures) std::printf("ok\n");
  return failures ? 1 : 0;
}

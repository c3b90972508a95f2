// What sums of attention weight and evictions launch, on a machine without a GPU: see the checks of each.
#include "keep_runtime.hpp"

#include <fstream>
#include <numeric>
#include <set>

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

fcg_cache* cache_of(int32_t dtype, int hq, int hkv, int d, int seqs, int tokens, int page, int pages) {
  const fcg_model_desc m{1, hq, hkv, d, 1e4, dtype, 0};
  fcg_cache* c = nullptr;
  if (fcg_cache_create(&m, seqs, tokens, page, pages, 0, &c)) std::abort();
  return c;
}

// Each launch adds up the splits of the blocks of keys whose first split is in it: all splits
// of a block have to be in that launch, and every block is in one.
void splits_meet_in_one_launch() {
  struct {
    int hq, tokens;  // tokens of the last sequence
  } cases[] = {{16, 2000}, {1, 8192}, {16, 8192}, {2, 1}};
  for (const auto& x : cases) {
    const int singles = 65530, n = singles + x.tokens;
    fcg_cache* c = cache_of(FCG_BF16, x.hq, 1, 64, singles + 1, 8192, 16, singles + 512);
    std::vector<int32_t> seq(n, singles), pos(n, 0);
    std::iota(seq.begin(), seq.begin() + singles, 0);
    std::iota(pos.begin() + singles, pos.end(), 0);
    CHECK(fcg_append(c, 0, 1, n, seq.data(), pos.data(), nullptr, nullptr, nullptr, nullptr, nullptr, 0, nullptr) == FCG_OK,
          "%s", fcg_last_error());
    std::vector<host::Weights> seen;
    host::weights = &seen;
    float y[4] = {};
    const fcg_tensor q{y, 0, 0, 0};
    CHECK(fcg_attend_weights(c, 0, -1, 0, n, seq.data(), pos.data(), &q, y, y, 0, nullptr) == FCG_OK, "%s", fcg_last_error());
    host::weights = nullptr;
    std::set<int> blocks;
    int most = 0;
    for (const auto& l : seen) {
      CHECK(!l.by_value && l.n_items > 0 && l.n_items <= 65535, "a launch of %d items", l.n_items);
      for (size_t i = 0; i < l.items.size() && failures < 20; ++i) {
        const fcg::WeightItem& it = l.items[i];
        most = std::max(most, it.n_split);
        if (it.split == 0) CHECK(blocks.insert(it.kb).second, "block %d of keys twice", it.kb);
        else CHECK(i && l.items[i - 1].kb == it.kb && l.items[i - 1].split == it.split - 1,
                   "split %d of %d of block %d of keys does not follow the one before in its launch", it.split, it.n_split, it.kb);
        if (i + 1 == l.items.size()) CHECK(it.split == it.n_split - 1, "a launch ends at split %d of %d", it.split, it.n_split);
        if (it.n_split > 1) CHECK(l.call.part, "splits without a workspace");
      }
    }
    CHECK((int)blocks.size() == singles + (x.tokens + seen[0].block - 1) / seen[0].block, "%zu blocks of keys", blocks.size());
    std::printf("%d query heads, %d tokens: %zu launches, up to %d splits\n", x.hq, x.tokens, seen.size(), most);
    fcg_cache_destroy(c);
  }
}

// The longest cache and many rows: tiles past blocks of keys are more than 32 bits count.
void largest_plans() {
  const int tokens = (1 << 25) - 16, n = 1 << 21;
  fcg_cache* c = cache_of(FCG_BF16, 16, 1, 64, 2, tokens, 0, 0);
  std::vector<int32_t> seq(tokens), pos(tokens);
  std::iota(pos.begin(), pos.end(), 0);
  CHECK(fcg_append(c, 0, 1, tokens, seq.data(), pos.data(), nullptr, nullptr, nullptr, nullptr, nullptr, 0, nullptr) == FCG_OK,
        "%s", fcg_last_error());
  seq.assign(n, 1);  // rows that see the prefix only
  pos.assign(n, tokens - 1);
  std::vector<host::Weights> seen;
  host::weights = &seen;
  float y[4] = {};
  const fcg_tensor q{y, 0, 0, 0};
  CHECK(fcg_attend_weights(c, 0, 0, tokens, n, seq.data(), pos.data(), &q, y, y, 0, nullptr) == FCG_OK, "%s", fcg_last_error());
  host::weights = nullptr;
  int64_t rows = 0, keys = 0;
  for (const auto& l : seen)
    for (const fcg::WeightItem& it : l.items) {
      if (failures > 20) break;
      CHECK(it.n_row > 0 && it.row0 >= 0 && (int64_t)it.row0 + it.n_row <= (int64_t)n * 16, "rows %d + %d", it.row0, it.n_row);
      CHECK(it.split >= 0 && it.split < it.n_split, "split %d of %d", it.split, it.n_split);
      rows += it.n_row;
      if (it.split == 0) keys += it.k1 - it.k0;
    }
  const int64_t blocks = seen.empty() ? 0 : (tokens + seen[0].block - 1) / seen[0].block;
  CHECK(keys == tokens && rows == blocks * n * 16, "%lld keys, %lld rows", (long long)keys, (long long)rows);
  fcg_cache_destroy(c);
}

// An eviction in place of more sequences than a launch takes, each of its HIP calls made to fail
// in turn: a sequence has its new length if its rows were moved, and its old one if not.
void failures_in_place() {
  const int seqs = 150, tokens = 40;
  for (int n = 0;; ++n) {
    fcg_cache* c = cache_of(FCG_BF16, 4, 2, 64, seqs, 64, 16, seqs * 4);
    std::vector<int32_t> seq, pos, all(seqs), keep(seqs);
    for (int s = 0; s < seqs; ++s) {
      for (int t = 0; t < tokens; ++t) seq.push_back(s), pos.push_back(t);
      all[s] = s;
      keep[s] = s % 7 * 5;  // (0: nothing to move)
    }
    CHECK(fcg_append(c, 0, 1, (int)seq.size(), seq.data(), pos.data(), nullptr, nullptr, nullptr, nullptr, nullptr, 0,
                     nullptr) == FCG_OK, "%s", fcg_last_error());
    std::vector<float> w((size_t)seqs * 2 * 64);
    std::vector<fcg::EvictItem> moved;
    host::moved = &moved;
    host::fail_hip = n;
    const fcg_status st = fcg_evict(c, seqs, all.data(), all.data(), keep.data(), 0, 0, nullptr, w.data(), nullptr, nullptr);
    const bool reached = host::fail_hip < 0;
    host::fail_hip = -1;
    host::moved = nullptr;
    CHECK((st == FCG_OK) == !reached, "call %d: status %d", n, st);
    std::vector<int> want(seqs, tokens);
    for (const auto& it : moved) want[it.src] = it.keep;
    for (int s = 0; s < seqs && failures < 20; ++s)
      CHECK(c->plan.seq_len(s, 0) == want[s], "call %d: sequence %d of length %d, not %d", n, s, c->plan.seq_len(s, 0), want[s]);
    fcg_cache_destroy(c);
    if (!reached) {
      CHECK((int)moved.size() == seqs, "%zu sequences moved", moved.size());
      std::printf("eviction in place: %d HIP calls\n", n);
      return;
    }
  }
}

// The calls of a file, a line each: dtype, query heads, kv heads, head dim, page size, prefix, the own
// positions of each sequence and the tokens: prints block size, whether the plan goes by value, whether rows are split.
void plans(const char* file) {
  std::ifstream in(file);
  int dtype, hq, hkv, d, page, P, n_own, n;
  while (in >> dtype >> hq >> hkv >> d >> page >> P >> n_own >> n) {
    std::vector<int32_t> own(n_own), seq(n), pos(n), rs, rp;
    for (auto* v : {&own, &seq, &pos})
      for (int32_t& x : *v) in >> x;
    int tokens = std::max(P, 1);
    for (int s = 0; s < n_own; ++s)
      for (int t = 0; t < own[s]; ++t) rs.push_back(s), rp.push_back(P + t), tokens = std::max(tokens, P + t + 1);
    for (int t = 0; t < P; ++t) rs.push_back(n_own), rp.push_back(t);
    fcg_cache* c = cache_of(dtype, hq, hkv, d, n_own + 1, tokens, page, page ? (n_own + 1) * (tokens / 16 + 1) : 0);
    CHECK(fcg_append(c, 0, 1, (int)rs.size(), rs.data(), rp.data(), nullptr, nullptr, nullptr, nullptr, nullptr, 0,
                     nullptr) == FCG_OK, "%s", fcg_last_error());
    std::vector<host::Weights> seen;
    host::weights = &seen;
    float y[4] = {};
    const fcg_tensor q{y, 0, 0, 0};
    CHECK(fcg_attend_weights(c, 0, n_own, P, n, seq.data(), pos.data(), &q, y, y, 0, nullptr) == FCG_OK, "%s", fcg_last_error());
    host::weights = nullptr;
    CHECK(seen.size() == 1, "%zu launches", seen.size());
    std::printf("plan %d %d %d\n", seen[0].block, (int)seen[0].by_value, seen[0].call.part != nullptr);
    fcg_cache_destroy(c);
  }
}

}  // namespace

int main(int argc, char** argv) {
  std::setvbuf(stdout, nullptr, _IOLBF, 0);
  if (argc > 1) {
    plans(argv[1]);
    return failures ? 1 : 0;
  }
  splits_meet_in_one_launch();
  largest_plans();
  failures_in_place();
  if (!failures) std::printf("ok\n");
  return failures ? 1 : 0;
}

// What calls launch, on a machine without a GPU: see the checks of each.
#include "host_runtime.hpp"

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

fcg_cache* cache_of(int32_t dtype, int hq, int hkv, int d, int seqs, int tokens, int page, int pages, int layers = 2) {
  const fcg_model_desc m{layers, hq, hkv, d, 1e4, dtype, 0};
  fcg_cache* c = nullptr;
  if (fcg_cache_create(&m, seqs, tokens, page, pages, 0, &c)) std::abort();
  return c;
}

// A reservation that maps no page launches nothing, stages nothing, and can be made
// while the stream is captured; one that maps pages uploads their rows, and cannot.
void reservations() {
  for (int page : {0, 16}) {
    fcg_cache* c = cache_of(FCG_BF16, 4, 2, 64, 3, 100, page, 20);
    std::vector<int32_t> seq(70), pos(70);
    std::iota(pos.begin(), pos.end(), 0);
    auto reserve = [&](int n, const int32_t* p) {
      return fcg_append(c, 0, 2, n, seq.data(), p, nullptr, nullptr, nullptr, nullptr, nullptr, 0, nullptr);
    };
    const int32_t one[2] = {1, 2};
    if (page) {
      host::capture = true;
      CHECK(reserve(1, one) == FCG_ESTATE, "a page mapped while capturing");
      host::capture = false;
      CHECK(reserve(1, one) == FCG_OK, "one position");
      CHECK(fcg_cache_truncate(c, 0, 1, nullptr) == FCG_OK, "cut");  // the page stays
    }
    const int before = host::launches;
    const size_t ring = c->ring.cap;
    host::capture = true;
    CHECK(reserve(2, one) == FCG_OK, "page %d, captured: %s", page, fcg_last_error());
    host::capture = false;
    CHECK(fcg_cache_truncate(c, 0, 1, nullptr) == FCG_OK, "cut");
    CHECK(reserve(2, one) == FCG_OK, "page %d", page);
    CHECK(host::launches == before && c->ring.cap == ring, "page %d: %d launches", page, host::launches - before);
    int32_t n;
    fcg_cache_export_layout(c, 0, 1, nullptr, &n, nullptr);
    CHECK(n == 3, "length %d", n);
    if (!page) CHECK(reserve(70, pos.data()) == FCG_EOVERLAP, "positions already written");
    fcg_cache_destroy(c);
  }
}

bool fits(const fcg::RopeRows& r, int64_t groups) {
  const int64_t slices = (r.tb * (r.Hq + r.Hk + r.Hv) + r.slice_rows - 1) / r.slice_rows;
  return groups * 256 < (int64_t)1 << 32 && slices <= 65535 && r.grid_layers <= 65535;
}

// Up to 2^30 tokens: launches of fewer than 2^32 threads along x that follow each other.
void long_encodings() {
  fcg_rope_desc rd{};
  rd.rotary_dim = 64;
  rd.theta = 1e4;
  rd.attn_factor = 1.0;
  fcg_rope* rope = nullptr;
  if (fcg_rope_create(&rd, &rope)) std::abort();
  std::vector<host::Apply> seen;
  host::applies = &seen;
  char* const base = (char*)0x100000;  // (nothing is read)
  const int32_t* const pos = (const int32_t*)0x40000000;
  struct {
    int32_t n, hq, hk;
  } cases[] = {{1 << 30, 1, 0}, {(1 << 28) + 5, 0, 1}, {20000000, 64, 1}, {20000000, 33, 0}, {1000, 8, 8}, {1 << 30, 4096, 4096}};
  for (const auto& x : cases)
    for (int32_t dtype : {FCG_BF16, FCG_F32}) {
      const int64_t es = dtype == FCG_F32 ? 4 : 2;
      seen.clear();
      const fcg_tensor q{base, 0, x.hq * 64, 64}, k{base + 64, 0, x.hk * 64, 64};
      CHECK(fcg_rope_apply(rope, dtype, 64, 1, x.n, pos, x.hq, &q, &q, x.hk, &k, &k, 0, nullptr) == FCG_OK, "%d tokens: %s",
            x.n, fcg_last_error());
      int64_t at = 0;
      for (const host::Apply& a : seen) {
        CHECK(fits(a.rows, (a.rows.n_tok + (int64_t)a.rows.tb - 1) / a.rows.tb), "%d tokens, %d + %d heads: a launch of %d tokens by %d",
              x.n, x.hq, x.hk, a.rows.n_tok, a.rows.tb);
        CHECK(a.pos == pos + at, "positions of token %lld", (long long)at);
        if (x.hq) CHECK((const char*)a.rows.q.p == base + at * x.hq * 64 * es && a.rows.q_out.p == a.rows.q.p, "q of token %lld", (long long)at);
        if (x.hk) CHECK((const char*)a.rows.k.p == base + 64 + at * x.hk * 64 * es && a.rows.k_out.p == a.rows.k.p, "k of token %lld", (long long)at);
        CHECK((a.rows.q.p != nullptr) == (x.hq > 0) && (a.rows.k.p != nullptr) == (x.hk > 0), "rows that are not given");
        at += a.rows.n_tok;
      }
      CHECK(at == x.n, "%d tokens: %lld launched", x.n, (long long)at);
    }
  host::applies = nullptr;
  fcg_rope_destroy(rope);
}

// More groups of tokens than a launch takes: several launches of the list.
void long_appends() {
  const int n = (1 << 24) + 3000;
  fcg_cache* c = cache_of(FCG_BF16, 32, 32, 64, 1, n, 0, 0, 1);
  std::vector<int32_t> seq(n), pos(n);
  std::iota(pos.begin(), pos.end(), 0);
  std::vector<host::Append> seen;
  host::appends = &seen;
  float x;
  const fcg_tensor kv{&x, 0, 0, 64};
  CHECK(fcg_append(c, 0, 1, n, seq.data(), pos.data(), nullptr, nullptr, nullptr, &kv, &kv, 0, nullptr) == FCG_OK, "%s",
        fcg_last_error());
  int64_t at = 0;
  for (const host::Append& a : seen) {
    CHECK(fits(a.rows, a.n_groups), "a launch of %d groups", a.n_groups);
    if (!a.groups) {
      CHECK(false, "a plan by value");
      break;
    }
    for (int i = 0; i < a.n_groups && failures < 20; at += a.groups[i++].n)
      CHECK(a.groups[i].tok0 == at && a.groups[i].pos0 == at, "group %d: token %d, not %lld", i, a.groups[i].tok0, (long long)at);
  }
  CHECK(at == n && seen.size() > 1, "%lld tokens in %zu launches", (long long)at, seen.size());
  // as many tokens that attend: refused, as documented
  const fcg_tensor q{&x, 0, 0, 0}, out{&x, 0, 32 * 64, 64};
  CHECK(fcg_prefix_attend(c, 0, 0, 0, 1 << 24, seq.data(), pos.data(), &q, &out, nullptr, nullptr) == FCG_EINVAL, "2^24 tokens");
  host::appends = nullptr;
  fcg_cache_destroy(c);
}

// The calls of rotary forms, appending and prefix attention run on their cache's device
// and leave the caller's current one as it was.
void devices() {
  const fcg_model_desc m{1, 4, 2, 64, 1e4, FCG_BF16, 0};
  fcg_rope_desc rd{};
  rd.rotary_dim = 64;
  rd.theta = 1e4;
  rd.attn_factor = 1.0;
  fcg_rope* rope = nullptr;
  fcg_lib* lib = nullptr;
  int32_t id;
  float x = 0;
  host::device = 3;
  fcg_cache* c = cache_of(FCG_BF16, 4, 2, 64, 3, 100, 16, 20, 1);
  if (fcg_rope_create(&rd, &rope) || fcg_lib_create(&m, 64, 1, 0, &lib) || fcg_lib_add_segment(lib, 40, 0, &x, &x, nullptr, &id))
    std::abort();
  host::device = 1;
  auto check = [&](fcg_status st, const char* what) {
    CHECK(st == FCG_OK, "%s: %s", what, fcg_last_error());
    CHECK(host::launch_device == 3, "%s: launched on device %d", what, host::launch_device);
    CHECK(host::device == 1, "%s: left device %d current", what, host::device);
    host::launch_device = -1;
  };
  const int32_t seq[1] = {0}, seg[1] = {0}, dst[1] = {0}, pos[1] = {40};
  const fcg_tensor q{&x, 0, 256, 64}, kv{&x, 0, 128, 64};
  check(fcg_graft_rope(c, lib, rope, 1, seq, seg, dst, nullptr), "graft_rope");
  check(fcg_append(c, 0, 1, 1, seq, pos, rope, &q, &q, &kv, &kv, 0, nullptr), "append");
  check(fcg_prefix_attend(c, 0, 0, 40, 1, seq, pos, &q, &q, nullptr, nullptr), "prefix_attend");
  CHECK(fcg_graft_rope(c, lib, rope, 1, seq, seg, dst, nullptr) == FCG_EOVERLAP && host::device == 1, "a refused graft");
  fcg_cache_destroy(c);
  fcg_lib_destroy(lib);
  fcg_rope_destroy(rope);
}

}  // namespace

int main() {
  std::setvbuf(stdout, nullptr, _IOLBF, 0);
  reservations();
  long_encodings();
  long_appends();
  devices();
  if (!failures) std::printf("ok\n");
  return failures ? 1 : 0;
}

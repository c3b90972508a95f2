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

}  // namespace

int main() {
  std::setvbuf(stdout, nullptr, _IOLBF, 0);
  reservations();
  if (!failures) std::printf("ok\n");
  return failures ? 1 : 0;
}

// Entry points of log probabilities (include/fcg.h): rows of logits, their gradient, and
// the perplexities that the locality score takes from them.
#include <algorithm>
#include <cmath>

#include "locality.hpp"
#include "objects.hpp"
#include "ops.hpp"

using namespace fcg;

namespace {

// Blocks that few rows are cut into, and the least elements of one.  (us a call, rows of 128K bf16, 20
// alternatives: 1 row in splits of 4096, 8192 and 16384 elements 12.4, 13.7, 18.8; 64 rows in
// 2048, 1024, 512 and 256 blocks 20.0, 17.1, 20.7, 27.3: more blocks leave more partials.)
constexpr int64_t kBlocks = 1024;
constexpr int32_t kSplitElements = 4096;

struct Cut {
  int32_t splits, split_len;
};
Cut cut_rows_of(int32_t n, int32_t vocab) {
  int64_t splits = std::min<int64_t>({(kBlocks + n - 1) / n, (vocab + kSplitElements - 1) / kSplitElements, kLogpSplits});
  splits = std::max<int64_t>(splits, 1);
  const int32_t len = (int32_t)(((vocab + splits - 1) / splits + 7) / 8 * 8);
  return Cut{(vocab + len - 1) / len, len};
}
int64_t workspace_of(int32_t n, int32_t vocab, int32_t n_top) {
  const Cut c = cut_rows_of(n, vocab);
  return c.splits == 1 ? 0 : (int64_t)n * c.splits * (16 + 8 * (int64_t)n_top);
}

fcg_status check_rows(int32_t dtype, int32_t n, int32_t vocab, int64_t stride) {
  if (dtype != FCG_F32 && dtype != FCG_BF16) return fail(FCG_EINVAL, "unknown dtype");
  if (n < 0) return fail(FCG_EINVAL, "negative row count");
  if (vocab < 1 || vocab > 1 << 30) return fail(FCG_EINVAL, "vocab must be in [1, 2^30]");
  if (stride < 0) return fail(FCG_EINVAL, "negative stride");
  return FCG_OK;
}

}  // namespace

fcg_status fcg_token_logprobs_workspace(int32_t n_rows, int32_t vocab, int32_t n_top, int64_t* bytes) {
  if (!bytes) return fail(FCG_EINVAL, "null output");
  if (fcg_status st = check_rows(FCG_F32, n_rows, vocab, 0)) return st;
  if (n_top < 0 || n_top > kLogpTop) return fail(FCG_EINVAL, "n_top must be in [0, 64]");
  *bytes = n_rows ? workspace_of(n_rows, vocab, n_top) : 0;
  return FCG_OK;
}

fcg_status fcg_token_logprobs(int32_t dtype, int32_t n_rows, int32_t vocab, const void* logits, int64_t row_stride,
                              const int32_t* targets, float* logprob, float* entropy, float* lse, int32_t n_top,
                              int32_t* top_id, float* top_logprob, void* workspace, int64_t workspace_bytes,
                              void* stream) {
  if (fcg_status st = check_rows(dtype, n_rows, vocab, row_stride)) return st;
  if (n_top < 0 || n_top > kLogpTop || n_top > vocab) return fail(FCG_EINVAL, "n_top must be in [0, 64] and at most vocab");
  if (n_rows == 0) return FCG_OK;
  if (!logits) return fail(FCG_EINVAL, "null logits");
  if (logprob && !targets) return fail(FCG_EINVAL, "log probabilities without targets");
  if (n_top && !top_id) return fail(FCG_EINVAL, "alternatives without top_id");
  if (!logprob && !entropy && !lse && !n_top) return FCG_OK;
  const Cut c = cut_rows_of(n_rows, vocab);
  const int64_t need = workspace_of(n_rows, vocab, n_top);
  if (need && (!workspace || (uintptr_t)workspace % 16)) return fail(FCG_EINVAL, "workspace: null or not 16-byte aligned");
  if (workspace_bytes < need) return fail(FCG_EINVAL, "the workspace is too small");
  constexpr int32_t kRows = 1 << 22;  // of a launch; only rows that are not split are as many
  for (int32_t r0 = 0; r0 < n_rows; r0 += std::min(kRows, n_rows - r0)) {
    LogpArgs a{};
    a.x = (const char*)logits + r0 * row_stride * (int64_t)esize(dtype);
    a.stride = row_stride;
    a.targets = targets ? targets + r0 : nullptr;
    a.logprob = logprob ? logprob + r0 : nullptr;
    a.entropy = entropy ? entropy + r0 : nullptr;
    a.lse = lse ? lse + r0 : nullptr;
    a.top_id = n_top ? top_id + (int64_t)r0 * n_top : nullptr;
    a.top_logprob = n_top && top_logprob ? top_logprob + (int64_t)r0 * n_top : nullptr;
    a.n = std::min(kRows, n_rows - r0);
    a.vocab = vocab;
    a.n_top = n_top;
    a.splits = c.splits;
    a.split_len = c.split_len;
    // more than the last-level cache holds (256 MB): nothing of it lies there (3001 fp32 rows of
    // 50021, 0.6 GB, read through the caches 102 us, past them 94)
    a.stream = (int64_t)n_rows * vocab * (int64_t)esize(dtype) > (int64_t)256 << 20;
    a.part = (float4*)workspace;
    a.part_top = (uint64_t*)((char*)workspace + (need ? (int64_t)n_rows * c.splits * 16 : 0));
    if (int rc = launch_logprobs(dtype, a, (hipStream_t)stream)) return hip_fail((hipError_t)rc, "log probability launch");
  }
  return FCG_OK;
}

fcg_status fcg_token_logprobs_backward(int32_t dtype, int32_t n_rows, int32_t vocab, const void* logits,
                                       int64_t row_stride, const int32_t* targets, const float* lse,
                                       const float* entropy, const float* g_logprob, const float* g_entropy,
                                       const float* g_lse, void* dlogits, int64_t d_stride, void* stream) {
  if (fcg_status st = check_rows(dtype, n_rows, vocab, row_stride)) return st;
  if (n_rows == 0) return FCG_OK;
  if (!logits || !lse || !dlogits) return fail(FCG_EINVAL, "null tensor");
  if (g_logprob && !targets) return fail(FCG_EINVAL, "a gradient of log probabilities without targets");
  if (g_entropy && !entropy) return fail(FCG_EINVAL, "a gradient of the entropy without the entropy");
  if (n_rows > 1 && d_stride < vocab) return fail(FCG_EINVAL, "rows of dlogits overlap");
  if (dlogits == logits && n_rows > 1 && d_stride != row_stride)
    return fail(FCG_EINVAL, "dlogits in the place of the logits needs their stride");
  LogpGradArgs a{};
  a.x = logits;
  a.dx = dlogits;
  a.stride = row_stride;
  a.d_stride = d_stride;
  a.targets = targets;
  a.lse = lse;
  a.entropy = entropy;
  a.g_logprob = g_logprob;
  a.g_entropy = g_entropy;
  a.g_lse = g_lse;
  a.n = n_rows;
  a.vocab = vocab;
  const int32_t each = kLogpGradVecs * 256 * 16 / (int32_t)esize(dtype);
  a.chunks = (vocab + each - 1) / each;
  if (int rc = launch_logprobs_grad(dtype, a, (hipStream_t)stream)) return hip_fail((hipError_t)rc, "gradient launch");
  return FCG_OK;
}

fcg_status fcg_locality_measure_ppl(fcg_locality* loc, int32_t n, const int32_t* funcs, const int32_t* n_tok,
                                    const float* logprob, void* stream) {
  if (!loc) return fail(FCG_EINVAL, "null handle");
  if (n < 0) return fail(FCG_EINVAL, "negative count");
  if (n == 0) return FCG_OK;
  if (!funcs || !n_tok || !logprob) return fail(FCG_EINVAL, "null argument");
  int64_t total = 0;
  for (int32_t i = 0; i < n; ++i) {
    if (n_tok[i] < 1) return fail(FCG_EINVAL, "a function without tokens");
    total += n_tok[i];
  }
  const int32_t n_funcs = locality_size(loc);
  for (int32_t i = 0; i < n; ++i)
    if (funcs[i] < 0 || funcs[i] >= n_funcs) return fail(FCG_ERANGE, "function id out of range");
  return guarded([&]() -> fcg_status {
    // a wait would end the capture
    if (capturing((hipStream_t)stream)) return fail(FCG_ESTATE, "perplexities cannot be measured while the stream is captured");
    std::vector<float> lp(total);
    std::vector<double> ppl(n);
    HIP_TRY(hipStreamSynchronize((hipStream_t)stream), "hipStreamSynchronize");
    HIP_TRY(hipMemcpy(lp.data(), logprob, total * sizeof(float), hipMemcpyDeviceToHost), "hipMemcpy(log probabilities)");
    const float* p = lp.data();
    for (int32_t i = 0; i < n; ++i) {
      double sum = 0.0;
      for (int32_t t = 0; t < n_tok[i]; ++t) sum += *p++;
      ppl[i] = std::exp(-sum / n_tok[i]);
      if (!std::isfinite(ppl[i])) return fail(FCG_EINVAL, "a perplexity is not finite");
    }
    for (int32_t i = 0; i < n; ++i)
      if (fcg_status st = fcg_locality_set_ppl(loc, funcs[i], ppl[i])) return st;
    return FCG_OK;
  });
}

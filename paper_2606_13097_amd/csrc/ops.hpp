// What the entry points around a cache share: checks of the tensors they are given,
// the cut of rows into blocks, appending, the workspace of partials.
#pragma once

#include <algorithm>
#include <string>
#include <utility>

#include "objects.hpp"

namespace fcg {

inline fcg_status fail(fcg_status s, const std::string& msg) { return report(s, msg); }

inline bool capturing(hipStream_t s) {
  hipStreamCaptureStatus st = hipStreamCaptureStatusNone;
  if (hipStreamIsCapturing(s, &st) == hipSuccess) return st != hipStreamCaptureStatusNone;
  (void)hipGetLastError();  // not this call's error
  return false;
}

inline RowView view_of(const fcg_tensor* t) {
  return t ? RowView{t->data, t->layer, t->token, t->head} : RowView{nullptr, 0, 0, 0};
}

// strides of a tensor [layers][tokens][heads][D]
inline fcg_status check_strides(const fcg_tensor* t, const char* what) {
  if (t && (t->layer < 0 || t->token < 0 || t->head < 0))
    return fail(FCG_EINVAL, std::string(what) + ": negative stride");
  return FCG_OK;
}

// Rows of an output must not meet: sorted by stride, each dimension steps over
// what the smaller ones cover.
inline fcg_status check_output(const fcg_tensor* t, int64_t layers, int64_t tokens, int64_t heads, int64_t D, const char* what) {
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

inline bool same_view(const fcg_tensor* a, const fcg_tensor* b) {
  return a->data == b->data && a->layer == b->layer && a->token == b->token && a->head == b->head;
}

// an output that starts where its input does is that input in place, or an error
inline fcg_status check_alias(const fcg_tensor* in, const fcg_tensor* out, const char* what) {
  if (in->data == out->data && !same_view(in, out))
    return fail(FCG_EINVAL, std::string(what) + ": an output in its input's place needs its strides");
  return FCG_OK;
}

// The cut of n_tok tokens' rows (H a token, nch pairs of vectors a row) into blocks.
void cut_rows(RopeRows* rows, int64_t n_tok, int64_t n_layers, int H, int nch);

// fcg_append with a launch of its own (launch_append's arguments; context: of the launch).
struct AppendLaunch {
  int (*fn)(const void* context, int dtype, bool pairs, const RopeRows& rows, const AppendArgs& args, int n_runs,
            const AppendGroup* groups, int n_groups, const CacheView& cv, int layer0, const RopeArgs& ra,
            const float2* tab, hipStream_t s);
  const void* context;
};
fcg_status append_tokens(fcg_cache* c, int32_t layer, int32_t n_layers, int32_t n_tok, const int32_t* seq,
                         const int32_t* pos, const fcg_rope* rope, const fcg_tensor* q, const fcg_tensor* q_out,
                         const fcg_tensor* k, const fcg_tensor* v, uint32_t flags, void* stream,
                         const AppendLaunch& launch);

// The cache's workspace of partials holds `bytes`; `cap`: for a call that is being
// captured, which the workspace is then kept for.
fcg_status prefix_workspace(fcg_cache* c, size_t bytes, bool cap, const char* call);

}  // namespace fcg

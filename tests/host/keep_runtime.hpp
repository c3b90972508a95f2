// The launches of norms, attention weights, eviction and log probabilities on a machine
// without a GPU: noted, for the programs that check what calls launch.
#pragma once

#include "host_runtime.hpp"

namespace host {

struct Weights {
  fcg::WeightCall call;
  bool by_value;
  std::vector<fcg::WeightItem> items;  // of a plan in memory
  int n_items, block;
};
inline std::vector<Weights>* weights = nullptr;
inline std::vector<fcg::EvictItem>* moved = nullptr;  // items whose move was launched

}  // namespace host

namespace fcg {

int launch_norm_rope(int, int, bool, const RopeRows&, const int32_t*, const RopeArgs&, const NormArgs<true>&, hipStream_t) {
  return host::launch();
}
int launch_append_norm(int dtype, bool pairs, const RopeRows& rows, const AppendArgs& args, int n_runs,
                       const AppendGroup* groups, int n_groups, const CacheView& cv, int layer0, const RopeArgs& ra,
                       const float2* tab, const NormArgs<true>&, hipStream_t s) {
  return launch_append(dtype, pairs, rows, args, n_runs, groups, n_groups, cv, layer0, ra, tab, s);
}
int launch_norm_rope_grad(int, int, bool, const NormGradArgs&, const RopeArgs&, hipStream_t) { return host::launch(); }
int launch_attend_weights(int, const WeightCall& call, const WeightArgs* args, const WeightItem* items, const WeightRank*,
                          int n_items, int block, const CacheView&, hipStream_t) {
  if (int rc = host::launch()) return rc;
  if (host::weights) {
    host::weights->push_back(host::Weights{call, args != nullptr, {}, n_items, block});
    if (items) host::weights->back().items.assign(items, items + n_items);
  }
  return 0;
}
int launch_evict_select(const EvictCall&, const EvictArgs&, const RopeArgs&, int, int, int, int, int, hipStream_t) {
  return host::launch();
}
int launch_evict_move(int, bool, bool, const EvictCall&, const EvictArgs& a, int, const CacheView&, int, int, hipStream_t) {
  if (int rc = host::launch()) return rc;
  if (host::moved) host::moved->insert(host::moved->end(), a.item, a.item + a.n);
  return 0;
}
int launch_logprobs(int, const LogpArgs&, hipStream_t) { return host::launch(); }
int launch_logprobs_grad(int, const LogpGradArgs&, hipStream_t) { return host::launch(); }

}  // namespace fcg

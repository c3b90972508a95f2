// The objects behind the C ABI's handles (segment library, composite cache) and
// the staging of per-call plans, shared by the files that implement the entry
// points.
#pragma once

#include <hip/hip_runtime.h>

#include <algorithm>
#include <cstring>
#include <deque>
#include <map>
#include <new>
#include <string>
#include <tuple>
#include <unordered_map>
#include <utility>
#include <vector>

#include "errors.hpp"
#include "fcg.h"
#include "kernels.hpp"
#include "planner.hpp"

namespace fcg {

fcg_status hip_fail(hipError_t e, const char* what);

#define HIP_TRY(expr, what)                               \
  do {                                                    \
    hipError_t e_ = (expr);                               \
    if (e_ != hipSuccess) return fcg::hip_fail(e_, what); \
  } while (0)

// The handle's device for the call, the caller's again afterwards.
struct OnDevice {
  int before = -1;
  hipError_t err = hipSuccess;
  explicit OnDevice(int device) {
    err = hipGetDevice(&before);
    if (err == hipSuccess && before != device) err = hipSetDevice(device);
    else if (err == hipSuccess) before = -1;
  }
  ~OnDevice() {
    if (before >= 0) (void)hipSetDevice(before);
  }
};

inline size_t esize(int32_t dtype) { return dtype == FCG_F32 ? 4 : 2; }

// Staging of per-call plans: a pinned host ring mirrored by a device ring.  A
// call packs its arrays into one blob, which one kernel on the call's stream
// takes from the host ring (upload), and records an event after its last kernel;
// a region is reused only after its event.  What can fail for want of memory is
// done when a region is acquired, before the call launches anything.
struct Ring {
  char* host = nullptr;
  char* dev = nullptr;
  size_t cap = 0, head = 0;
  bool open = false;  // a region is acquired and not retired
  std::deque<std::tuple<size_t, size_t, hipEvent_t>> inflight;
  std::vector<hipEvent_t> spare;

  ~Ring() { release(); }
  void release() {
    for (auto& f : inflight) {
      hipEventSynchronize(std::get<2>(f));
      hipEventDestroy(std::get<2>(f));
    }
    inflight.clear();
    for (auto e : spare) hipEventDestroy(e);
    spare.clear();
    if (host) hipHostFree(host);
    if (dev) hipFree(dev);
    host = dev = nullptr;
    cap = head = 0;
  }
  fcg_status reserve(size_t n) {
    if (n <= cap) return FCG_OK;
    size_t nc = std::max<size_t>(cap * 2, std::max<size_t>(n, 1 << 20));
    release();
    HIP_TRY(hipHostMalloc((void**)&host, nc, hipHostMallocDefault), "hipHostMalloc(staging)");
    HIP_TRY(hipMalloc((void**)&dev, nc), "hipMalloc(staging)");
    cap = nc;
    return FCG_OK;
  }
  // Region [off, off + n) of both rings, free for writing.
  fcg_status acquire(size_t n, size_t* off) {
    if (open) {  // by a call that failed before it could retire it: its kernels may still read it
      HIP_TRY(hipDeviceSynchronize(), "hipDeviceSynchronize(staging)");
      open = false;
    }
    fcg_status st = reserve(n);
    if (st) return st;
    if (head + n > cap) head = 0;
    const size_t a = head, b = head + n;
    for (auto it = inflight.begin(); it != inflight.end();) {
      if (std::get<1>(*it) <= a || std::get<0>(*it) >= b) {
        ++it;
        continue;
      }
      HIP_TRY(hipEventSynchronize(std::get<2>(*it)), "hipEventSynchronize(staging)");
      spare.push_back(std::get<2>(*it));
      it = inflight.erase(it);
    }
    if (spare.empty()) {
      spare.reserve(inflight.size() + 1);  // room for every event to come back
      hipEvent_t e;
      HIP_TRY(hipEventCreateWithFlags(&e, hipEventDisableTiming), "hipEventCreate");
      spare.push_back(e);
    }
    inflight.emplace_back(a, b, spare.back());
    spare.pop_back();
    open = true;
    head = b;
    *off = a;
    return FCG_OK;
  }
  // The last region acquired is free once the stream has come here.
  fcg_status retire(hipStream_t s) {
    HIP_TRY(hipEventRecord(std::get<2>(inflight.back()), s), "hipEventRecord");
    open = false;
    return FCG_OK;
  }
};

// Packs host arrays into one blob with 256-byte aligned members.
struct Blob {
  std::vector<char> bytes;
  size_t add(const void* p, size_t n) {
    size_t off = (bytes.size() + 255) & ~size_t(255);
    bytes.resize(off + n);
    if (n) std::memcpy(bytes.data() + off, p, n);
    return off;
  }
};

}  // namespace fcg

struct fcg_rope {
  int32_t rot = 0, layout = 0;
  double attn_factor = 1.0;
  std::vector<double> freqs;  // [rot / 2] after scaling

  bool pairs() const { return layout == FCG_ROPE_PAIRS; }
  fcg::RopeArgs args() const {
    fcg::RopeArgs a{};
    for (size_t i = 0; i < freqs.size(); ++i) a.turns[i] = freqs[i] / 6.283185307179586477;
    a.m = (float)attn_factor;
    a.rot = rot;
    return a;
  }
};

struct Segment {
  int64_t tok_off;  // first token in the device slabs, -1 while offloaded
  int32_t len, src_pos0;
  int64_t host_off = -1;  // first token in the pinned host slabs, -1 without a host copy
  mutable int32_t pins = 0;  // FCG_ALIAS_V caches reading this segment's values in place
};

struct fcg_lib {
  fcg_model_desc desc;
  int64_t cap = 0, used = 0;              // device slab tokens: capacity, high-water mark
  std::map<int64_t, int64_t> free_tok;    // device token ranges below `used` freed by offloads (start -> length)
  int32_t max_segments = 0;
  uint32_t flags = 0;
  std::vector<Segment> segs;
  void* k = nullptr;
  void* v = nullptr;
  int device = 0;
  // host tier (fcg_lib_host_reserve): pinned [L][Hkv][host_cap][D] slabs, filled once per segment
  int64_t host_cap = 0, host_used = 0;
  void* host_k = nullptr;
  void* host_v = nullptr;
  hipEvent_t freed = nullptr;  // after the copies that read the last freed device range
  // Ordering across streams (offload / reload on a side stream beside grafts):
  // a graft waits for the last reload; a reload or an ingest into a freed
  // range waits for the last graft (which may still read that range) and the
  // offload that freed it.
  mutable hipEvent_t graft_done = nullptr;
  hipEvent_t reload_done = nullptr;

  // first fit among freed ranges, else past the high-water mark; -1 if nothing fits
  int64_t alloc(int64_t len) {
    for (auto it = free_tok.begin(); it != free_tok.end(); ++it)
      if (it->second >= len) {
        const int64_t off = it->first, rest = it->second - len;
        auto node = free_tok.extract(it);  // (a new one could fail after the range is gone)
        if (rest) {
          node.key() = off + len;
          node.mapped() = rest;
          free_tok.insert(std::move(node));
        }
        return off;
      }
    if (used + len > cap) return -1;
    used += len;
    return used - len;
  }
  void release(int64_t off, int64_t len) {
    auto it = free_tok.emplace(off, len).first;
    auto nx = std::next(it);
    if (nx != free_tok.end() && it->first + it->second == nx->first) {
      it->second += nx->second;
      free_tok.erase(nx);
    }
    if (it != free_tok.begin()) {
      auto pv = std::prev(it);
      if (pv->first + pv->second == it->first) {
        pv->second += it->second;
        free_tok.erase(it);
        it = pv;
      }
    }
    if (it->first + it->second == used) {  // the top range returns to the high-water mark
      used = it->first;
      free_tok.erase(it);
    }
  }
};

struct fcg_cache {
  fcg_model_desc desc;
  int32_t n_seqs, max_tokens, page_size, n_pages;
  uint32_t flags;
  fcg::Planner plan;
  void* k = nullptr;
  void* v = nullptr;
  int64_t layer_stride = 0;
  int32_t* d_page_table = nullptr;
  double* d_inv_freq = nullptr;
  float2* d_rope = nullptr;   // (cos, sin) per position and rotary pair [max_tokens][D/2]
  int device = 0;
  fcg::Ring ring;
  // workspaces, grown on demand
  void* qws = nullptr;
  size_t qws_bytes = 0;
  float* part = nullptr;
  size_t part_bytes = 0;
  void* xpart = nullptr;      // partials of fcg_prefix_attend
  size_t xpart_bytes = 0;
  bool xpart_captured = false;  // a captured graph uses xpart
  std::vector<void*> xkept;     // former xparts that captured graphs use
  float* dpart = nullptr;     // decode split partials
  size_t dpart_bytes = 0;
  const fcg_lib* alias_lib = nullptr;  // FCG_ALIAS_V: the library value pages map onto (bound by the first graft)
  std::vector<std::vector<int32_t>> alias_segs;  // per sequence: segments it pins in alias_lib
  int32_t* d_count = nullptr; // decode merge arrival counters [kMaxDecodeSeqs][Hkv] (kCountStride apart), zero between launches
  // kernel timing (fcg_cache_timing): recorded (start, end) event pairs per kind
  bool timing = false;
  std::vector<std::pair<hipEvent_t, hipEvent_t>> spans[5];
  std::vector<hipEvent_t> ev_pool;
  std::unordered_map<hipEvent_t, int> ev_refs;

  fcg_cache(const fcg_model_desc& d, int32_t ns, int32_t mt, int32_t ps, int32_t np, uint32_t fl)
      : desc(d), n_seqs(ns), max_tokens(mt), page_size(ps), n_pages(np), flags(fl),
        plan(d.n_layers, ns, mt, ps, np, (fl & FCG_ALIAS_V) != 0) {}
  bool layout_only() const { return flags & FCG_LAYOUT_ONLY; }

  fcg::CacheView view() const {
    fcg::CacheView c;
    c.k = k;
    c.v = v;
    c.layer_stride = layer_stride;
    c.page_table = d_page_table;
    c.v_alias = plan.alias_v() && d_page_table ? d_page_table + plan.n_logical_pages() : nullptr;
    c.lib_v = alias_lib ? alias_lib->v : nullptr;
    c.lib_cap = alias_lib ? alias_lib->cap : 0;
    c.n_seqs = n_seqs;
    c.max_tokens = max_tokens;
    c.page_size = page_size;
    c.n_lp = plan.n_logical_pages();
    c.n_kv_heads = desc.n_kv_heads;
    c.head_dim = desc.head_dim;
    return c;
  }
};

namespace fcg {

// Enlarge a workspace (waits for the device when it replaces one).
fcg_status grow(void** p, size_t* have, size_t need, const char* what);

// What a call changes in the planner before its last step that can fail: taken
// back when the call ends without keep().  Otherwise the planner would have pages
// that the device table has not, which a later call would not enter, and read.
class Staged {
 public:
  Staged(fcg_cache* c, const std::vector<std::pair<int32_t, int32_t>>& new_pages) : c_(c), pages_(new_pages) {}
  Staged(const Staged&) = delete;
  Staged& operator=(const Staged&) = delete;
  ~Staged() {
    if (!c_) return;
    if (mapped_) c_->plan.unmap_pages(pages_);
    if (!spans_) return;
    for (const Span& x : *spans_) c_->plan.unalias_pages(x.seq, x.dst, x.len, sent_);
    c_->alias_lib = bound_;
  }
  // Values of the pages that the spans cover read from the library.  *again (room for
  // all spans) receives the sequences of which a page mapped before is among them.
  void alias(const fcg_lib* lib, const std::vector<Span>& spans, std::vector<int32_t>* again) {
    bound_ = c_->alias_lib;
    spans_ = &spans;
    c_->alias_lib = lib;
    for (const Span& x : spans)
      if (c_->plan.alias_pages(x.seq, x.dst, x.len, lib->segs[x.seg].tok_off)) again->push_back(x.seq);
  }
  void map() {
    c_->plan.map_pages(pages_);
    mapped_ = true;
  }
  void sent() { sent_ = true; }  // page rows may be in the device table from here on
  void keep() { c_ = nullptr; }

 private:
  fcg_cache* c_;
  const std::vector<std::pair<int32_t, int32_t>>& pages_;
  const std::vector<Span>* spans_ = nullptr;
  const fcg_lib* bound_ = nullptr;
  bool mapped_ = false, sent_ = false;
};

// After the call's pages are mapped: prepare the device copies of the page-table
// rows that change (appended to the blob): those of the new pages' sequences and
// of `seqs`.
void stage_pages(fcg_cache* c, const std::vector<std::pair<int32_t, int32_t>>& new_pages, Blob* blob,
                 std::vector<std::pair<int32_t, size_t>>* rows, std::vector<int32_t> seqs = {});

// Upload a plan: the staged page rows (at the front of the blob, in the order
// staged) into the device page table, the rest of the blob into the device ring,
// both read by one small kernel from the pinned ring.  *dev receives the blob's place
// in the device ring, which the caller retires after its last kernel.  staged (may be
// null) learns that page rows are on their way.
fcg_status upload(fcg_cache* c, const Blob& blob, const std::vector<std::pair<int32_t, size_t>>& rows, hipStream_t s,
                  char** dev, Staged* staged);

}  // namespace fcg

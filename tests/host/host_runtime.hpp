// The library's host side on a machine without a GPU: the HIP calls it makes, on
// ordinary memory, and its kernel launches, of which those that write the device page
// table do so and the others are only noted.  Any call or host allocation can be made
// to fail, by its number.
#pragma once

#include <sys/mman.h>

#include <cstdio>
#include <cstdlib>
#include <cstring>
#include <new>
#include <vector>

#include "objects.hpp"

namespace host {

// number of calls (allocations) until the one that fails; negative: none does
inline long fail_alloc = -1, fail_hip = -1;
inline bool capture = false;            // streams report a capture
inline int device = 0;                  // the current device
inline int launches = 0;                // kernels launched
inline int launch_device = -1;          // the device of the last one
inline bool next_hip_fails() { return fail_hip >= 0 && fail_hip-- == 0; }
inline hipError_t hip() { return next_hip_fails() ? hipErrorUnknown : hipSuccess; }
inline int launch() {
  if (next_hip_fails()) return (int)hipErrorUnknown;
  ++launches;
  launch_device = device;
  return 0;
}

// what launches were given
struct Apply {
  fcg::RopeRows rows;
  const int32_t* pos;
};
struct Append {
  fcg::RopeRows rows;
  int n_runs, n_groups;
  const fcg::AppendGroup* groups;
};
inline std::vector<Apply>* applies = nullptr;
inline std::vector<Append>* appends = nullptr;

}  // namespace host

void* operator new(size_t n) {
  if (host::fail_alloc >= 0 && host::fail_alloc-- == 0) throw std::bad_alloc();
  if (void* p = std::malloc(n ? n : 1)) return p;
  throw std::bad_alloc();
}
void* operator new(size_t n, const std::nothrow_t&) noexcept {
  if (host::fail_alloc >= 0 && host::fail_alloc-- == 0) return nullptr;
  return std::malloc(n ? n : 1);
}
void operator delete(void* p) noexcept { std::free(p); }
void operator delete(void* p, size_t) noexcept { std::free(p); }

extern "C" {
hipError_t hipGetDevice(int* d) { *d = host::device; return host::hip(); }
hipError_t hipSetDevice(int d) {
  if (host::next_hip_fails()) return hipErrorUnknown;
  host::device = d;
  return hipSuccess;
}
// (zeros; pages that nothing touches take no memory, so caches may be larger than the machine's)
hipError_t hipMalloc(void** p, size_t n) {
  if (host::next_hip_fails()) return hipErrorOutOfMemory;
  char* a = (char*)mmap(nullptr, n + 4096, PROT_READ | PROT_WRITE, MAP_PRIVATE | MAP_ANONYMOUS | MAP_NORESERVE, -1, 0);
  if (a == (char*)MAP_FAILED) return hipErrorOutOfMemory;
  *(size_t*)a = n + 4096;
  *p = a + 4096;
  return hipSuccess;
}
hipError_t hipHostMalloc(void** p, size_t n, unsigned) { return hipMalloc(p, n); }
hipError_t hipFree(void* p) {
  if (p) munmap((char*)p - 4096, *(size_t*)((char*)p - 4096));
  return hipSuccess;
}
hipError_t hipHostFree(void* p) { return hipFree(p); }
hipError_t hipMemset(void* p, int v, size_t n) { std::memset(p, v, n); return host::hip(); }
hipError_t hipMemcpy(void* d, const void* s, size_t n, hipMemcpyKind) { std::memcpy(d, s, n); return host::hip(); }
hipError_t hipMemcpy2DAsync(void*, size_t, const void*, size_t, size_t, size_t, hipMemcpyKind, hipStream_t) {
  return host::hip();
}
hipError_t hipMemGetInfo(size_t* f, size_t* t) { *f = *t = (size_t)1 << 38; return host::hip(); }
hipError_t hipDeviceSynchronize() { return hipSuccess; }
hipError_t hipGetLastError() { return hipSuccess; }
const char* hipGetErrorString(hipError_t) { return "made to fail"; }
hipError_t hipEventCreate(hipEvent_t* e) {
  if (host::next_hip_fails()) return hipErrorUnknown;
  *e = (hipEvent_t)std::malloc(1);
  return hipSuccess;
}
hipError_t hipEventCreateWithFlags(hipEvent_t* e, unsigned) { return hipEventCreate(e); }
hipError_t hipEventDestroy(hipEvent_t e) { std::free((void*)e); return hipSuccess; }
hipError_t hipEventRecord(hipEvent_t, hipStream_t) { return host::hip(); }
hipError_t hipEventSynchronize(hipEvent_t) { return hipSuccess; }
hipError_t hipEventElapsedTime(float* ms, hipEvent_t, hipEvent_t) { *ms = 0.f; return hipSuccess; }
hipError_t hipStreamWaitEvent(hipStream_t, hipEvent_t, unsigned) { return host::hip(); }
hipError_t hipStreamSynchronize(hipStream_t) { return hipSuccess; }
hipError_t hipStreamIsCapturing(hipStream_t, hipStreamCaptureStatus* st) {
  *st = host::capture ? hipStreamCaptureStatusActive : hipStreamCaptureStatusNone;
  return hipSuccess;
}
}

namespace fcg {

int launch_rope_table(const double*, int, int, float2*, hipStream_t) { return host::launch(); }
int launch_lib_ingest(int, const void*, const void*, void*, void*, int, int, int, int, int64_t, int64_t, hipStream_t) {
  return host::launch();
}
int launch_graft(int, const GraftChunk*, const GraftArgs&, int, const void*, const void*, int64_t, const CacheView&,
                 const double*, int, hipStream_t, KTime) {
  return host::launch();
}
int launch_graft_rope(int, bool, const GraftChunk*, const GraftArgs&, int, const void*, const void*, int64_t,
                      const CacheView&, const RopeArgs&, int, hipStream_t, KTime) {
  return host::launch();
}
int launch_upload(const UploadArgs& a, hipStream_t) {
  if (int rc = host::launch()) return rc;
  if (a.bytes) std::memcpy(a.dev, a.host, (size_t)a.bytes);
  for (int i = 0; i < a.n_rows; ++i)
    std::memcpy(a.page_table + (int64_t)a.seq[i] * a.row_ints, a.rows + i * a.row_stride, (size_t)a.row_ints * 4);
  return 0;
}
int launch_unalias(int, const UnaliasItem*, int, const void*, int64_t, const CacheView&, int, hipStream_t) {
  return host::launch();
}
int launch_rope_append(int, const TokenMeta*, int, const void*, const void*, const void*, const CacheView&, int,
                       const float2*, int, void*, hipStream_t, KTime) {
  return host::launch();
}
int launch_attn_mfma(const PrefillArgs&, const TokenMeta*, const void*, int, const CacheView&, int, int, void*, float*,
                     float*, int, int, hipStream_t, KTime, FusedIn, int) {
  return host::launch();
}
int launch_attn_rows(const AttnItem*, int, const TokenMeta*, const void*, int, const CacheView&, int, int, void*, float*,
                     float*, int, int, hipStream_t, KTime) {
  return host::launch();
}
int launch_combine(const CombineArgs&, const TokenMeta*, int, int, int, const float*, const float*, int, void*,
                   hipStream_t, bool, KTime) {
  return host::launch();
}
inline int enter_decoded(const DecodeArgs& a, const CacheView& cv) {
  if (int rc = host::launch()) return rc;
  for (int i = 0; i < a.n; ++i)
    if (a.new_page[i] >= 0) {
      int32_t* row = const_cast<int32_t*>(cv.page_table) + (int64_t)a.seq[i] * 2 * cv.n_lp + a.pos[i] / 16;
      row[0] = a.new_page[i];
      row[cv.n_lp] = -1;
    }
  return 0;
}
int launch_decode(const DecodeArgs& a, const void*, const void*, const void*, const CacheView& cv, int, const float2*, int,
                  void*, float*, float*, int*, hipStream_t, KTime) {
  return enter_decoded(a, cv);
}
int launch_decode_mfma(const DecodeArgs& a, const void*, const void*, const void*, const CacheView& cv, int, const float2*,
                       int, void*, float*, float*, int*, int, hipStream_t, KTime) {
  return enter_decoded(a, cv);
}
int noalloc_scratch(hipStream_t, void** base) {
  static std::vector<char> scratch(kNoAllocScratchBytes);
  *base = scratch.data();
  return host::next_hip_fails() ? (int)hipErrorUnknown : 0;
}
int launch_rope_apply(int, int, bool, const RopeRows& rows, const int32_t* pos, const RopeArgs&, hipStream_t) {
  if (int rc = host::launch()) return rc;
  if (host::applies) host::applies->push_back(host::Apply{rows, pos});
  return 0;
}
int launch_append(int, bool, const RopeRows& rows, const AppendArgs& args, int n_runs, const AppendGroup* groups,
                  int n_groups, const CacheView& cv, int, const RopeArgs&, const float2*, hipStream_t) {
  if (int rc = host::launch()) return rc;
  if (host::appends) host::appends->push_back(host::Append{rows, n_runs, n_groups, groups});
  for (int i = 0; !groups && i < n_runs; ++i) {
    const AppendRun& r = args.run[i];
    for (int p = r.pos0 / 16; r.page0 < 0 && p <= (r.pos0 + r.n - 1) / 16; ++p) {
      int32_t* row = const_cast<int32_t*>(cv.page_table) + (int64_t)r.seq * 2 * cv.n_lp + p;
      row[0] = args.page[(r.page0 & 0x7FFFFFFF) + p - r.pos0 / 16];
      row[cv.n_lp] = -1;
    }
  }
  return 0;
}
int launch_prefix_attend(int, const PrefixCall&, const PrefixArgs*, const PrefixItem*, const PrefixRank*, int, int,
                         const CacheView&, hipStream_t) {
  return host::launch();
}
int launch_prefix_merge(int, const PrefixCall&, const PrefixArgs*, const PrefixRank*, int, int, int, hipStream_t) {
  return host::launch();
}

}  // namespace fcg

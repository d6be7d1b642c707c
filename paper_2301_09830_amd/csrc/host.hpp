// Host helpers shared by the translation units of liboptcc: optional timing of
// every launch, and the checks of arguments.
#pragma once

#include <hip/hip_runtime.h>
#include <stddef.h>
#include <stdint.h>

#include <algorithm>
#include <vector>

#include "optcc.h"

namespace occ {

// ----------------------------------------------------------------------------
// optional per-kernel event timing
// ----------------------------------------------------------------------------
struct ProfRec {
  const char* name;
  hipEvent_t a, b;
};

struct Profiler {
  bool on = false;
  std::vector<ProfRec> recs;
  std::vector<hipEvent_t> free_events;

  hipEvent_t take() {
    if (!free_events.empty()) {
      hipEvent_t e = free_events.back();
      free_events.pop_back();
      return e;
    }
    hipEvent_t e = nullptr;
    if (hipEventCreate(&e) != hipSuccess) return nullptr;
    return e;
  }
};

inline Profiler g_prof;

template <typename F>
occ_status_t launch(const char* name, hipStream_t s, F&& f) {
  hipEvent_t a = nullptr;
  if (g_prof.on) {
    a = g_prof.take();
    if (a) (void)hipEventRecord(a, s);
  }
  f();
  const hipError_t e = hipGetLastError();
  if (g_prof.on && a) {
    hipEvent_t b = g_prof.take();
    if (b) {
      (void)hipEventRecord(b, s);
      g_prof.recs.push_back({name, a, b});
    }
  }
  return e == hipSuccess ? OCC_OK : OCC_E_HIP;
}

#define OCC_TRY(x)                       \
  do {                                   \
    const occ_status_t st_ = (x);        \
    if (st_ != OCC_OK) return st_;       \
  } while (0)

// ----------------------------------------------------------------------------
// validation helpers
// ----------------------------------------------------------------------------
struct Span {
  uintptr_t lo, hi;
  bool writable;
};

inline bool aligned(const void* p, size_t a) { return ((uintptr_t)p % a) == 0; }

inline size_t elem_size(int dt) { return dt == OCC_BF16 ? 2 : 4; }

inline Span span2d(const void* p, int64_t rows, int64_t cols, int64_t ld, size_t es, bool w) {
  const uintptr_t lo = (uintptr_t)p;
  return {lo, lo + (uintptr_t)(((rows - 1) * ld + cols) * (int64_t)es), w};
}

inline bool overlaps(std::vector<Span> v) {
  std::sort(v.begin(), v.end(), [](const Span& a, const Span& b) { return a.lo < b.lo; });
  // any writable interval must be disjoint from every other interval
  for (size_t i = 0; i < v.size(); ++i) {
    for (size_t j = i + 1; j < v.size() && v[j].lo < v[i].hi; ++j) {
      if (v[i].writable || v[j].writable) return true;
    }
  }
  return false;
}

constexpr int64_t kMaxDim = (int64_t)1 << 31;

inline occ_status_t check_shape(int64_t m, int64_t n, int64_t ld) {
  if (m < 1 || n < 1 || m >= kMaxDim || n >= kMaxDim) return OCC_E_SHAPE;
  if (ld < n || ld >= kMaxDim) return OCC_E_SHAPE;
  if (m * ld >= ((int64_t)1 << 46)) return OCC_E_SHAPE;
  return OCC_OK;
}

}  // namespace occ

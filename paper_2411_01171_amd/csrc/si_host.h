// Host side shared by the translation units of the library: stage timing, pointer checks, launch checks.
#pragma once
#include "../../include/si.h"

#include <hip/hip_runtime.h>

#include <vector>

namespace si {

struct StageEvent {
  int stage;
  hipEvent_t a, b;
};
extern bool g_timing;
extern std::vector<StageEvent> g_events;
int stage_id(const char* name);

struct StageScope {
  hipStream_t st;
  StageEvent ev;
  bool on;
  StageScope(const char* name, hipStream_t s) : st(s), on(g_timing) {
    if (!on) return;
    ev.stage = stage_id(name);
    if (hipEventCreate(&ev.a) != hipSuccess || hipEventCreate(&ev.b) != hipSuccess) {
      on = false;
      return;
    }
    (void)hipEventRecord(ev.a, st);
  }
  ~StageScope() {
    if (!on) return;
    (void)hipEventRecord(ev.b, st);
    g_events.push_back(ev);
  }
};

static inline size_t align_up(size_t v, size_t a) { return (v + a - 1) / a * a; }
static inline bool aligned16(const void* p) { return (reinterpret_cast<uintptr_t>(p) & 15u) == 0; }
static bool ranges_overlap(const void* a, size_t na, const void* b, size_t nb) {
  const uintptr_t a0 = reinterpret_cast<uintptr_t>(a), b0 = reinterpret_cast<uintptr_t>(b);
  return a0 < b0 + nb && b0 < a0 + na;
}

#define SI_CHECK_LAUNCH()                         \
  do {                                            \
    if (hipGetLastError() != hipSuccess) return SI_ERR_HIP; \
  } while (0)

#define SI_TRY(expr)                  \
  do {                                \
    si_status st__ = (expr);          \
    if (st__ != SI_OK) return st__;   \
  } while (0)

}  // namespace si

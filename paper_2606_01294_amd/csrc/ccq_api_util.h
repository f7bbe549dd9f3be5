// ccq_api_util.h -- helpers shared by the files that implement the C ABI: the
// timing hook, type sizes and pointer checks.  Internal.
#pragma once
#include <hip/hip_runtime.h>

#include "ccq.h"

namespace ccq_api {

// Per-host-thread kernel timing hook (ccq_trace_events).
struct Trace {
  hipEvent_t* ev = nullptr;
  int n = 0;
  int next = 0;
  bool nested = false;  // inside an entry point that wraps another one
};
inline thread_local Trace g_trace;

inline void trace_begin_call() {
  if (!g_trace.nested) g_trace.next = 0;
}
// An entry point built on another one numbers its own launches and the inner
// call's in one sequence.
struct TraceScope {
  TraceScope() {
    trace_begin_call();
    g_trace.nested = true;
  }
  ~TraceScope() { g_trace.nested = false; }
};

// Runs one launcher between the trace events of its slot, if tracing is on.
template <typename F>
hipError_t traced(hipStream_t st, F&& launch) {
  const int i = g_trace.next++;
  const bool on = g_trace.ev && 2 * i + 1 < g_trace.n;
  if (on && hipEventRecord(g_trace.ev[2 * i], st) != hipSuccess) return hipErrorUnknown;
  hipError_t e = launch();
  if (e == hipSuccess && on && hipEventRecord(g_trace.ev[2 * i + 1], st) != hipSuccess)
    return hipErrorUnknown;
  return e;
}

constexpr size_t kAlign = 256;
inline size_t align_up(size_t x) { return (x + kAlign - 1) / kAlign * kAlign; }

inline size_t esize(ccq_dtype d) { return d == CCQ_BF16 ? 2 : 4; }
inline bool dtype_ok(ccq_dtype d) { return d == CCQ_F32 || d == CCQ_BF16; }
inline bool aligned(const void* p) { return (reinterpret_cast<uintptr_t>(p) & 15u) == 0; }

}  // namespace ccq_api

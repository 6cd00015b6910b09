// What every entry point enqueues through: the HIP error report and the optional kernel timing.
#pragma once
#include <cstdio>
#include <mutex>
#include <vector>

#include "nf_internal.h"

// A HIP error while enqueueing is reported on stderr with the failing expression (the status code
// alone cannot say which launch it was), then returned as NF_ERR_DEVICE.
#define NF_HIP(expr)                                                                     \
  do {                                                                                   \
    const hipError_t e_ = (expr);                                                        \
    if (e_ != hipSuccess) {                                                              \
      std::fprintf(stderr, "libnf: %s: %s\n", hipGetErrorString(e_), #expr);             \
      return NF_ERR_DEVICE;                                                              \
    }                                                                                    \
  } while (0)

namespace nf {
// ---- optional kernel timing (nf_prof_begin / nf_prof_end): one HIP-event pair per launch ----
struct ProfEvent {
  const char *name;
  hipEvent_t a, b;
  double flops, bytes;
};
struct ProfState {
  bool on = false;
  bool apart = false;  // kernels that share a launch are launched one by one
  std::vector<ProfEvent> ev;
  std::mutex mu;  // guards ev: launches from several host threads may record while profiling is on
};
extern ProfState g_prof;

struct ProfScope {
  hipStream_t st;
  hipEvent_t a = nullptr, b = nullptr;
  bool on;
  explicit ProfScope(hipStream_t s) : st(s), on(g_prof.on) {
    if (on) {
      on = hipEventCreate(&a) == hipSuccess && hipEventCreate(&b) == hipSuccess && hipEventRecord(a, st) == hipSuccess;
    }
  }
  void done(const char *name, double flops, double bytes) {
    if (on && hipEventRecord(b, st) == hipSuccess) {
      std::lock_guard<std::mutex> lk(g_prof.mu);
      g_prof.ev.push_back({name, a, b, flops, bytes});
    }
  }
};

// The same for a file that has its launches to itself: a launch, its error, its record.
template <typename F>
inline hipError_t recorded(hipStream_t st, const char *name, double flops, double bytes, F launch) {
  ProfScope sc(st);
  launch();
  const hipError_t e = hipGetLastError();
  if (e == hipSuccess) sc.done(name, flops, bytes);
  return e;
}

}  // namespace nf

#define NF_RUN(st, name, flops, bytes, call) \
  do {                                       \
    ProfScope sc_(st);                       \
    NF_HIP(call);                            \
    sc_.done(name, flops, bytes);            \
  } while (0)


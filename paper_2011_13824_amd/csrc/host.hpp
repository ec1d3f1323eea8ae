// Host side shared by the translation units of liblirpa.so: the error message of a thread's last
// failed call, and the event pairs of lirpa_timing_begin / lirpa_timing_end.
#pragma once

#include <hip/hip_runtime.h>

#include <cstdarg>
#include <cstdio>
#include <string>
#include <vector>

#include "lirpa.h"

namespace lirpa_host {

inline thread_local std::string g_err;

// Never throws: it ends the C entries, the one for sizes too.  Without memory for it the message is
// left out.
inline int fail(int code, const char* fmt, ...) noexcept {
  char buf[512];
  va_list ap;
  va_start(ap, fmt);
  vsnprintf(buf, sizeof buf, fmt, ap);
  va_end(ap);
  try {
    g_err = buf;
  } catch (...) {
    g_err.clear();
  }
  return code;
}

// Kernel timing (lirpa_timing_begin / lirpa_timing_end): event pairs around every launch.
struct TimingRec {
  std::string cls;
  size_t ev;  // index of the first event of the pair in the pool
};
struct TimingState {
  bool on = false;
  std::vector<hipEvent_t> pool;
  size_t used = 0;
  std::vector<TimingRec> recs;
};
inline thread_local TimingState g_tim;

// Enqueue one kernel through `launch`, bracketed by events when timing is on.
template <typename F>
int launch_k(const std::string& cls, hipStream_t st, F&& launch) {
  size_t ev = 0;
  if (g_tim.on) {
    while (g_tim.pool.size() < g_tim.used + 2) {
      hipEvent_t e;
      if (hipEventCreate(&e) != hipSuccess) return fail(LIRPA_EDEVICE, "hipEventCreate failed");
      g_tim.pool.push_back(e);
    }
    ev = g_tim.used;
    g_tim.used += 2;
    if (hipEventRecord(g_tim.pool[ev], st) != hipSuccess)
      return fail(LIRPA_EDEVICE, "hipEventRecord failed");
  }
  launch();
  hipError_t e = hipGetLastError();
  if (e != hipSuccess) return fail(LIRPA_EDEVICE, "%s: %s", cls.c_str(), hipGetErrorString(e));
  if (g_tim.on) {
    if (hipEventRecord(g_tim.pool[ev + 1], st) != hipSuccess)
      return fail(LIRPA_EDEVICE, "hipEventRecord failed");
    g_tim.recs.push_back(TimingRec{cls, ev});
  }
  return LIRPA_OK;
}

}  // namespace lirpa_host

// What the files with C entry points share: refusals, which become a status and a text, and the guard around every call.
#pragma once

#include <new>
#include <string>

#include "common.h"

namespace hyp {
namespace {

thread_local std::string t_error;  // of this file's entry points

struct Refused {
  hyp_status_t status;
  const char *text;
};
inline void need(bool ok, hyp_status_t status, const char *text) {
  if (!ok) throw Refused{status, text};
}

// A launch has fewer than 2^32 lanes; one that is refused would leave the launches after it without what it writes.
inline void check_launch(int64_t workgroups, int threads) { need(workgroups < (1ll << 32) / threads, HYP_ESHAPE, "too much work for a launch"); }

inline bool apart(int64_t stride, int64_t n) { return n <= 1 || stride != 0; }

inline bool aligned(const void *p, int64_t to) { return (uintptr_t)p % to == 0; }

inline void run(hipError_t e) {
  if (e != hipSuccess) {
    t_error = std::string("HIP: ") + hipGetErrorString(e);
    throw Refused{HYP_EDEVICE, nullptr};
  }
}

// No exception may cross the C ABI.
template <typename F> hyp_status_t guarded(F &&body) {
  try {
    try {
      body();
      return HYP_OK;
    } catch (const Refused &r) {
      if (r.text) t_error = r.text;
      return r.status;
    }
  } catch (const std::bad_alloc &) {
    return HYP_ENOMEM;
  } catch (...) {
    return HYP_EDEVICE;
  }
}

}  // namespace
}  // namespace hyp

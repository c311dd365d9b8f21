// Host helpers shared by the C entry points: the per-thread error message,
// error mapping, pointer checks and roctx ranges.
#pragma once

#include <hip/hip_runtime.h>
#include <rocprofiler-sdk-roctx/roctx.h>

#include <cstdarg>
#include <cstdint>
#include <cstdio>
#include <cstdlib>
#include <mutex>
#include <new>
#include <set>
#include <string>
#include <utility>

#include "../../include/mtdao.h"

namespace mtdao {

// Message of the last failing call without a handle on this thread
// (mtdao_last_error(NULL)); defined in mtdao.hip.
extern thread_local std::string g_err;

// roctx ranges around every enqueueing call, for timelines of
// rocprofv3 --marker-trace: on when MTDAO_ROCTX=1 in the environment.
inline bool roctx_on() {
  static const bool on = [] {
    const char* e = std::getenv("MTDAO_ROCTX");
    return e != nullptr && e[0] == '1';
  }();
  return on;
}

struct RoctxRange {
  bool on;
  explicit RoctxRange(const char* fmt, ...) : on(roctx_on()) {
    if (!on) return;
    char buf[128];
    va_list ap;
    va_start(ap, fmt);
    vsnprintf(buf, sizeof buf, fmt, ap);
    va_end(ap);
    roctxRangePushA(buf);
  }
  ~RoctxRange() {
    if (on) roctxRangePop();
  }
};

// The code, with a message in sink; no message where there is no memory for one
// (nothing is thrown: this runs at C entries, and in their catch blocks).
inline int32_t fail(std::string* sink, int32_t code, const char* fmt, ...) noexcept {
  char buf[512];
  va_list ap;
  va_start(ap, fmt);
  vsnprintf(buf, sizeof buf, fmt, ap);
  va_end(ap);
  try {
    *sink = buf;
  } catch (...) {
    sink->clear();
  }
  return code;
}

inline int64_t esize(int32_t dt) { return dt == MTDAO_BF16 ? 2 : 4; }  // bytes of an element
inline size_t up256(size_t n) { return (n + 255) / 256 * 256; }

inline bool aligned_to(const void* p, uintptr_t n) { return (reinterpret_cast<uintptr_t>(p) & (n - 1)) == 0; }
inline bool aligned16(const void* p) { return aligned_to(p, 16); }

// Non-overlap of two [lo, lo + bytes) device ranges.
inline bool overlap(const void* a, int64_t abytes, const void* b, int64_t bbytes) {
  const uintptr_t a0 = (uintptr_t)a, b0 = (uintptr_t)b;
  return a0 < b0 + (uintptr_t)bbytes && b0 < a0 + (uintptr_t)abytes;
}

// A grid of at least n workgroups of up to 1024 threads: a launch takes fewer than
// 2^32 threads along x (and 65535 rows of workgroups along y).
inline constexpr int64_t kGridRow = INT64_C(1) << 21, kGridMost = kGridRow * 65535;
inline dim3 grid_of(int64_t n) {
  const int64_t y = n > kGridRow ? (n + kGridRow - 1) / kGridRow : 1;
  return dim3((unsigned)(y > 1 ? kGridRow : n), (unsigned)y);
}

inline int32_t hip_check(std::string* e, hipError_t r, const char* what) {
  if (r != hipSuccess) return fail(e, MTDAO_ERR_HIP, "%s: %s", what, hipGetErrorString(r));
  return MTDAO_OK;
}

// More than 64 KiB of LDS for a kernel, asked for once per kernel and device.
inline int32_t allow_lds(const void* kernel, int bytes, std::string* e) try {
  static std::mutex lock;
  static std::set<std::pair<const void*, int>> done;
  int device = 0;
  int32_t r = hip_check(e, hipGetDevice(&device), "device");
  if (r != MTDAO_OK) return r;
  std::lock_guard<std::mutex> held(lock);
  if (done.count({kernel, device})) return MTDAO_OK;
  r = hip_check(e, hipFuncSetAttribute(kernel, hipFuncAttributeMaxDynamicSharedMemorySize, bytes), "LDS of a kernel");
  if (r == MTDAO_OK) done.insert({kernel, device});
  return r;
} catch (const std::bad_alloc&) {
  return fail(e, MTDAO_ERR_WORKSPACE, "out of host memory");
}

}  // namespace mtdao

// What the C entry points over a paged cache share: the device of a call's stream, and checks of their arguments.
#pragma once

#include <hip/hip_runtime.h>
#include <stdint.h>

#include "api_status.h"

namespace cosa {

// Makes the device of `stream` current for the launches of one call (null, legacy and per-thread streams belong to the current device).
class OnDevice {
 public:
  explicit OnDevice(hipStream_t stream) {
    // the null stream, the legacy and the per-thread one belong to whichever device is current
    if (stream == nullptr || stream == hipStreamLegacy || stream == hipStreamPerThread) return;
    hipDevice_t dev;
    if ((err_ = hipGetDevice(&before_)) != hipSuccess) return;
    if ((err_ = hipStreamGetDevice(stream, &dev)) != hipSuccess) return;
    if ((int)dev == before_) return;
    err_ = hipSetDevice((int)dev);
    moved_ = err_ == hipSuccess;
  }
  ~OnDevice() {
    if (moved_) (void)hipSetDevice(before_);
  }
  OnDevice(const OnDevice&) = delete;
  OnDevice& operator=(const OnDevice&) = delete;
  hipError_t error() const { return err_; }

 private:
  int before_ = 0;
  bool moved_ = false;
  hipError_t err_ = hipSuccess;
};

template <class F>
cosa_status launch(void* stream, const char* what, F&& f) {
  const hipStream_t s = as_stream(stream);
  const OnDevice device(s);
  hipError_t e = device.error();
  if (e != hipSuccess) return hip_fail(e, "device of the stream");
  e = f(s);
  return e == hipSuccess ? ok() : hip_fail(e, what);
}

inline bool misaligned(const void* p, size_t to) { return reinterpret_cast<uintptr_t>(p) % to != 0; }

// A range of memory that a call reads or writes.
struct Span {
  const void* p;
  int64_t bytes;
  bool meets(const Span& o) const {
    const uintptr_t a = reinterpret_cast<uintptr_t>(p), b = reinterpret_cast<uintptr_t>(o.p);
    return p && o.p && bytes > 0 && o.bytes > 0 && a < b + (uintptr_t)o.bytes && b < a + (uintptr_t)bytes;
  }
};

inline cosa_status check_page_size(int ps, int& log2_page) {
  if (ps < 16 || ps > (1 << 20) || (ps & (ps - 1)) != 0)
    return fail(COSA_ERR_INVALID_ARG, "page_size %d is not a power of two in [16, 2^20]", ps);
  log2_page = 0;
  while ((1 << log2_page) < ps) ++log2_page;
  return ok();
}

inline cosa_status check_n_pages(int64_t n) {
  if (n < 1 || n > (1ll << 31))
    return fail(COSA_ERR_INVALID_ARG, "n_pages (%lld) outside [1, 2^31]", (long long)n);
  return ok();
}

inline cosa_status check_workspace(const void* ws, size_t bytes, size_t need) {
  if (!ws || bytes < need) return fail(COSA_ERR_WORKSPACE, "workspace of %zu bytes at %p, need %zu", bytes, ws, need);
  if (misaligned(ws, 16)) return fail(COSA_ERR_INVALID_ARG, "workspace must be 16-byte aligned");
  return ok();
}

inline const uint16_t* u16(const void* p) { return static_cast<const uint16_t*>(p); }

}  // namespace cosa

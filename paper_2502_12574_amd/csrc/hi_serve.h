// What the entry points of a served batch share on the host.
#pragma once
#include <hip/hip_runtime.h>
#include "hi_internal.h"

namespace hi {

inline bool aligned_to(const void* p, uintptr_t n) { return (reinterpret_cast<uintptr_t>(p) & (n - 1)) == 0; }

// A launch goes to a stream of the current device: makes the stream's device current for the call.
class StreamDevice {
 public:
  explicit StreamDevice(void* stream) {
    int now = 0;
    hipDevice_t wanted = 0;
    if (stream == nullptr || hipGetDevice(&now) != hipSuccess || hipStreamGetDevice((hipStream_t)stream, &wanted) != hipSuccess) return;
    if (wanted != now && hipSetDevice(wanted) == hipSuccess) before_ = now;
  }
  ~StreamDevice() {
    if (before_ >= 0) (void)hipSetDevice(before_);
  }
  StreamDevice(const StreamDevice&) = delete;
  StreamDevice& operator=(const StreamDevice&) = delete;

 private:
  int before_ = -1;
};

inline hi_status launched(const char* what) {
  const hipError_t e = hipGetLastError();
  if (e == hipSuccess) return HI_OK;
  set_last_error("%s launch: %s", what, hipGetErrorString(e));
  return HI_ERR_HIP;
}

}  // namespace hi

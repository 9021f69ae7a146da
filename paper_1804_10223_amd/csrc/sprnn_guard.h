// What every C entry point does around its HIP calls: name a failing one when asked to, work on the caller's device.
#ifndef SPRNN_GUARD_H_
#define SPRNN_GUARD_H_

#include <hip/hip_runtime.h>

#include <cstdio>
#include <cstdlib>

namespace sprnn {

// With SPRNN_DEBUG set in the environment, a failing HIP call is named on stderr.
inline bool hip_ok(hipError_t e, const char* what) {
  if (e == hipSuccess) return true;
  static const bool verbose = std::getenv("SPRNN_DEBUG") != nullptr;
  if (verbose) std::fprintf(stderr, "sprnn: %s failed: %s\n", what, hipGetErrorString(e));
  (void)hipGetLastError();
  return false;
}
#define SPRNN_HIP(call) hip_ok((call), #call)

struct DeviceGuard {
  int prev = -1;
  bool ok = false;
  explicit DeviceGuard(int dev) {
    if (!SPRNN_HIP(hipGetDevice(&prev))) return;
    ok = (prev == dev) || SPRNN_HIP(hipSetDevice(dev));
    if (prev == dev) prev = -1;
  }
  ~DeviceGuard() { if (prev >= 0) (void)hipSetDevice(prev); }
};

}  // namespace sprnn
#endif

// Host-side helpers shared by the C ABI's sources.
#pragma once

#include <stddef.h>
#include <stdint.h>

#include "../../include/vda.h"

namespace vda {

constexpr int kMaxDevices = 64;

inline bool supported_dim(int d) { return d == 32 || d == 64 || d == 128; }

inline size_t round_up(size_t x, size_t a) { return (x + a - 1) / a * a; }

inline bool aligned(const void* p, uintptr_t a) { return (reinterpret_cast<uintptr_t>(p) % a) == 0; }

struct Range {
  uintptr_t lo, hi;  // [lo, hi)
};

inline Range range_of(const void* p, size_t bytes) {
  const uintptr_t lo = reinterpret_cast<uintptr_t>(p);
  return Range{lo, lo + bytes};
}

inline bool overlaps(Range a, Range b) { return a.lo < b.hi && b.lo < a.hi; }

inline int hip_status(hipError_t e) { return e == hipSuccess ? VDA_OK : VDA_ERR_HIP; }

inline int current_device_cus() {
  static int cus[kMaxDevices] = {0};
  int dev = 0;
  if (hipGetDevice(&dev) != hipSuccess || dev < 0 || dev >= kMaxDevices) return 256;
  if (cus[dev] == 0) {
    int c = 0;
    if (hipDeviceGetAttribute(&c, hipDeviceAttributeMultiprocessorCount, dev) != hipSuccess || c <= 0)
      c = 256;
    cus[dev] = c;
  }
  return cus[dev];
}

}  // namespace vda

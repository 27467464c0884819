// Host only: the GPU's number of CUs.
#pragma once

#include <hip/hip_runtime_api.h>

namespace tr {

// CUs of the current device (the tile-shape choice counts rounds of them), asked for once by
// whichever thread comes first.
inline int cu_count() {
  static const int n = [] {
    int dev = 0, v = 0;
    return hipGetDevice(&dev) == hipSuccess &&
                   hipDeviceGetAttribute(&v, hipDeviceAttributeMultiprocessorCount, dev) == hipSuccess && v > 0
               ? v
               : 256;
  }();
  return n;
}

}  // namespace tr

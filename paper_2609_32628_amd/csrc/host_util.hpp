// Host helpers shared by the library's entry points. Internal to libda2.
#pragma once

#include <hip/hip_runtime.h>

#include <atomic>
#include <cstring>

#include "../../include/da2.h"

namespace da2 {

// gfx950 check, cached per device ordinal (0 unknown, 1 ok, 2 unsupported).
inline std::atomic<int8_t> g_arch_ok[64];

inline int32_t check_device() {
  int dev = -1;
  if (hipGetDevice(&dev) != hipSuccess || dev < 0) return DA2_ERR_UNSUPPORTED;
  if (dev < 64) {
    int8_t c = g_arch_ok[dev].load(std::memory_order_relaxed);
    if (c == 1) return DA2_OK;
    if (c == 2) return DA2_ERR_UNSUPPORTED;
  }
  hipDeviceProp_t prop;
  if (hipGetDeviceProperties(&prop, dev) != hipSuccess) return DA2_ERR_HIP;
  const bool ok = std::strncmp(prop.gcnArchName, "gfx950", 6) == 0;
  if (dev < 64) g_arch_ok[dev].store(ok ? 1 : 2, std::memory_order_relaxed);
  return ok ? DA2_OK : DA2_ERR_UNSUPPORTED;
}

inline int32_t hip_status(hipError_t e) { return e == hipSuccess ? DA2_OK : DA2_ERR_HIP; }

}  // namespace da2

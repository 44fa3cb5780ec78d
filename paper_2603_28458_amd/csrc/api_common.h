// Host-side helpers that the translation units of the C ABI share: limits, checks, launch status.
#pragma once

#include <hip/hip_runtime.h>
#include <stdint.h>

#include <atomic>

#include "../../include/hisa.h"

namespace hisa {

inline long round_up(long x, long a) { return (x + a - 1) / a * a; }
inline bool aligned16(const void* p) { return (reinterpret_cast<uintptr_t>(p) & 15u) == 0; }
inline int launch_status() { return hipGetLastError() == hipSuccess ? HISA_OK : HISA_ERR_LAUNCH; }

constexpr int kMaxK = 8192, kMaxM = 1024, kMaxCand = 65536;
constexpr int kMaxT = 1 << 22;        // queries per call
constexpr int kMaxSeq = 65535;        // sequences per key array (the y extent of the pooling grids)
constexpr long kMaxGrid = 1L << 30;   // workgroups per launch (the x extent of a grid stops at 2^31 - 1)
constexpr int kMaxDevices = 64;

// A kernel that asks for more than 64 KB of dynamic LDS needs its limit raised first.  Done once
// per kernel instance and device (again only if a later call needs more than any earlier one), not
// on every call.
template <auto Kern>
int raise_lds_limit(size_t bytes) {
  static std::atomic<int> granted[kMaxDevices];
  int dev = 0;
  if (hipGetDevice(&dev) != hipSuccess || dev < 0 || dev >= kMaxDevices) return HISA_ERR_LAUNCH;
  if ((int)bytes <= granted[dev].load(std::memory_order_acquire)) return HISA_OK;
  if (hipFuncSetAttribute(reinterpret_cast<const void*>(Kern), hipFuncAttributeMaxDynamicSharedMemorySize,
                          (int)bytes) != hipSuccess)
    return HISA_ERR_LAUNCH;
  granted[dev].store((int)bytes, std::memory_order_release);
  return HISA_OK;
}

}  // namespace hisa

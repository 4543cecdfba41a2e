// What every entry point that launches kernels needs: facts of the device, the launch call itself.  Host code only.
#pragma once

#include <hip/hip_runtime.h>
#include <stdint.h>
#include <stdlib.h>

#include <mutex>
#include <tuple>
#include <utility>

#include "../../include/swz.h"
#include "transpose_dispatch.h"

namespace swz {

constexpr int kCusPerXcd = 32;   // gfx950: 8 XCDs x 32 CUs
constexpr int kMaxDevices = 64;
constexpr int kWholeCus = 256;   // compute units assumed where no device can be asked (a whole MI355X)

struct DeviceFacts {
  bool known = false;
  int num_xcd = 0, cus = 0, l2_bytes = 0, lds_bytes = 0;   // num_xcd 0: could not be derived
};
inline DeviceFacts g_facts[kMaxDevices];
inline std::mutex g_mu;

// SWZ_NUM_XCD in the environment (read once per process): the XCD count to assume instead of the
// one derived from the CU count, for partitioned devices.  0 = not set or not a number in 1..1024.
inline int env_num_xcd() {
  static const int value = [] {
    const char* e = getenv("SWZ_NUM_XCD");
    if (e == nullptr || *e == 0) return 0;
    char* end = nullptr;
    const long v = strtol(e, &end, 10);
    return (end != nullptr && *end == 0 && v >= 1 && v <= 1024) ? (int)v : 0;
  }();
  return value;
}

inline int query_device(DeviceFacts* out) {
  int dev = 0;
  if (hipGetDevice(&dev) != hipSuccess || dev < 0 || dev >= kMaxDevices) return SWZ_ERR_HIP;
  std::lock_guard<std::mutex> lock(g_mu);
  DeviceFacts& f = g_facts[dev];
  if (!f.known) {
    int cus = 0, l2 = 0, lds = 0;
    if (hipDeviceGetAttribute(&cus, hipDeviceAttributeMultiprocessorCount, dev) != hipSuccess) return SWZ_ERR_HIP;
    if (hipDeviceGetAttribute(&l2, hipDeviceAttributeL2CacheSize, dev) != hipSuccess) return SWZ_ERR_HIP;
    if (hipDeviceGetAttribute(&lds, hipDeviceAttributeMaxSharedMemoryPerBlock, dev) != hipSuccess) return SWZ_ERR_HIP;
    f.cus = cus;
    f.l2_bytes = l2;
    f.lds_bytes = lds;
    // XCDs come in whole units of 32 CUs (a partitioned device exposes fewer of them); any other
    // CU count is not guessed at: the caller then has to name the XCD count.
    if (env_num_xcd() > 0) f.num_xcd = env_num_xcd();
    else f.num_xcd = (cus >= kCusPerXcd && cus % kCusPerXcd == 0) ? cus / kCusPerXcd : 0;
    f.known = true;
  }
  *out = f;
  return SWZ_OK;
}

// Launch through the call that returns the launch's own status: hipGetLastError() after a launch
// would also report (and clear) an error some earlier, unrelated HIP call left behind.
template <class... KArgs, size_t... Is>
int launch_impl(void (*kernel)(KArgs...), dim3 grid, dim3 block, size_t lds, hipStream_t stream,
                std::tuple<KArgs...>& vals, std::index_sequence<Is...>) {
  void* ptrs[] = {static_cast<void*>(&std::get<Is>(vals))...};
  return hipLaunchKernel(reinterpret_cast<const void*>(kernel), grid, block, ptrs, lds, stream) == hipSuccess ? SWZ_OK
                                                                                                             : SWZ_ERR_HIP;
}
template <class... KArgs, class... Args>
int launch(void (*kernel)(KArgs...), dim3 grid, dim3 block, size_t lds, hipStream_t stream, Args... args) {
  static_assert(sizeof...(KArgs) == sizeof...(Args), "argument count");
  if ((int64_t)grid.x * block.x > kLaunchThreads) return SWZ_ERR_OVERFLOW;
  std::tuple<KArgs...> vals{static_cast<KArgs>(args)...};
  return launch_impl(kernel, grid, block, lds, stream, vals, std::index_sequence_for<KArgs...>{});
}

}  // namespace swz

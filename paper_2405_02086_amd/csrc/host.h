// mlproj: what the host code of every translation unit shares: kernel launches and their status, the
// device's size, the per-kernel trace.
#ifndef MLPROJ_HOST_H
#define MLPROJ_HOST_H

#include <hip/hip_runtime.h>

#include <atomic>
#include <cstdint>
#include <tuple>
#include <utility>

#include "../../include/mlproj.h"

namespace mlproj {

inline bool aligned(const void* p, size_t a) { return (reinterpret_cast<uintptr_t>(p) % a) == 0; }

// Every kernel goes out through hipLaunchKernel, whose return value is the status of that launch
// alone: the process-wide "last error" of the HIP runtime, which an unrelated earlier call of the
// application may have set, is neither read nor cleared.  A refused launch is remembered for the
// calling thread until the entry point returns (launch_status), which also stops what the call
// had still to enqueue from going out behind it.
inline thread_local bool g_launch_refused = false;

template <typename... KArgs, typename... Args>
inline void launch(void (*kernel)(KArgs...), dim3 grid, dim3 block, hipStream_t stream, Args&&... args) {
  static_assert(sizeof...(KArgs) == sizeof...(Args), "one argument per kernel parameter");
  if (g_launch_refused) return;
  std::tuple<std::decay_t<KArgs>...> held(static_cast<std::decay_t<KArgs>>(args)...);
  const hipError_t e = std::apply(
      [&](auto&... a) {
        void* ptrs[] = {static_cast<void*>(&a)...};
        return hipLaunchKernel(reinterpret_cast<const void*>(kernel), grid, block, ptrs, 0, stream);
      },
      held);
  if (e != hipSuccess) g_launch_refused = true;
}

inline int launch_status() {
  const bool refused = g_launch_refused;
  g_launch_refused = false;
  return refused ? MLPROJ_ERR_LAUNCH : MLPROJ_OK;
}

// Compute units of the current device (0 when there is none to ask).  A device's count never
// changes, so it is asked for once per device and remembered.
inline int compute_units() {
  constexpr int MAX_DEVICES = 64;
  static std::atomic<int> known[MAX_DEVICES];   // 0: not asked yet
  int dev = -1, cus = 0;
  if (hipGetDevice(&dev) != hipSuccess || dev < 0) return 0;
  if (dev < MAX_DEVICES && (cus = known[dev].load(std::memory_order_relaxed)) > 0) return cus;
  if (hipDeviceGetAttribute(&cus, hipDeviceAttributeMultiprocessorCount, dev) != hipSuccess || cus <= 0) return 0;
  if (dev < MAX_DEVICES) known[dev].store(cus, std::memory_order_relaxed);
  return cus;
}

// Optional per-kernel timing: while a trace is open on the calling thread, an event is
// recorded on the stream before every kernel of a call and after its last one.
struct Trace {
  hipEvent_t* events = nullptr;
  int capacity = 0;
  int count = 0;
};
inline thread_local Trace g_trace;

inline void mark(hipStream_t stream) {
  if (g_trace.events && g_trace.count < g_trace.capacity)
    (void)hipEventRecord(g_trace.events[g_trace.count++], stream);
}

}  // namespace mlproj
#endif

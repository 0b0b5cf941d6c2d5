// Host helpers of the context-free operators that live outside thinfer_api.cu: error text, launch, device queries.
#pragma once
#include <cuda_runtime.h>
#include <stdint.h>

#include <cstdarg>
#include <cstdio>

#include "../../include/thinfer.h"
#include "smem_opt_in.cuh"

namespace thinfer {

// Text that thinfer_last_error(NULL) returns (thread-local; defined in thinfer_api.cu).
void op_set_error(const char* text) noexcept;

inline int op_fail(int code, const char* fmt, ...) {
  char buf[256];
  va_list ap;
  va_start(ap, fmt);
  vsnprintf(buf, sizeof(buf), fmt, ap);
  va_end(ap);
  op_set_error(buf);
  return code;
}

// The opt-in of one kernel to dynamic shared memory (a function-local static per kernel instantiation), on each device that
// it is launched on.
struct SmemOptIn {
  static constexpr int kMaxDevices = SmemAllowance::kMaxDevices;
  SmemAllowance allowance;
  template <typename K>
  bool ensure(K kernel, int bytes) {
    int dev = 0;
    if (cudaGetDevice(&dev) != cudaSuccess) dev = -1;
    return allowance.ensure(dev, bytes, [&](int n) { return cudaFuncSetAttribute(kernel, cudaFuncAttributeMaxDynamicSharedMemorySize, n) == cudaSuccess; });
  }
};

// SM count of the current device (asked once per device).
int op_sm_count();

// One launch, chained to its predecessor in the stream by programmatic dependent launch: the kernel may be scheduled while
// the predecessor is still running and waits for it (pdl_wait) before it touches anything in memory.
// Kernels launched this way read what earlier kernels may write with ordinary loads, never through the read-only path:
// the data need not be final when the kernel starts.
template <typename... KArgs, typename... Args>
int op_launch(void (*kernel)(KArgs...), dim3 grid, dim3 block, size_t smem, cudaStream_t st, Args&&... args) {
  cudaLaunchConfig_t lc{};
  lc.gridDim = grid;
  lc.blockDim = block;
  lc.dynamicSmemBytes = smem;
  lc.stream = st;
  cudaLaunchAttribute attr[1];
  lc.attrs = attr;
  attr[0].id = cudaLaunchAttributeProgrammaticStreamSerialization;
  attr[0].val.programmaticStreamSerializationAllowed = 1;
  lc.numAttrs = 1;
  const cudaError_t e = cudaLaunchKernelEx(&lc, kernel, static_cast<KArgs>(args)...);
  if (e != cudaSuccess) return op_fail(THINFER_ECUDA, "kernel launch failed: %s", cudaGetErrorString(e));
  return THINFER_OK;
}

inline bool aligned16(const void* p) { return (reinterpret_cast<uintptr_t>(p) & 15u) == 0; }
inline bool aligned8(const void* p) { return (reinterpret_cast<uintptr_t>(p) & 7u) == 0; }
inline bool aligned4(const void* p) { return (reinterpret_cast<uintptr_t>(p) & 3u) == 0; }

}  // namespace thinfer

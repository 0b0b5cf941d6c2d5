// Host helpers of the context-free operators that live outside thinfer_api.cu: error text, launch, device queries.
#pragma once
#include <cuda.h>
#include <cuda_runtime.h>
#include <stdint.h>

#include <cstdarg>
#include <cstdio>
#include <initializer_list>

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

// Tensor map of 32-bit words [d2][d1][d0], rows of d0 side by side, boxes [box2][1][d0], nothing swizzled, 0 outside.
bool op_tensor_map(CUtensorMap* map, const void* base, uint64_t d0, uint64_t d1, uint64_t d2, uint32_t box2);

// One launch, chained to its predecessor in the stream by programmatic dependent launch: the kernel may be scheduled while
// the predecessor is still running and waits for it (pdl_wait) before it touches anything in memory.
// Kernels launched this way read what earlier kernels may write with ordinary loads, never through the read-only path:
// the data need not be final when the kernel starts.
// cluster: CTAs of a thread-block cluster, side by side along x.
template <typename... KArgs, typename... Args>
int op_launch_clusters(void (*kernel)(KArgs...), unsigned cluster, dim3 grid, dim3 block, size_t smem, cudaStream_t st, Args&&... args) {
  cudaLaunchConfig_t lc{};
  lc.gridDim = grid;
  lc.blockDim = block;
  lc.dynamicSmemBytes = smem;
  lc.stream = st;
  cudaLaunchAttribute attr[2];
  lc.attrs = attr;
  attr[0].id = cudaLaunchAttributeProgrammaticStreamSerialization;
  attr[0].val.programmaticStreamSerializationAllowed = 1;
  attr[1].id = cudaLaunchAttributeClusterDimension;
  attr[1].val.clusterDim.x = cluster;
  attr[1].val.clusterDim.y = attr[1].val.clusterDim.z = 1;
  lc.numAttrs = cluster > 1 ? 2 : 1;
  const cudaError_t e = cudaLaunchKernelEx(&lc, kernel, static_cast<KArgs>(args)...);
  if (e != cudaSuccess) return op_fail(THINFER_ECUDA, "kernel launch failed: %s", cudaGetErrorString(e));
  return THINFER_OK;
}

template <typename... KArgs, typename... Args>
int op_launch(void (*kernel)(KArgs...), dim3 grid, dim3 block, size_t smem, cudaStream_t st, Args&&... args) {
  return op_launch_clusters(kernel, 1, grid, block, smem, st, static_cast<Args&&>(args)...);
}

inline bool aligned16(const void* p) { return (reinterpret_cast<uintptr_t>(p) & 15u) == 0; }
inline bool aligned8(const void* p) { return (reinterpret_cast<uintptr_t>(p) & 7u) == 0; }
inline bool aligned4(const void* p) { return (reinterpret_cast<uintptr_t>(p) & 3u) == 0; }

inline bool overlap(const void* a, size_t na, const void* b, size_t nb) {
  const uintptr_t x = reinterpret_cast<uintptr_t>(a), y = reinterpret_cast<uintptr_t>(b);
  return x < y + nb && y < x + na;
}

// n rows of wa (wb) bytes, sa (sb) bytes apart; with different strides any overlap of the whole ranges counts.
inline bool rows_overlap(const void* a, int64_t sa, int64_t wa, const void* b, int64_t sb, int64_t wb, int64_t n) {
  if (!overlap(a, static_cast<size_t>((n - 1) * sa + wa), b, static_cast<size_t>((n - 1) * sb + wb))) return false;
  if (sa != sb || n == 1) return true;
  const int64_t apart = static_cast<int64_t>(reinterpret_cast<uintptr_t>(a)) - static_cast<int64_t>(reinterpret_cast<uintptr_t>(b));
  const int64_t at = (apart % sa + sa) % sa;   // where a's row begins behind the beginning of one of b's
  return at < wb || at + wa > sa;
}

struct Span {
  const void* at;
  size_t bytes;
};
inline bool meet(std::initializer_list<Span> a, std::initializer_list<Span> b) {
  for (const Span& x : a)
    for (const Span& y : b)
      if (overlap(x.at, x.bytes, y.at, y.bytes)) return true;
  return false;
}

// n rows of `wide` bytes, `stride` bytes apart, and one block of memory, which may lie between them.
inline bool rows_meet(const void* first, int64_t stride, int64_t wide, int64_t n, const Span& block) {
  if (block.bytes == 0) return false;
  const int64_t at = reinterpret_cast<intptr_t>(block.at) - reinterpret_cast<intptr_t>(first);
  const int64_t i = at < wide ? 0 : (at - wide) / stride + 1;   // the first row that ends behind the block's beginning
  return i < n && i * stride < at + static_cast<int64_t>(block.bytes);
}

// Opts a kernel in to its dynamic shared memory, small sizes too: what it may have without being asked depends on its static
// shared memory.  Internal to each source file: a static of a function with external linkage is one object for the whole
// process, also where it loads the builds of both storage types, whose kernels bear the same names.
template <auto Kernel>
static int opt_in(size_t bytes) {
  static SmemOptIn opt;
  if (!opt.ensure(Kernel, static_cast<int>(bytes))) return op_fail(THINFER_ECUDA, "cannot reserve %zu bytes of shared memory", bytes);
  return THINFER_OK;
}

}  // namespace thinfer

// Host-side pieces that the entry points share: allocation (with its test hook), error codes, counts, launches.
#pragma once
#include <cuda_runtime.h>
#include <atomic>
#include <cstdint>
#include <utility>

#include "../../include/gnn.h"

namespace gnn {

// Test hook: the next g_fail_allocs device allocations made by the library fail (host-side fault
// injection for the allocation-failure paths; see gnn_debug_fail_allocs).
inline std::atomic<int> g_fail_allocs{0};

inline cudaError_t dev_alloc(void** p, size_t bytes) {
  int n = g_fail_allocs.load();
  while (n > 0 && !g_fail_allocs.compare_exchange_weak(n, n - 1)) {
  }
  if (n > 0) {
    *p = nullptr;
    return cudaErrorMemoryAllocation;
  }
  return cudaMalloc(p, bytes);
}

inline int cuda_fail(cudaError_t e) {
  (void)cudaGetLastError();
  return e == cudaErrorMemoryAllocation ? GNN_ERR_OOM : GNN_ERR_CUDA;
}

// Every count a call accepts (nodes, edges, output capacity) lies in [0, GNN_MAX_COUNT], so that
// the kernels' 32-bit row indices stay in range after rounding up to a whole block or radix tile
// (at most 8192 rows).
inline bool count_ok(int64_t n) { return n >= 0 && n <= (int64_t)GNN_MAX_COUNT; }

// Blocks of `per_block` threads (or rows) covering n, computed in 64 bits.
inline unsigned blocks_for(int64_t n, int64_t per_block) { return (unsigned)((n + per_block - 1) / per_block); }

// Launch as a programmatic dependent of the previous kernel in the stream: the kernel may start
// while that one finishes its last CTAs, and waits for it (pdl_wait) before touching its data.
// Every kernel launched this way calls pdl_wait before its first access to data an earlier
// kernel writes.  Returns the launch status.
template <typename... KArgs, typename... Args>
cudaError_t launch_pdl(void (*kernel)(KArgs...), unsigned grid, unsigned block, size_t smem, cudaStream_t st,
                       Args&&... args) {
  cudaLaunchConfig_t cfg = {};
  cfg.gridDim = dim3(grid);
  cfg.blockDim = dim3(block);
  cfg.dynamicSmemBytes = smem;
  cfg.stream = st;
  cudaLaunchAttribute attr[1];
  attr[0].id = cudaLaunchAttributeProgrammaticStreamSerialization;
  attr[0].val.programmaticStreamSerializationAllowed = 1;
  cfg.attrs = attr;
  cfg.numAttrs = 1;
  return cudaLaunchKernelEx(&cfg, kernel, std::forward<Args>(args)...);
}

}  // namespace gnn

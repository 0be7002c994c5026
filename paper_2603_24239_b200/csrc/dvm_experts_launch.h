// Launch-side declarations of the translation units of the operators of a layer of experts.
#pragma once
#include <cuda_runtime.h>

#include "dvm_experts.h"
#include "dvm_launch.h"

int dvm_launch_routing(const dvm_routing_desc& d, void* const* t, cudaStream_t stream);
int dvm_launch_quantize(const dvm_quantize_desc& d, void* const* t, cudaStream_t stream);
int dvm_launch_scaled_matmul(const dvm_scaled_matmul_desc& d, void* const* t, cudaStream_t stream);
int dvm_launch_combine(const dvm_combine_desc& d, void* const* t, cudaStream_t stream);

// These kernels too are set up while the kernel before them on the stream ends (dvm_launch_early): each waits (grid_wait)
// before its first access to memory and before it asks for tensor memory.  (Before that the scaled product for few rows asks L2 for a
// dense weight's first tiles, which reads nothing: what the launch before still writes there is found when they are loaded.)
template <class... P, class... A>
inline int dvm_launch_next(void (*kernel)(P...), dim3 grid, int threads, size_t smem, cudaStream_t stream, const A&... args) {
  return dvm_launch_early(kernel, grid, threads, smem, stream, args...);
}

// Launch-side declarations shared by the CUDA translation units of libdvm (not part of the ABI).
#pragma once
#include <cuda_runtime.h>
#include <stddef.h>
#include <stdint.h>

#include <atomic>

#include "../../include/dvm.h"

// Device status word values (read back by dvm_last_device_status).
namespace dvm {
enum { ST_OK = 0, ST_BAD_CODE = 1, ST_TIMEOUT = 2 };
}

void dvm_note_cuda_error(int e);

// Records a failed CUDA runtime call (dvm_last_cuda_error) and returns DVM_ERR_CUDA from the caller.  The runtime's own record
// of it is cleared: the check behind a later launch would find it there and report a launch that did not fail.
#define DVM_CUDA(call)                \
  do {                                \
    cudaError_t e_ = (call);          \
    if (e_ != cudaSuccess) {          \
      dvm_note_cuda_error((int)e_);   \
      (void)cudaGetLastError();       \
      return DVM_ERR_CUDA;            \
    }                                 \
  } while (0)

struct DvmDeviceInfo {
  unsigned int* scratch;  // library-owned device words: [0] status, then work-queue counter pairs
  int sm_count;
  int device;
};

// Per-device lazy set-up (scratch allocation, occupancy) for the current device.  Reserves nothing: launches with a work queue
// take their slot themselves.
int dvm_device_state(DvmDeviceInfo* info);
// Lets `kernel` have `bytes` of dynamic shared memory; `done` (a bit per device) spares the driver call from the second time on.
inline int dvm_allow_smem(const void* kernel, int bytes, int device, std::atomic<uint64_t>* done) {
  const uint64_t bit = 1ull << (device & 63);
  if (done->load(std::memory_order_acquire) & bit) return DVM_OK;
  DVM_CUDA(cudaFuncSetAttribute(kernel, cudaFuncAttributeMaxDynamicSharedMemorySize, bytes));
  done->fetch_or(bit, std::memory_order_release);
  return DVM_OK;
}
void dvm_count_launch();

// A launch that may start while the kernel before it on the stream ends: its CTAs are set up and wait (grid_wait) until that
// kernel has finished and what it wrote can be read.  Every thread of such a kernel calls grid_wait before its first access
// to memory and before it asks for tensor memory, grid_ready lets the next launch of this kind do the same.  (Another kernel before or after orders as ever.)
// Measured in a chain of launches: one token's rotary 2.8 -> 1.8 us, and 0.7 us less of the host's time.
template <class... P, class... A>
int dvm_launch_early(void (*kernel)(P...), dim3 grid, int threads, size_t smem, cudaStream_t stream, const A&... args) {
  cudaLaunchConfig_t cfg = {};
  cudaLaunchAttribute at[1];
  at[0].id = cudaLaunchAttributeProgrammaticStreamSerialization;
  at[0].val.programmaticStreamSerializationAllowed = 1;
  cfg.gridDim = grid;
  cfg.blockDim = dim3(threads);
  cfg.dynamicSmemBytes = smem;
  cfg.stream = stream;
  cfg.attrs = at;
  cfg.numAttrs = 1;
  DVM_CUDA(cudaLaunchKernelEx(&cfg, kernel, args...));
  dvm_count_launch();
  return DVM_OK;
}
#ifdef __CUDACC__
namespace dvm {
__device__ __forceinline__ void grid_wait() { asm volatile("griddepcontrol.wait;" ::: "memory"); }
__device__ __forceinline__ void grid_ready() { asm volatile("griddepcontrol.launch_dependents;" ::: "memory"); }
}  // namespace dvm
#endif

int dvm_launch_matmul(const uint32_t* code, size_t n_words, void* const* tensors, int n_tensors,
                      cudaStream_t stream);

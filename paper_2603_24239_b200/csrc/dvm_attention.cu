// Attention meta-kernel: host launch, and the kernel without tensor cores.
//
// dvm_attention_plain_kernel takes any type, stride and head size: one warp per row and head walks the visible tokens.
// It is what inputs get that the tensor-core kernels cannot load (fp32, odd head sizes, odd strides or pointers).
#include <cuda_runtime.h>

#include <atomic>

#include "dvm_attention.cuh"
#include "dvm_attention_launch.h"
#include "dvm_launch.h"
#include "dvm_sm100.cuh"

namespace dvm {
namespace att {

constexpr int PLAIN_WARPS = 8;

template <class T>
__global__ void __launch_bounds__(PLAIN_WARPS * 32) dvm_attention_plain_kernel(const __grid_constant__ Args a) {
  const long long item = (long long)blockIdx.x * PLAIN_WARPS + (threadIdx.x >> 5);
  if (item >= (long long)a.rows * a.hq) return;
  const int row = (int)(item / a.hq), head = (int)(item % a.hq);
  int lo = 0, hi = a.n + 1;  // first i with starts[i] > row
  while (lo < hi) {
    const int mid = (lo + hi) >> 1;
    if (a.starts[mid] > row) hi = mid; else lo = mid + 1;
  }
  const int i = lo - 1;
  if (i < 0 || i >= a.n) return;
  const Request r = request_at(a, i);
  const int j = row - r.s0;
  if (j < 0 || j >= min(r.q_len, a.max_q)) return;
  attend_row<T>(a, i, r.pos0 + j, row, head);
}

}  // namespace att
}  // namespace dvm

static thread_local int t_last_kernel = -1;

namespace {
typedef CUresult (*EncodeTiledFn)(CUtensorMap*, CUtensorMapDataType, cuuint32_t, void*, const cuuint64_t*, const cuuint64_t*, const cuuint32_t*,
                                  const cuuint32_t*, CUtensorMapInterleave, CUtensorMapSwizzle, CUtensorMapL2promotion, CUtensorMapFloatOOBfill);

int encode_map(CUtensorMap* map, const void* ptr, const cuuint64_t (&dims)[4], const cuuint64_t (&strides)[3], const cuuint32_t (&box)[4]) {
  static std::atomic<EncodeTiledFn> cached{nullptr};
  EncodeTiledFn fn = cached.load();
  if (!fn) {
    void* p = nullptr;
    cudaDriverEntryPointQueryResult found;
    const cudaError_t e = cudaGetDriverEntryPoint("cuTensorMapEncodeTiled", &p, cudaEnableDefault, &found);
    if (e != cudaSuccess || found != cudaDriverEntryPointSuccess || !p) {
      dvm_note_cuda_error(e != cudaSuccess ? (int)e : (int)cudaErrorNotSupported);
      (void)cudaGetLastError();
      return DVM_ERR_CUDA;
    }
    fn = (EncodeTiledFn)p;
    cached.store(fn);
  }
  const cuuint32_t one[4] = {1, 1, 1, 1};
  if (fn(map, CU_TENSOR_MAP_DATA_TYPE_BFLOAT16, 4, const_cast<void*>(ptr), dims, strides, box, one, CU_TENSOR_MAP_INTERLEAVE_NONE,
         CU_TENSOR_MAP_SWIZZLE_128B, CU_TENSOR_MAP_L2_PROMOTION_L2_256B, CU_TENSOR_MAP_FLOAT_OOB_FILL_NONE) != CUDA_SUCCESS) {
    dvm_note_cuda_error((int)cudaErrorInvalidValue);
    return DVM_ERR_CUDA;
  }
  return DVM_OK;
}

// (the stride of a dim of size 1 is never walked: any legal one)
inline cuuint64_t map_stride(int64_t size, int64_t stride) { return size > 1 ? (cuuint64_t)stride * 2 : 16; }
}  // namespace

int dvm_cache_map(const dvm_attention_desc& d, const int64_t* stride, const void* ptr, int most, CUtensorMap* map) {
  const cuuint64_t dims[4] = {(cuuint64_t)d.head_dim, (cuuint64_t)d.page_size, (cuuint64_t)d.kv_heads, (cuuint64_t)d.pages};
  const cuuint64_t strides[3] = {map_stride(d.page_size, stride[1]), map_stride(d.kv_heads, stride[2]), map_stride(d.pages, stride[0])};
  const cuuint32_t box[4] = {64, (cuuint32_t)(d.page_size < most ? d.page_size : most), 1, 1};
  return encode_map(map, ptr, dims, strides, box);
}

extern "C" int dvm_last_attention_kernel(int* kernel) {
  if (!kernel || t_last_kernel < 0) return DVM_ERR_INVALID_ARG;
  *kernel = t_last_kernel;
  return DVM_OK;
}

int dvm_query_map(const dvm_attention_desc& d, const void* ptr, int tokens, CUtensorMap* map) {
  const int64_t group = d.q_heads / d.kv_heads;
  const cuuint64_t dims[4] = {(cuuint64_t)d.head_dim, (cuuint64_t)group, (cuuint64_t)d.kv_heads, (cuuint64_t)d.rows};
  const cuuint64_t strides[3] = {map_stride(group, d.q_stride[1]), map_stride(d.kv_heads, group * d.q_stride[1]), map_stride(d.rows, d.q_stride[0])};
  const cuuint32_t box[4] = {64, (cuuint32_t)group, 1, (cuuint32_t)tokens};
  return encode_map(map, ptr, dims, strides, box);
}

int dvm_launch_attention(const dvm_attention_desc& d, void* const* t, cudaStream_t stream) {
  using namespace dvm::att;
  DvmDeviceInfo dev;
  int st = dvm_device_state(&dev);
  if (st != DVM_OK) return st;
  Args a = {};
  a.q = t[AT_Q]; a.k = t[AT_K]; a.v = t[AT_V];
  a.table = (const int*)t[AT_TABLE]; a.starts = (const int*)t[AT_STARTS]; a.lengths = (const int*)t[AT_LENGTHS];
  a.out = t[AT_OUT]; a.ws = (float*)t[AT_WS]; a.status = dev.scratch;
  for (int i = 0; i < 2; ++i) { a.qs[i] = d.q_stride[i]; a.os[i] = d.out_stride[i]; }
  for (int i = 0; i < 3; ++i) { a.ks[i] = d.k_stride[i]; a.vs[i] = d.v_stride[i]; }
  a.n = (int)d.requests; a.rows = (int)d.rows; a.hq = (int)d.q_heads; a.hk = (int)d.kv_heads; a.group = a.hq / a.hk; a.D = (int)d.head_dim;
  a.pages = (int)d.pages; a.max_blocks = (int)d.max_blocks;
  while ((1ll << a.page_log) < d.page_size) ++a.page_log;
  a.window = (int)d.window; a.sinks = (int)d.sinks; a.max_q = (int)d.max_q; a.out_bf16 = d.out_dtype == DVM_BF16; a.scale = d.scale;
  const bool aligned = (((uintptr_t)a.q | (uintptr_t)a.k | (uintptr_t)a.v) & 15) == 0;
  auto stores = [&](int n) { return a.out_bf16 && (uintptr_t)a.out % (2 * n) == 0 && d.out_stride[0] % n == 0 && d.out_stride[1] % n == 0; };
  a.out_vec = stores(16) && a.D % 16 == 0 ? 2 : stores(8) ? 1 : 0;
  if (aligned && dvm_attention_tensor_cores(d)) {
    const bool single = dvm_attention_single(d);
    st = single ? dvm_launch_attention_single(d, a, dev.device, stream) : dvm_launch_attention_prompt(d, a, dev.device, stream);
    if (st == DVM_OK) t_last_kernel = single ? 1 : 2;
    return st;
  }
  const int64_t items = d.rows * d.q_heads, grid = (items + PLAIN_WARPS - 1) / PLAIN_WARPS;
  if (grid >= (1ll << 31)) return DVM_ERR_TOO_LARGE;
  if (d.dtype == DVM_BF16) dvm_attention_plain_kernel<__nv_bfloat16><<<(int)grid, PLAIN_WARPS * 32, 0, stream>>>(a);
  else dvm_attention_plain_kernel<float><<<(int)grid, PLAIN_WARPS * 32, 0, stream>>>(a);
  DVM_CUDA(cudaGetLastError());
  dvm_count_launch();
  t_last_kernel = 0;
  return DVM_OK;
}

// ---- self-tests of the attention kernels' bounded waits (see dvm_selftest_bounded_wait) ----
namespace dvm {
namespace att {
using namespace sm100;
constexpr int WAIT_FLAT = 3, WAIT_POLL = 4, WAIT_DRAIN = 5;  // `which`
__global__ void dvm_selftest_attention_wait_kernel(int which, unsigned int* status) {
  constexpr uint32_t STAGES = 3, LATE_NS = 20000000;
  __shared__ __align__(8) unsigned long long bars[1 + STAGES];
  __shared__ volatile uint32_t words[3];  // abort flag, signs of work
  const uint32_t never = smem_u32(bars), full = never + 8;
  const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
  if (threadIdx.x == 0) {
    words[0] = words[1] = words[2] = 0;
    mbar_init(never, 2);  // two arrivals expected, one ever made: the phase never completes
    for (uint32_t s = 0; s < STAGES; ++s) mbar_init(full + 8 * s, 1);
    asm volatile("fence.mbarrier_init.release.cluster;" ::: "memory");
    mbar_arrive(never);
    mbar_arrive(full);       // five fills of three stages, of which the last will land long after the wait below has run out:
    mbar_arrive(full + 8);   // in stages 0 and 1 the second one
    mbar_arrive(full + 16);
    mbar_arrive(full);
  }
  __syncthreads();
  bool ok = true;
  if (warp == 0)
    ok = which == WAIT_FLAT ? mbar_wait_flat(never, 0, words, words + 1) : which == WAIT_POLL ? mbar_poll(never, 0, words, words + 1) : mbar_wait(never, 0, words);
  __syncthreads();
  if (!words[0]) return;
  if (which == WAIT_DRAIN) {
    if (warp == 1 && lane == 0) {  // the fill that is late
      const unsigned long long t0 = gtimer();
      for (uint32_t i = 0; i < WAIT_SPINS && gtimer() - t0 < LATE_NS; ++i) {}
      mbar_arrive(full + 8);
    }
    if (threadIdx.x == 0) {
      mbar_drain(full, STAGES, 5, 2, 1, words);
      ok = !(mbar_test(full, 1) && mbar_test(full + 8, 1) && mbar_test(full + 16, 0));
    }
  }
  if (threadIdx.x == 0) atomicMax(status, (unsigned int)(ok ? ST_BAD_CODE : ST_TIMEOUT));
}
}  // namespace att
}  // namespace dvm

int dvm_selftest_attention_wait(int which, unsigned int* status, cudaStream_t stream) {
  dvm::att::dvm_selftest_attention_wait_kernel<<<1, 64, 0, stream>>>(which, status);
  DVM_CUDA(cudaGetLastError());
  dvm_count_launch();
  return DVM_OK;
}

// ---- dvm_launch's entry for the serving codes (verified) ----
int dvm_launch_serving(const uint32_t* w, void* const* tensors, int n_tensors, cudaStream_t stream) {
  const int nt = w[DVM_H_COUNTS] & 0xff;
  if (n_tensors != nt) return DVM_ERR_INVALID_ARG;
  if (w[DVM_H_N_TILES] == 0) return DVM_OK;
  int64_t need[DVM_MAX_TENSORS];
  dvm_extents_serving(w, need);
  for (int i = 0; i < nt; ++i)
    if (need[i] > 0 && !tensors[i]) return DVM_ERR_INVALID_ARG;
  const uint32_t type = w[DVM_H_KERNEL_TYPE];
  // An output that begins where another tensor does overlaps it (the dense ones of paging: that shares a byte with it).
  // Rotary may work in place: each run is read and written by one thread.
  int may[2][2] = {{-1, -1}, {-1, -1}};
  if (type == DVM_KERNEL_ROTARY) {
    dvm_rotary_desc d;
    dvm_serving_desc(w, &d);
    const RotarySlots s = dvm_rotary_slots(d);
    auto same = [&](const int64_t* x, const int64_t* y) { return d.dtype == d.out_dtype && x[0] == y[0] && x[1] == y[1]; };
    if (same(d.q_stride, d.q_out_stride)) { may[0][0] = s.q; may[0][1] = s.q_out; }
    if (!d.paged && same(d.k_stride, d.k_out_stride)) { may[1][0] = s.k; may[1][1] = s.k_out; }
  }
  for (int i = (w[DVM_H_COUNTS] >> 8) & 0xff; i < nt; ++i)
    for (int j = 0; j < nt; ++j) {
      if (i == j || need[i] <= 0 || need[j] <= 0 || (j == may[0][0] && i == may[0][1]) || (j == may[1][0] && i == may[1][1])) continue;
      const uintptr_t x = (uintptr_t)tensors[i], y = (uintptr_t)tensors[j];
      if (type == DVM_KERNEL_PAGING ? x < y + (uintptr_t)need[j] && y < x + (uintptr_t)need[i] : x == y) return DVM_ERR_INVALID_ARG;
    }
  auto aligned = [&](int slot, int dtype) { return slot < 0 || ((uintptr_t)tensors[slot] & (dtype == DVM_BF16 ? 1 : 3)) == 0; };
  if (type == DVM_KERNEL_PAGING) {
    dvm_paging_desc d;
    dvm_serving_desc(w, &d);
    for (int i = 0; i < PG_N; ++i)
      if (!aligned(i, DVM_F32)) return DVM_ERR_INVALID_ARG;
    return dvm_launch_paging(d, tensors, stream);
  }
  if (type == DVM_KERNEL_ROTARY) {
    dvm_rotary_desc d;
    dvm_serving_desc(w, &d);
    const RotarySlots s = dvm_rotary_slots(d);
    if (!aligned(s.q, d.dtype) || !aligned(s.k, d.dtype) || !aligned(s.v, d.dtype) || !aligned(s.wq, d.weight_dtype) || !aligned(s.wk, d.weight_dtype) ||
        !aligned(s.angles, DVM_F32) || !aligned(s.positions, DVM_F32) || !aligned(s.slots, DVM_F32) || !aligned(s.q_out, d.out_dtype) ||
        !aligned(s.k_out, d.out_dtype) || !aligned(s.v_out, d.out_dtype))
      return DVM_ERR_INVALID_ARG;
    return dvm_launch_rotary(d, tensors, stream);
  }
  dvm_attention_desc d;
  dvm_serving_desc(w, &d);
  if (!aligned(AT_Q, d.dtype) || !aligned(AT_K, d.dtype) || !aligned(AT_V, d.dtype) || !aligned(AT_TABLE, DVM_F32) || !aligned(AT_STARTS, DVM_F32) ||
      !aligned(AT_LENGTHS, DVM_F32) || !aligned(AT_OUT, d.out_dtype) || (need[AT_WS] > 0 && ((uintptr_t)tensors[AT_WS] & 15)))
    return DVM_ERR_INVALID_ARG;
  return dvm_launch_attention(d, tensors, stream);
}

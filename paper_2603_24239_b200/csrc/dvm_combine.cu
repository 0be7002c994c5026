// Combine meta-kernel: every token's rows added up by weight, out[t] = base[t] + sum_j weights[t, j] y[places[t, j]].
//
// Bound by memory: each row is read once.  A thread takes twice 16 bytes of columns of one token and asks for up to 8 rows at
// once; sums are fp32, in the order of j, rounded once.  8192 tokens of 8 rows of 4096, with a base: 113 us, 5.9 TB/s (124 with one
// run of 16 bytes to a thread); rows at odd places, a column to a load, 237 without a base (100 at even ones); 64 tokens of 6: 2.5 us in a
// chain of launches.
#include <cuda_bf16.h>
#include <cuda_runtime.h>

#include "dvm_experts_launch.h"

namespace dvm {
namespace combine {

constexpr int THREADS = 256, AHEAD = 8, RUNS = 2;

struct Args {
  const void *y, *base;
  const int* places;
  const float* weights;
  void* out;
  long long ys, bs, os;
  int tokens, top_k, rows, cols, runs;   // runs: of a thread's columns in a row
};

// A thread's columns: W of them, in 16 bytes, or one.
template <class T, int W> struct Run;
template <> struct Run<__nv_bfloat16, 8> {
  uint4 w;
  __device__ __forceinline__ void load(const __nv_bfloat16* p) { w = *(const uint4*)p; }
  __device__ __forceinline__ void add(float by, float (&v)[8]) const {
    const uint32_t u[4] = {w.x, w.y, w.z, w.w};
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      v[2 * i] = fmaf(by, __uint_as_float(u[i] << 16), v[2 * i]);
      v[2 * i + 1] = fmaf(by, __uint_as_float(u[i] & 0xffff0000u), v[2 * i + 1]);
    }
  }
  static __device__ __forceinline__ void store(__nv_bfloat16* p, const float (&v)[8]) {
    uint32_t u[4];
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      const __nv_bfloat162 h = __floats2bfloat162_rn(v[2 * i], v[2 * i + 1]);
      u[i] = *(const uint32_t*)&h;
    }
    *(uint4*)p = make_uint4(u[0], u[1], u[2], u[3]);
  }
};
template <> struct Run<float, 4> {
  float4 w;
  __device__ __forceinline__ void load(const float* p) { w = *(const float4*)p; }
  __device__ __forceinline__ void add(float by, float (&v)[4]) const {
    v[0] = fmaf(by, w.x, v[0]); v[1] = fmaf(by, w.y, v[1]); v[2] = fmaf(by, w.z, v[2]); v[3] = fmaf(by, w.w, v[3]);
  }
  static __device__ __forceinline__ void store(float* p, const float (&v)[4]) { *(float4*)p = make_float4(v[0], v[1], v[2], v[3]); }
};
template <class T> struct Run<T, 1> {
  T w;
  __device__ __forceinline__ void load(const T* p) { w = *p; }
  __device__ __forceinline__ void add(float by, float (&v)[1]) const { v[0] = fmaf(by, (float)w, v[0]); }
  static __device__ __forceinline__ void store(T* p, const float (&v)[1]) { *p = (T)v[0]; }
};

template <class T, int W> __global__ void __launch_bounds__(THREADS) dvm_combine_kernel(const __grid_constant__ Args a) {
  const int lane = threadIdx.x & 31;
  grid_ready();
  grid_wait();
  // a warp's item: RUNS * 32 runs of a token
  const int parts = (int)(((uint32_t)a.runs + (RUNS * 32 - 1)) / (RUNS * 32));   // (a row may have 2^31 - 1 columns)
  const long long items = (long long)a.tokens * parts, step = (long long)gridDim.x * (THREADS / 32);
  for (long long item = (long long)blockIdx.x * (THREADS / 32) + (threadIdx.x >> 5); item < items; item += step) {
    const int t = (int)(item / parts), run0 = (int)(item - (long long)t * parts) * (RUNS * 32) + lane;
    float v[RUNS][W] = {};
    if (a.base) {
#pragma unroll
      for (int r = 0; r < RUNS; ++r)
        if (run0 + 32 * r < a.runs) {
          Run<T, W> b;
          b.load((const T*)a.base + t * a.bs + (run0 + 32 * r) * W);
          b.add(1.f, v[r]);
        }
    }
    bool any = false;
    for (int j0 = 0; j0 < a.top_k; j0 += AHEAD) {
      int place[AHEAD];
      float by[AHEAD];
#pragma unroll
      for (int j = 0; j < AHEAD; ++j) {
        place[j] = j0 + j < a.top_k ? a.places[(long long)t * a.top_k + j0 + j] : -1;
        by[j] = j0 + j < a.top_k ? a.weights[(long long)t * a.top_k + j0 + j] : 0.f;
      }
      Run<T, W> y[AHEAD][RUNS];
#pragma unroll
      for (int j = 0; j < AHEAD; ++j)
        if (place[j] >= 0 && place[j] < a.rows) {
#pragma unroll
          for (int r = 0; r < RUNS; ++r)
            if (run0 + 32 * r < a.runs) y[j][r].load((const T*)a.y + place[j] * a.ys + (run0 + 32 * r) * W);
        }
#pragma unroll
      for (int j = 0; j < AHEAD; ++j)
        if (place[j] >= 0 && place[j] < a.rows) {
          any = true;
#pragma unroll
          for (int r = 0; r < RUNS; ++r)
            if (run0 + 32 * r < a.runs) y[j][r].add(by[j], v[r]);
        }
    }
    if (any)
#pragma unroll
      for (int r = 0; r < RUNS; ++r)
        if (run0 + 32 * r < a.runs) Run<T, W>::store((T*)a.out + t * a.os + (run0 + 32 * r) * W, v[r]);
  }
}

}  // namespace combine
}  // namespace dvm

int dvm_launch_combine(const dvm_combine_desc& d, void* const* t, cudaStream_t stream) {
  using namespace dvm::combine;
  const CombineSlots s = dvm_slots(d);
  DvmDeviceInfo dev;
  int st = dvm_device_state(&dev);
  if (st != DVM_OK) return st;
  Args a = {};
  a.y = t[s.y]; a.places = (const int*)t[s.places]; a.weights = (const float*)t[s.weights];
  a.base = s.base >= 0 ? t[s.base] : nullptr;
  a.out = t[s.out];
  a.ys = d.y_stride; a.bs = d.base_stride; a.os = d.out_stride;
  a.tokens = (int)d.tokens; a.top_k = (int)d.top_k; a.rows = (int)d.rows; a.cols = (int)d.cols;
  const bool bf16 = d.dtype == DVM_BF16;
  const int run = bf16 ? 8 : 4;
  auto aligned = [&](const void* p, int64_t size, int64_t stride) { return !p || ((uintptr_t)p % 16 == 0 && (size <= 1 || stride % run == 0)); };
  const bool vec = d.cols % run == 0 && aligned(a.y, d.rows, a.ys) && aligned(a.base, d.tokens, a.bs) && aligned(a.out, d.tokens, a.os);
  a.runs = vec ? a.cols / run : a.cols;
  const int64_t ctas = dvm_up(a.tokens * dvm_up(a.runs, RUNS * 32), THREADS / 32), most = 8ll * dev.sm_count;
  auto launch = [&](auto kernel) { return dvm_launch_next(kernel, (int)(ctas < most ? ctas : most), THREADS, 0, stream, a); };
  if (bf16) return vec ? launch(dvm_combine_kernel<__nv_bfloat16, 8>) : launch(dvm_combine_kernel<__nv_bfloat16, 1>);
  return vec ? launch(dvm_combine_kernel<float, 4>) : launch(dvm_combine_kernel<float, 1>);
}

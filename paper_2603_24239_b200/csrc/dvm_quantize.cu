// Quantize meta-kernel: rows, gated pairs of rows or weights as e4m3 codes with a scale for each block of 128.
//
//   scale = max(max |v| / 448, 2^-126),   code = the e4m3 value nearest to v / scale (exactly), v = x or silu(gate) up
//
// Bound by memory: every value is read once; half a warp holds a block of a row, 8 values to a lane, so the maximum
// takes four exchanges and a block's codes leave as one run of 128 bytes, to as many rows as the token has experts.
// Quotients lie on the border between two codes often (bf16 values over their maximum are quotients of small numbers),
// so a rounded quotient would decide by its rounding.  Each is computed by a product with the reciprocal, which is off by
// less than 4 units in the last place; where that is as near to a border, the sign of v - border * scale, one exact
// multiply-add, decides.
#include <cuda_bf16.h>
#include <cuda_runtime.h>
#include <math.h>

#include "dvm_experts_launch.h"

namespace dvm {
namespace quantize {

constexpr int THREADS = 256, LANES = 16;

struct Args {
  const void* x;
  const int* places;
  uint8_t* codes;
  float* scales;
  long long xs, cs, ss;
  int rows, cols, out_rows, blocks, copies;   // blocks: of a row
};

__device__ __forceinline__ uint16_t pack_e4m3(float lo, float hi) {
  uint16_t r;
  asm("cvt.rn.satfinite.e4m3x2.f32 %0, %1, %2;" : "=h"(r) : "f"(hi), "f"(lo));
  return r;
}
// 8 values as they lie in memory -> fp32
template <bool VEC> __device__ __forceinline__ void load8(const __nv_bfloat16* p, float (&v)[8]) {
  if (VEC) {
    const uint4 w = *(const uint4*)p;
    const uint32_t u[4] = {w.x, w.y, w.z, w.w};
#pragma unroll
    for (int i = 0; i < 4; ++i) { v[2 * i] = __uint_as_float(u[i] << 16); v[2 * i + 1] = __uint_as_float(u[i] & 0xffff0000u); }
  } else {
#pragma unroll
    for (int i = 0; i < 8; ++i) v[i] = __bfloat162float(p[i]);
  }
}
template <bool VEC> __device__ __forceinline__ void load8(const float* p, float (&v)[8]) {
  if (VEC) {
    const float4 a = *(const float4*)p, b = *(const float4*)(p + 4);
    v[0] = a.x; v[1] = a.y; v[2] = a.z; v[3] = a.w; v[4] = b.x; v[5] = b.y; v[6] = b.z; v[7] = b.w;
  } else {
#pragma unroll
    for (int i = 0; i < 8; ++i) v[i] = p[i];
  }
}
__device__ __forceinline__ float silu(float z) { return z / (1.f + __expf(-z)); }
__device__ __forceinline__ uint32_t abs_bits(const float (&v)[8]) {  // of the largest magnitude; NaN is above infinity
  uint32_t m = 0;
#pragma unroll
  for (int i = 0; i < 8; ++i) m = max(m, __float_as_uint(v[i]) & 0x7fffffffu);
  return m;
}
// The scale of a block whose largest magnitude has these bits.
__device__ __forceinline__ float scale_of(uint32_t bits) {
  return bits >= 0x7f800000u ? __uint_as_float(0x7fc00000u) : fmaxf(__fdiv_rn(__uint_as_float(bits), 448.f), 0x1p-126f);
}
// r, near the border between two codes: moved to the side of it that a / s is on (a, s > 0)
__device__ __noinline__ float decide(float r, float a, float s) {
  // codes are 2^-9 apart below 2^-6 as they are from 2^-6 to 2^-5
  const bool low = r < 0x1p-6f;
  const float t = low ? r + 0x1p-6f : r;
  const float edge_t = __uint_as_float(((__float_as_uint(t) + 8u) & ~0xfffffu) | 0x80000u);
  const float edge = low ? edge_t - 0x1p-6f : edge_t;
  const float up = s < 0x1p-60f ? 0x1p64f : 1.f;   // (keeps the difference out of the subnormals)
  const float d = fmaf(-edge, s * up, a * up);
  return d > 0.f ? __uint_as_float(__float_as_uint(edge) + 1u) : d < 0.f ? __uint_as_float(__float_as_uint(edge) - 1u) : edge;
}
// Codes of 8 values of a block with scale s.  EXACT: borders are decided exactly.
template <bool EXACT> __device__ __forceinline__ uint2 codes8(const float (&v)[8], float s) {
  if (s != s) return make_uint2(0u, 0u);
  const float inv = __frcp_rn(s);
  float r[8];
  uint32_t near = 0;
#pragma unroll
  for (int i = 0; i < 8; ++i) {
    r[i] = v[i] * inv;
    if (EXACT) {
      const float m = fabsf(r[i]), t = m < 0x1p-6f ? m + 0x1p-6f : m;
      near |= (((__float_as_uint(t) - 0x7fffcu) & 0xfffffu) <= 8u ? 1u : 0u) << i;
    }
  }
  if (EXACT && near) {
#pragma unroll
    for (int i = 0; i < 8; ++i)
      if ((near >> i) & 1u) r[i] = copysignf(decide(fabsf(r[i]), fabsf(v[i]), s), v[i]);
  }
  return make_uint2(pack_e4m3(r[0], r[1]) | ((uint32_t)pack_e4m3(r[2], r[3]) << 16), pack_e4m3(r[4], r[5]) | ((uint32_t)pack_e4m3(r[6], r[7]) << 16));
}

// Blocks of rows: half a warp per block of 128 columns, one row-block after another.
template <class T, bool GATED, bool VEC> __global__ void __launch_bounds__(THREADS) dvm_quantize_kernel(const __grid_constant__ Args a) {
  const int lane = threadIdx.x % LANES;
  const uint32_t half = 0xffffu << (threadIdx.x & 16);
  const long long items = (long long)a.rows * a.blocks, step = (long long)gridDim.x * (THREADS / LANES);
  grid_ready();
  grid_wait();
  for (long long item = (long long)blockIdx.x * (THREADS / LANES) + threadIdx.x / LANES; item < items; item += step) {
    const int row = (int)(item / a.blocks), b = (int)(item - (long long)row * a.blocks), col = b * DVM_SCALE_BLOCK + 8 * lane;
    float v[8] = {};
    if (col < a.cols) {
      const T* x = (const T*)a.x + row * a.xs + col;
      load8<VEC>(x, v);
      if (GATED) {
        float u[8];
        load8<VEC>(x + a.cols, u);
#pragma unroll
        for (int i = 0; i < 8; ++i) v[i] = silu(v[i]) * u[i];
      }
    }
    uint32_t m = abs_bits(v);
#pragma unroll
    for (int d = LANES / 2; d > 0; d >>= 1) m = max(m, __shfl_xor_sync(half, m, d));
    const float s = scale_of(m);
    const uint2 c = codes8<!GATED>(v, s);
    for (int j = 0; j < max(a.copies, 1); ++j) {
      const int to = a.copies ? a.places[(long long)row * a.copies + j] : row;
      if (to < 0 || to >= a.out_rows) continue;
      if (col < a.cols) *(uint2*)(a.codes + to * a.cs + col) = c;
      if (lane == 0) a.scales[to * a.ss + b] = s;
    }
  }
}

// Blocks of 128 x 128: a CTA per block, 16 rows to a warp.
template <class T, bool VEC> __global__ void __launch_bounds__(THREADS) dvm_quantize_block_kernel(const __grid_constant__ Args a) {
  constexpr int ROWS = DVM_SCALE_BLOCK / (THREADS / LANES);   // of a thread
  __shared__ uint32_t most[THREADS / 32];
  const int lane = threadIdx.x % LANES, b = blockIdx.x % a.blocks, rb = blockIdx.x / a.blocks;
  const int col = b * DVM_SCALE_BLOCK + 8 * lane, row0 = rb * DVM_SCALE_BLOCK + threadIdx.x / LANES;
  grid_ready();
  grid_wait();
  float v[ROWS][8];
  uint32_t m = 0;
#pragma unroll
  for (int i = 0; i < ROWS; ++i) {
    const int row = row0 + i * (THREADS / LANES);
#pragma unroll
    for (int k = 0; k < 8; ++k) v[i][k] = 0.f;
    if (row < a.rows && col < a.cols) load8<VEC>((const T*)a.x + row * a.xs + col, v[i]);
  }
#pragma unroll
  for (int i = 0; i < ROWS; ++i) m = max(m, abs_bits(v[i]));
  m = __reduce_max_sync(0xffffffffu, m);
  if ((threadIdx.x & 31) == 0) most[threadIdx.x >> 5] = m;
  __syncthreads();
#pragma unroll
  for (int i = 0; i < THREADS / 32; ++i) m = max(m, most[i]);
  const float s = scale_of(m);
#pragma unroll
  for (int i = 0; i < ROWS; ++i) {
    const int row = row0 + i * (THREADS / LANES);
    const uint2 c = codes8<true>(v[i], s);
    if (row < a.rows && col < a.cols) *(uint2*)(a.codes + row * a.cs + col) = c;
  }
  if (threadIdx.x == 0) a.scales[rb * a.ss + b] = s;
}

}  // namespace quantize
}  // namespace dvm

int dvm_launch_quantize(const dvm_quantize_desc& d, void* const* t, cudaStream_t stream) {
  using namespace dvm::quantize;
  const QuantizeSlots s = dvm_slots(d);
  DvmDeviceInfo dev;
  int st = dvm_device_state(&dev);
  if (st != DVM_OK) return st;
  Args a = {};
  a.x = t[s.x];
  a.places = s.places >= 0 ? (const int*)t[s.places] : nullptr;
  a.codes = (uint8_t*)t[s.codes]; a.scales = (float*)t[s.scales];
  a.xs = d.x_stride; a.cs = d.codes_stride; a.ss = d.scales_stride;
  a.rows = (int)d.rows; a.cols = (int)d.cols; a.out_rows = (int)d.out_rows; a.blocks = (int)dvm_up(d.cols, DVM_SCALE_BLOCK); a.copies = d.copies;
  const bool bf16 = d.dtype == DVM_BF16;
  const bool vec = (uintptr_t)a.x % 16 == 0 && (d.rows <= 1 || d.x_stride % (bf16 ? 8 : 4) == 0);
  if (d.block_rows == DVM_SCALE_BLOCK) {
    const int64_t grid = dvm_up(d.rows, DVM_SCALE_BLOCK) * a.blocks;
    if (grid >= (1ll << 31)) return DVM_ERR_TOO_LARGE;
    auto launch = [&](auto kernel) { return dvm_launch_next(kernel, (int)grid, THREADS, 0, stream, a); };
    if (bf16) return vec ? launch(dvm_quantize_block_kernel<__nv_bfloat16, true>) : launch(dvm_quantize_block_kernel<__nv_bfloat16, false>);
    return vec ? launch(dvm_quantize_block_kernel<float, true>) : launch(dvm_quantize_block_kernel<float, false>);
  }
  const int64_t ctas = dvm_up(d.rows * a.blocks, THREADS / LANES), most = 8ll * dev.sm_count;
  auto launch = [&](auto kernel) { return dvm_launch_next(kernel, (int)(ctas < most ? ctas : most), THREADS, 0, stream, a); };
  if (bf16 && d.gated) return vec ? launch(dvm_quantize_kernel<__nv_bfloat16, true, true>) : launch(dvm_quantize_kernel<__nv_bfloat16, true, false>);
  if (bf16) return vec ? launch(dvm_quantize_kernel<__nv_bfloat16, false, true>) : launch(dvm_quantize_kernel<__nv_bfloat16, false, false>);
  if (d.gated) return vec ? launch(dvm_quantize_kernel<float, true, true>) : launch(dvm_quantize_kernel<float, true, false>);
  return vec ? launch(dvm_quantize_kernel<float, false, true>) : launch(dvm_quantize_kernel<float, false, false>);
}

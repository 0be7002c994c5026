// Quantize meta-kernel: rows, gated pairs of rows or weights as e4m3 codes with a scale for each block of 128.
//
//   scale = max(max |v| / 448, 2^-126),   code = the e4m3 value nearest to v / scale (exactly), v = x or silu(gate) up
//
// Bound by memory: every value is read once.  A block of a row is held by 8 lanes (16 in fp32), 16 (8) values to a lane, so the
// maximum takes three (four) exchanges and the codes leave 16 (8) bytes to a lane, as one run of 128 bytes, to as many rows as
// the token has experts; two elements to an instruction where there is one.
// Quotients lie on the border between two codes often (bf16 values over their maximum are quotients of small numbers),
// so a rounded quotient would decide by its rounding.  Each value is multiplied by a reciprocal a little too large and by one a
// little too small: where both products have one code, it is the quotient's; where not, the sign of v - border * scale, one
// exact multiply-add, decides, in a loop over the few that want it (nearly every warp has one in bf16 rows), which reads the
// value again: with a place in the code for each of the 16, 8192 rows of 4096 without copies took 33 us, now 27.
// A gated value is fp32 within a bound; its products take the bound in, and the largest of a block and the values at a border
// are computed again to 2^-40: in fp32 alone 1 of 600000 codes was the neighbour of the right one.
// 8192 tokens of 4096 to 8 rows each: 64 us, 5.4 TB/s; 49157 rows of 1408 gated: 73 us in a chain, 77 in calls, 4.8 and 4.5 (the largest
// again 9 us, the second product 4; 330 instructions to a warp's four blocks, one step after another); weights of 11008 x 4096 from fp32: 36 us, 6.2.
#include <cuda_bf16.h>
#include <cuda_fp16.h>
#include <cuda_runtime.h>
#include <math.h>

#include "dvm_experts_launch.h"
#include "dvm_sm100.cuh"

namespace dvm {
namespace quantize {

using namespace sm100;

constexpr int THREADS = 256, LANES = 16;   // LANES: of a row of a block of 128 x 128
constexpr uint32_t ALL = 0xffffffffu;

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
// N values as they lie in memory, and as fp32 pairs.
template <class T, int N> struct Raw;
template <int N> struct Raw<__nv_bfloat16, N> {
  uint32_t w[N / 2];
  template <bool VEC> __device__ __forceinline__ void load(const __nv_bfloat16* p) {
    if (VEC) {
#pragma unroll
      for (int i = 0; i < N / 8; ++i) {
        const uint4 q = ((const uint4*)p)[i];
        w[4 * i] = q.x; w[4 * i + 1] = q.y; w[4 * i + 2] = q.z; w[4 * i + 3] = q.w;
      }
    } else {
      const uint16_t* h = (const uint16_t*)p;
#pragma unroll
      for (int i = 0; i < N / 2; ++i) w[i] = h[2 * i] | ((uint32_t)h[2 * i + 1] << 16);
    }
  }
  __device__ __forceinline__ void clear() {
#pragma unroll
    for (int i = 0; i < N / 2; ++i) w[i] = 0u;
  }
  __device__ __forceinline__ float2 pair(int i) const { return make_float2(__uint_as_float(w[i] << 16), __uint_as_float(w[i] & 0xffff0000u)); }
  __device__ __forceinline__ Raw<__nv_bfloat16, 2> raw_pair(int i) const { return {{w[i]}}; }
};
template <int N> struct Raw<float, N> {
  float w[N];
  template <bool VEC> __device__ __forceinline__ void load(const float* p) {
    if (VEC) {
#pragma unroll
      for (int i = 0; i < N / 4; ++i) {
        const float4 q = ((const float4*)p)[i];
        w[4 * i] = q.x; w[4 * i + 1] = q.y; w[4 * i + 2] = q.z; w[4 * i + 3] = q.w;
      }
    } else {
#pragma unroll
      for (int i = 0; i < N; ++i) w[i] = p[i];
    }
  }
  __device__ __forceinline__ void clear() {
#pragma unroll
    for (int i = 0; i < N; ++i) w[i] = 0.f;
  }
  __device__ __forceinline__ float2 pair(int i) const { return make_float2(w[2 * i], w[2 * i + 1]); }
  __device__ __forceinline__ Raw<float, 2> raw_pair(int i) const { return {{w[2 * i], w[2 * i + 1]}}; }
};
__device__ __forceinline__ float wide(__nv_bfloat16 x) { return __bfloat162float(x); }
__device__ __forceinline__ float wide(float x) { return x; }
__device__ __forceinline__ float ex2(float x) {
  float y;
  asm("ex2.approx.ftz.f32 %0, %1;" : "=f"(y) : "f"(x));
  return y;
}
__device__ __forceinline__ float rcp(float x) {
  float y;
  asm("rcp.approx.ftz.f32 %0, %1;" : "=f"(y) : "f"(x));
  return y;
}
// silu(z) u: z (u / (1 + 2^(-z log2 e))); most: the largest 1 + 2^(-z log2 e).  (The quotient first: what it loses as a subnormal number
// is lost of a value below 2^-119, while a small z before a large u would lose bits of values of any size.)
__device__ __forceinline__ float2 gated(float2 z, float2 u, float& most) {
  const float2 e = mul2(z, make_float2(-1.4426950408889634f, -1.4426950408889634f));
  const float2 d = add2(make_float2(ex2(e.x), ex2(e.y)), make_float2(1.f, 1.f));
  asm("max.f32 %0, %0, %1, %2;" : "+f"(most) : "f"(d.x), "f"(d.y));
  return mul2(z, mul2(make_float2(rcp(d.x), rcp(d.y)), u));
}
// How far off the above is, relative to it, with the product of it and a rounded reciprocal of the scale: the exponent's rounding
// and that of log2 e cost |z| (2^-24 + 2^-26.2) where the exponential counts (z < 0), the instructions and roundings 11 x 2^-24 at
// most: 2^-19.6 while 1 + e < 2^12 (z > -8.4), less than 2^-16 up to where silu is 0 in fp32.
// In blocks of a small scale s what subnormal quotients lose may count: |z| 2^-150 < 2^-143.5 (|z| < 88, beyond 17 for z < 0 alone), 2^-7.5 of
// the least border, 2^-10 s >= 2^-136; from s = 2^-96 on it is 2^-37 of that.  (2^-6 to both sides still has one border at most.)
__device__ __forceinline__ float off_by(float most, float s) { return s < 0x1p-96f ? 0x1p-6f : most < 0x1p12f ? 0x1.6ap-20f : 0x1p-16f; }
// The same to 2^-40: 2^f by its series (the 11th term is below 2^-42), a reciprocal and a step of Newton's.  By a quarter of 1 + 2^(-z log2 e):
// where the above is zero, its reciprocal below 2^-126, is for the above alone to say, so that scale and codes see one place.
__device__ __forceinline__ double gated_exactly(float z, float u) {
  const double x = fminf(fmaxf(z, -200.f), 200.f), t = fma(x, -1.4426950408889634, 0x1.8p52), f = fma(x, -1.4426950408889634, 0x1.8p52 - t);
  double p = 7.054911620801121e-09;
  const double c[10] = {1.0178086009239696e-07, 1.3215486790144305e-06, 1.5252733804059838e-05, 0.00015403530393381606, 0.0013333558146428441,
                        0.009618129107628477, 0.055504108664821576, 0.2402265069591007, 0.6931471805599453, 1.0};
#pragma unroll
  for (int i = 0; i < 10; ++i) p = fma(p, f, c[i]);
  const double d = fma(p, __hiloint2double((__double2loint(t) + 1021) << 20, 0), 0.25), r = (double)rcp((float)d);
  return (double)z * fma(fma(-d, r, 1.0), r, r) * ((double)u * 0.25);
}
__device__ __forceinline__ float max_abs(float m, float x) {  // NaN if either is
  asm("max.NaN.f32 %0, %1, %2;" : "=f"(m) : "f"(m), "f"(fabsf(x)));
  return m;
}
__device__ __forceinline__ float max_abs(float m, float2 v) {  // (one instruction)
  asm("max.NaN.abs.f32 %0, %1, %2, %3;" : "=f"(m) : "f"(m), "f"(v.x), "f"(v.y));
  return m;
}
// The scale of a block of this largest magnitude.
__device__ __forceinline__ float scale_of(float most) {
  return most < INFINITY ? fmaxf(__fdiv_rn(most, 448.f), 0x1p-126f) : __uint_as_float(0x7fc00000u);
}
// The magnitude half way between the values of two neighbouring codes: 2^-10 times an odd number at least, 9 bits.
__device__ __forceinline__ float border(uint32_t lo, uint32_t hi) {
  uint32_t both;
  asm("cvt.rn.f16x2.e4m3x2 %0, %1;" : "=r"(both) : "h"((uint16_t)(lo | hi << 8)));
  const float2 f = __half22float2(*(const __half2*)&both);
  return fabsf(0.5f * (f.x + f.y));
}
// The sign of |v| / s - edge.
__device__ __forceinline__ int side(float v, float s, float edge) {
  const float up = s < 0x1p-60f ? 0x1p64f : 1.f;   // (keeps the difference out of the subnormals)
  const float d = fmaf(-edge, s * up, fabsf(v) * up);
  return (d > 0.f) - (d < 0.f);
}
__device__ __forceinline__ int side_gated(float z, float u, float s, float edge) {
  const double d = fabs(gated_exactly(z, u)) - (double)edge * (double)s;
  return (d > 0.) - (d < 0.);
}
// Codes of N values of a block with scale s, 4 to a word; off: how far from the quotients the products may be, relative to them;
// side_of(i, edge): on which side of a border value i lies (it reads the value again: few come here, in one loop).
template <int N, class Side> __device__ __forceinline__ void codes_of(const float2 (&v)[N / 2], float s, float off, uint32_t (&c)[N / 4], Side side_of) {
  if (s != s) {
#pragma unroll
    for (int i = 0; i < N / 4; ++i) c[i] = 0u;
    return;
  }
  const float inv = __frcp_rn(s), above = inv * (1.f + off), below = inv * (1.f - off);
  uint32_t low[N / 4], differ = 0u;
#pragma unroll
  for (int i = 0; i < N / 4; ++i) {
    const float2 p = mul2(v[2 * i], make_float2(above, above)), q = mul2(v[2 * i + 1], make_float2(above, above));
    c[i] = pack_e4m3(p.x, p.y) | ((uint32_t)pack_e4m3(q.x, q.y) << 16);
    const float2 r = mul2(v[2 * i], make_float2(below, below)), t = mul2(v[2 * i + 1], make_float2(below, below));
    low[i] = pack_e4m3(r.x, r.y) | ((uint32_t)pack_e4m3(t.x, t.y) << 16);
    differ |= c[i] ^ low[i];
  }
  if (differ) {
    uint32_t open = 0u;   // bit 8 b + 7 - k: byte b of word k differs
#pragma unroll
    for (int k = 0; k < N / 4; ++k) {
      const uint32_t x = c[k] ^ low[k];
      open |= ((((x & 0x7f7f7f7fu) + 0x7f7f7f7fu) | x) & 0x80808080u) >> k;
    }
#pragma unroll 1
    do {
      const int bit = __ffs(open) - 1, k = 7 - (bit & 7), b = bit & 24;
      open &= open - 1u;
      uint32_t high = c[0], other = low[0];
#pragma unroll
      for (int x = 1; x < N / 4; ++x)
        if (k == x) { high = c[x]; other = low[x]; }
      const uint32_t hi = (high >> b) & 0xffu, lo = (other >> b) & 0xffu;
      const int is = side_of(4 * k + (b >> 3), border(lo, hi));
      const uint32_t flip = is < 0 || (is == 0 && (hi & 1u)) ? (hi ^ lo) << b : 0u;
#pragma unroll
      for (int x = 0; x < N / 4; ++x)
        if (k == x) c[x] ^= flip;
    } while (open);
  }
}

// Blocks of rows: L lanes to a block of 128 columns; four CTAs per SM, since what counts is loads on their way (8192 tokens to 8
// rows each 64 us, 70 with as many registers as the compiler likes and two blocks of a row at once).
template <class T, bool GATED, bool VEC> __global__ void __launch_bounds__(THREADS, 4) dvm_quantize_kernel(const __grid_constant__ Args a) {
  constexpr int L = sizeof(T) == 2 ? 8 : 16, N = DVM_SCALE_BLOCK / L, GROUPS = THREADS / L;
  const int lane = threadIdx.x % L, group = threadIdx.x / L;
  const long long items = (long long)a.rows * a.blocks, step = (long long)gridDim.x * GROUPS;
  grid_ready();
  grid_wait();
  // row and block of the next item: a division once, then steps of both
  const int step_rows = (int)(step / a.blocks), step_blocks = (int)(step - (long long)step_rows * a.blocks);
  long long item = (long long)blockIdx.x * GROUPS + group;
  int row = (int)(item / a.blocks), b = (int)(item - (long long)row * a.blocks);
  for (; item - group % (32 / L) < items; item += step) {   // (all lanes of a warp together)
    const int col = b * DVM_SCALE_BLOCK + N * lane;
    const bool here = item < items, in = here && col < a.cols;
    const T* const from = (const T*)a.x + row * a.xs + col;
    Raw<T, N> x, up;
    if (in) {
      x.template load<VEC>(from);
      if (GATED) up.template load<VEC>(from + a.cols);
    } else {
      x.clear();
      if (GATED) up.clear();
    }
    float2 v[N / 2];
    float most = 0.f, worst = 0.f, s;
#pragma unroll
    for (int i = 0; i < N / 2; ++i) {
      v[i] = GATED ? gated(x.pair(i), up.pair(i), worst) : x.pair(i);
      most = max_abs(most, v[i]);
    }
    const float own = most;
#pragma unroll
    for (int d = L / 2; d > 0; d >>= 1) most = max_abs(most, __shfl_xor_sync(ALL, most, d));
    uint32_t c[N / 4];
    if (GATED) {
      // the lanes whose largest may be the block's compute it again, to more than fp32
      s = 0.f;
      if (own > most * (1.f - 0x1p-15f)) {   // (not where all are zero)
        Raw<T, 2> z = {}, u = {};
        float first = 0.f;
#pragma unroll
        for (int i = 0; i < N / 2; ++i)
          if (max_abs(0.f, v[i]) == own) {
            z = x.raw_pair(i);
            u = up.raw_pair(i);
            first = v[i].x;
          }
        const float2 zs = z.pair(0), us = u.pair(0);
        const bool x_is = fabsf(first) == own;
        s = (float)(fabs(gated_exactly(x_is ? zs.x : zs.y, x_is ? us.x : us.y)) * (1. / 448.));
      }
#pragma unroll
      for (int d = L / 2; d > 0; d >>= 1) s = fmaxf(s, __shfl_xor_sync(ALL, s, d));
      s = most < INFINITY ? fmaxf(s, 0x1p-126f) : __uint_as_float(0x7fc00000u);
      codes_of<N>(v, s, off_by(worst, s), c, [&](int i, float edge) { return side_gated(wide(from[i]), wide(from[a.cols + i]), s, edge); });
    } else {
      s = scale_of(most);
      codes_of<N>(v, s, 0x1p-21f, c, [&](int i, float edge) { return side(wide(from[i]), s, edge); });
    }
    auto put = [&](uint8_t* p) {
      if (N == 16) *(uint4*)p = make_uint4(c[0], c[1], c[N / 4 - 2], c[N / 4 - 1]);
      else *(uint2*)p = make_uint2(c[0], c[1]);
    };
    if (!a.copies) {
      if (in) put(a.codes + row * a.cs + col);
      if (here && lane == 0) a.scales[row * a.ss + b] = s;
    } else {
      for (int j0 = 0; j0 < a.copies; j0 += L) {
        // lane l: place j0 + l, whose scale it stores
        int place = -1;
        if (here && j0 + lane < a.copies) place = a.places[(long long)row * a.copies + j0 + lane];
        if (place >= a.out_rows) place = -1;
        if (place >= 0) a.scales[place * a.ss + b] = s;
        // (the lanes' places beyond the last are -1)
#pragma unroll
        for (int j = 0; j < L; ++j) {
          const int to = __shfl_sync(ALL, place, j, L);
          if (to >= 0 && in) put(a.codes + to * a.cs + col);
        }
      }
    }
    row += step_rows;
    b += step_blocks;
    if (b >= a.blocks) { b -= a.blocks; ++row; }
  }
}

// Blocks of 128 x 128: a CTA per block, 16 rows to a warp.
template <class T, bool VEC> __global__ void __launch_bounds__(THREADS) dvm_quantize_block_kernel(const __grid_constant__ Args a) {
  constexpr int ROWS = DVM_SCALE_BLOCK / (THREADS / LANES);   // of a thread
  __shared__ float most[THREADS / 32];
  const int lane = threadIdx.x % LANES, b = blockIdx.x % a.blocks, rb = blockIdx.x / a.blocks;
  const int col = b * DVM_SCALE_BLOCK + 8 * lane, row0 = rb * DVM_SCALE_BLOCK + threadIdx.x / LANES;
  grid_ready();
  grid_wait();
  float2 v[ROWS][4];
  float m = 0.f;
#pragma unroll
  for (int i = 0; i < ROWS; ++i) {
    const int row = row0 + i * (THREADS / LANES);
    Raw<T, 8> x;
    x.clear();
    if (row < a.rows && col < a.cols) x.template load<VEC>((const T*)a.x + row * a.xs + col);
#pragma unroll
    for (int k = 0; k < 4; ++k) v[i][k] = x.pair(k);
  }
#pragma unroll
  for (int i = 0; i < ROWS; ++i)
#pragma unroll
    for (int k = 0; k < 4; ++k) m = max_abs(m, v[i][k]);
#pragma unroll
  for (int d = 16; d > 0; d >>= 1) m = max_abs(m, __shfl_xor_sync(ALL, m, d));
  if ((threadIdx.x & 31) == 0) most[threadIdx.x >> 5] = m;
  __syncthreads();
#pragma unroll
  for (int i = 0; i < THREADS / 32; ++i) m = max_abs(m, most[i]);
  const float s = scale_of(m);
#pragma unroll
  for (int i = 0; i < ROWS; ++i) {
    const int row = row0 + i * (THREADS / LANES);
    uint32_t c[2];
    const T* const from = (const T*)a.x + row * a.xs + col;
    codes_of<8>(v[i], s, 0x1p-21f, c, [&](int k, float edge) { return side(wide(from[k]), s, edge); });
    if (row < a.rows && col < a.cols) *(uint2*)(a.codes + row * a.cs + col) = make_uint2(c[0], c[1]);
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
  const int64_t ctas = dvm_up(d.rows * a.blocks, THREADS / (bf16 ? 8 : 16)), most = 8ll * dev.sm_count;
  auto launch = [&](auto kernel) { return dvm_launch_next(kernel, (int)(ctas < most ? ctas : most), THREADS, 0, stream, a); };
  if (bf16 && d.gated) return vec ? launch(dvm_quantize_kernel<__nv_bfloat16, true, true>) : launch(dvm_quantize_kernel<__nv_bfloat16, true, false>);
  if (bf16) return vec ? launch(dvm_quantize_kernel<__nv_bfloat16, false, true>) : launch(dvm_quantize_kernel<__nv_bfloat16, false, false>);
  if (d.gated) return vec ? launch(dvm_quantize_kernel<float, true, true>) : launch(dvm_quantize_kernel<float, true, false>);
  return vec ? launch(dvm_quantize_kernel<float, false, true>) : launch(dvm_quantize_kernel<float, false, false>);
}

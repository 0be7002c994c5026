// Rotary meta-kernel: norms of the query and key heads, rotation by position, keys and values into the paged cache.
//
// One pass: a head of D elements is read once and written once, by a group of 8, 16 or 32 lanes with 8 elements each
// (16 bytes of bf16 per load).  The mean of squares is a sum over the group's lanes; the partner of element i in a pair
// (i, i +- R/2) lies R/16 lanes away, four elements shifted when R/2 is not a multiple of 8; neighbouring pairs are in
// one lane.  A CTA works on the heads of one token, so position, slot and the angles are read once per thread and serve
// all its heads.  Everything between load and store is fp32; the store rounds once.
#include <cuda_bf16.h>
#include <cuda_runtime.h>

#include "dvm_launch.h"
#include "dvm_serving.h"

namespace dvm {
namespace rotary {

constexpr int THREADS = 256;
constexpr int UNROLL = 4;  // heads a group loads before it works on the first

struct Args {
  const void *q, *k, *v, *wq, *wk;
  const float* angles;
  const int *positions, *slots;
  void *q_out, *k_out, *v_out;
  long long qs[2], ks[2], vs[2], qo[2], ko[3], vo[3];
  int tokens, hq, hk, D, rot, angle_rows, n_slots, page, chunks;
  int lanes;       // lanes of a group
  int vec_in, vec_out, vec_w, vec_a;  // 16-byte accesses are aligned
  int norm, interleaved, paged, w_bf16;
  float eps;
};

__device__ __forceinline__ void load8(const __nv_bfloat16* p, bool vec, float (&x)[8]) {
  if (vec) {
    const uint4 r = *(const uint4*)p;
    const uint32_t w[4] = {r.x, r.y, r.z, r.w};
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      x[2 * i] = __uint_as_float(w[i] << 16);
      x[2 * i + 1] = __uint_as_float(w[i] & 0xffff0000u);
    }
  } else {
#pragma unroll
    for (int i = 0; i < 8; ++i) x[i] = __bfloat162float(p[i]);
  }
}
__device__ __forceinline__ void load8(const float* p, bool vec, float (&x)[8]) {
  if (vec) {
    const float4 a = ((const float4*)p)[0], b = ((const float4*)p)[1];
    x[0] = a.x; x[1] = a.y; x[2] = a.z; x[3] = a.w; x[4] = b.x; x[5] = b.y; x[6] = b.z; x[7] = b.w;
  } else {
#pragma unroll
    for (int i = 0; i < 8; ++i) x[i] = p[i];
  }
}
__device__ __forceinline__ void store8(__nv_bfloat16* p, bool vec, const float (&x)[8]) {
  if (vec) {
    uint32_t w[4];
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      const __nv_bfloat162 h = __floats2bfloat162_rn(x[2 * i], x[2 * i + 1]);
      w[i] = *(const uint32_t*)&h;
    }
    *(uint4*)p = make_uint4(w[0], w[1], w[2], w[3]);
  } else {
#pragma unroll
    for (int i = 0; i < 8; ++i) p[i] = __float2bfloat16_rn(x[i]);
  }
}
__device__ __forceinline__ void store8(float* p, bool vec, const float (&x)[8]) {
  if (vec) {
    ((float4*)p)[0] = make_float4(x[0], x[1], x[2], x[3]);
    ((float4*)p)[1] = make_float4(x[4], x[5], x[6], x[7]);
  } else {
#pragma unroll
    for (int i = 0; i < 8; ++i) p[i] = x[i];
  }
}

template <class TI, class TO>
__global__ void __launch_bounds__(THREADS) dvm_rotary_kernel(const __grid_constant__ Args a) {
  const int L = a.lanes, group = threadIdx.x / L, lane = threadIdx.x & (L - 1), groups = THREADS / L;
  const int e0 = lane * 8;                       // first element of this lane
  const bool live = e0 < a.D;
  const int heads = a.hq + a.hk * (a.paged ? 2 : 1);
  const int half = a.rot >> 1;

  float wq[8], wk[8];
  if (a.norm && live) {
    if (a.w_bf16) {
      load8((const __nv_bfloat16*)a.wq + e0, a.vec_w, wq);
      load8((const __nv_bfloat16*)a.wk + e0, a.vec_w, wk);
    } else {
      load8((const float*)a.wq + e0, a.vec_w, wq);
      load8((const float*)a.wk + e0, a.vec_w, wk);
    }
  }
  const long long items = (long long)a.tokens * a.chunks;
  for (long long item = blockIdx.x; item < items; item += gridDim.x) {
    const int t = (int)(item / a.chunks), chunk = (int)(item % a.chunks);
    const int pos = a.positions[t];
    if (pos < 0 || pos >= a.angle_rows) continue;  // (the whole CTA: t is the same for all its threads)
    long long k_at = 0, v_at = 0;
    bool stored = true;
    if (a.paged) {
      const int slot = a.slots[t];
      stored = slot >= 0 && slot < a.n_slots;
      const int page = slot / a.page, off = slot % a.page;
      k_at = page * a.ko[0] + off * a.ko[1];
      v_at = page * a.vo[0] + off * a.vo[1];
    } else {
      k_at = t * a.ko[0];
    }
    // cos and sin of this lane's elements: of pair (i mod R/2) for halves, of pair i / 2 for neighbours
    float c[8], s[8];
    if (e0 < a.rot) {
      const float* row = a.angles + (long long)pos * a.rot;
      if (a.interleaved) {
#pragma unroll
        for (int g = 0; g < 2; ++g) {  // (an element past rot stays: R is a multiple of 8, so whole lanes are in or out)
#pragma unroll
          for (int i = 0; i < 2; ++i) {
            const int k = (e0 >> 1) + 2 * g + i;
            c[4 * g + 2 * i] = c[4 * g + 2 * i + 1] = row[k];
            s[4 * g + 2 * i] = s[4 * g + 2 * i + 1] = row[half + k];
          }
        }
      } else {
#pragma unroll
        for (int g = 0; g < 2; ++g) {
          const int i = e0 + 4 * g, k = i < half ? i : i - half;
          if (a.vec_a) {
            const float4 cc = *(const float4*)(row + k), ss = *(const float4*)(row + half + k);
            c[4 * g] = cc.x; c[4 * g + 1] = cc.y; c[4 * g + 2] = cc.z; c[4 * g + 3] = cc.w;
            s[4 * g] = ss.x; s[4 * g + 1] = ss.y; s[4 * g + 2] = ss.z; s[4 * g + 3] = ss.w;
          } else {
#pragma unroll
            for (int e = 0; e < 4; ++e) { c[4 * g + e] = row[k + e]; s[4 * g + e] = row[half + k + e]; }
          }
        }
      }
    }
    const int per = (heads + a.chunks - 1) / a.chunks, h_end = min(heads, (chunk + 1) * per);
    for (int hb = chunk * per; hb < h_end; hb += groups * UNROLL) {
      float x[UNROLL][8];
#pragma unroll
      for (int u = 0; u < UNROLL; ++u) {
        const int h = hb + u * groups + group;
#pragma unroll
        for (int i = 0; i < 8; ++i) x[u][i] = 0.f;
        if (h < h_end && live) {
          const TI* p = h < a.hq          ? (const TI*)a.q + t * a.qs[0] + h * a.qs[1]
                        : h < a.hq + a.hk ? (const TI*)a.k + t * a.ks[0] + (h - a.hq) * a.ks[1]
                                          : (const TI*)a.v + t * a.vs[0] + (h - a.hq - a.hk) * a.vs[1];
          load8(p + e0, a.vec_in, x[u]);
        }
      }
#pragma unroll
      for (int u = 0; u < UNROLL; ++u) {
        const int h = hb + u * groups + group;
        if (hb + u * groups >= h_end) break;  // (the same for the whole CTA: the shuffles below stay converged)
        const bool is_q = h < a.hq, is_v = h >= a.hq + a.hk;
        float y[8];
        float r = 1.f;
        if (a.norm) {
          float sum = 0.f;
#pragma unroll
          for (int i = 0; i < 8; ++i) sum = fmaf(x[u][i], x[u][i], sum);
          for (int d = L >> 1; d > 0; d >>= 1) sum += __shfl_xor_sync(0xffffffffu, sum, d);
          r = rsqrtf(sum / (float)a.D + a.eps);
#pragma unroll
          for (int i = 0; i < 8; ++i) y[i] = live ? x[u][i] * r * (is_q ? wq[i] : wk[i]) : 0.f;
        } else {
#pragma unroll
          for (int i = 0; i < 8; ++i) y[i] = x[u][i];
        }
        float z[8];
        if (a.interleaved) {
#pragma unroll
          for (int i = 0; i < 8; i += 2) { z[i] = -y[i + 1]; z[i + 1] = y[i]; }
        } else {
          // the partner of element i: i + R/2 below R/2, i - R/2 from there on (elsewhere unused)
          const int shift = half & 7;  // 0 or 4
#pragma unroll
          for (int g = 0; g < 2; ++g) {
            const int i = e0 + 4 * g, from = i < half ? i + half : i - half;
            const int src = (from >> 3) & (L - 1);
#pragma unroll
            for (int e = 0; e < 4; ++e) {
              const float same = __shfl_sync(0xffffffffu, y[4 * g + e], src, L);
              const float other = __shfl_sync(0xffffffffu, y[4 * (1 - g) + e], src, L);
              const float p = shift ? other : same;
              z[4 * g + e] = i < half ? -p : p;
            }
          }
        }
        if (e0 < a.rot) {
#pragma unroll
          for (int i = 0; i < 8; ++i) y[i] = fmaf(z[i], s[i], y[i] * c[i]);
        }
        if (h < h_end && live) {
          if (is_v) {
            if (stored) store8((TO*)a.v_out + v_at + (h - a.hq - a.hk) * a.vo[2] + e0, a.vec_out, x[u]);
          } else if (is_q) {
            store8((TO*)a.q_out + t * a.qo[0] + h * a.qo[1] + e0, a.vec_out, y);
          } else if (stored) {
            store8((TO*)a.k_out + k_at + (h - a.hq) * (a.paged ? a.ko[2] : a.ko[1]) + e0, a.vec_out, y);
          }
        }
      }
    }
  }
}

}  // namespace rotary
}  // namespace dvm

int dvm_launch_rotary(const dvm_rotary_desc& d, void* const* t, cudaStream_t stream) {
  using namespace dvm::rotary;
  DvmDeviceInfo dev;
  const int st = dvm_device_state(&dev);
  if (st != DVM_OK) return st;
  const RotarySlots sl = dvm_rotary_slots(d);
  Args a = {};
  a.q = t[sl.q]; a.k = t[sl.k]; a.angles = (const float*)t[sl.angles]; a.positions = (const int*)t[sl.positions];
  a.q_out = t[sl.q_out]; a.k_out = t[sl.k_out];
  if (d.norm) { a.wq = t[sl.wq]; a.wk = t[sl.wk]; }
  if (d.paged) { a.v = t[sl.v]; a.slots = (const int*)t[sl.slots]; a.v_out = t[sl.v_out]; }
  const int64_t ei = d.dtype == DVM_BF16 ? 2 : 4, eo = d.out_dtype == DVM_BF16 ? 2 : 4;
  // 16-byte accesses: a lane's 8 elements start a multiple of 8 elements into a row of strides and pointers to 16 bytes
  auto aligned = [](const void* p, const long long* s, int n, int64_t es) {
    bool ok = ((uintptr_t)p & 15) == 0;
    for (int i = 0; i < n; ++i) ok = ok && s[i] * es % 16 == 0;
    return ok;
  };
  for (int i = 0; i < 2; ++i) { a.qs[i] = d.q_stride[i]; a.ks[i] = d.k_stride[i]; a.vs[i] = d.v_stride[i]; a.qo[i] = d.q_out_stride[i]; a.ko[i] = d.k_out_stride[i]; }
  if (d.paged) for (int i = 0; i < 3; ++i) { a.ko[i] = d.k_cache_stride[i]; a.vo[i] = d.v_cache_stride[i]; }
  a.vec_in = aligned(a.q, a.qs, 2, ei) && aligned(a.k, a.ks, 2, ei) && (!d.paged || aligned(a.v, a.vs, 2, ei));
  a.vec_out = aligned(a.q_out, a.qo, 2, eo) && aligned(a.k_out, a.ko, d.paged ? 3 : 2, eo) && (!d.paged || aligned(a.v_out, a.vo, 3, eo));
  a.vec_w = d.norm && ((uintptr_t)a.wq & 15) == 0 && ((uintptr_t)a.wk & 15) == 0;
  a.vec_a = ((uintptr_t)a.angles & 15) == 0;
  a.tokens = (int)d.tokens; a.hq = (int)d.q_heads; a.hk = (int)d.kv_heads; a.D = (int)d.head_dim; a.rot = (int)d.rotary_dim;
  a.angle_rows = (int)d.angle_rows; a.n_slots = d.paged ? (int)(d.pages * d.page_size) : 0; a.page = d.paged ? (int)d.page_size : 1;
  a.norm = d.norm; a.interleaved = d.interleaved; a.paged = d.paged; a.w_bf16 = d.weight_dtype == DVM_BF16; a.eps = d.eps;
  a.lanes = d.head_dim <= 64 ? 8 : d.head_dim <= 128 ? 16 : 32;
  // few tokens: their heads are spread over CTAs until every SM has some
  const int heads = a.hq + a.hk * (d.paged ? 2 : 1), groups = THREADS / a.lanes, most = (heads + groups - 1) / groups;
  const int64_t want = 4 * (int64_t)dev.sm_count / d.tokens;
  a.chunks = (int)(want < 1 ? 1 : want < most ? want : most);
  const int64_t items = d.tokens * a.chunks, cap = 64 * (int64_t)dev.sm_count;
  const int grid = (int)(items < cap ? items : cap);
  if (d.dtype == DVM_BF16) {
    if (d.out_dtype == DVM_BF16) dvm_rotary_kernel<__nv_bfloat16, __nv_bfloat16><<<grid, THREADS, 0, stream>>>(a);
    else dvm_rotary_kernel<__nv_bfloat16, float><<<grid, THREADS, 0, stream>>>(a);
  } else {
    if (d.out_dtype == DVM_BF16) dvm_rotary_kernel<float, __nv_bfloat16><<<grid, THREADS, 0, stream>>>(a);
    else dvm_rotary_kernel<float, float><<<grid, THREADS, 0, stream>>>(a);
  }
  DVM_CUDA(cudaGetLastError());
  dvm_count_launch();
  return DVM_OK;
}

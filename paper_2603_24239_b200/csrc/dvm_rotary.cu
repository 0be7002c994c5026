// Rotary meta-kernel: norms of the query and key heads, rotation by position, keys and values into the paged cache.
//
// One pass, bound by memory: a head of D elements is read once and written once, by a group of 8, 16 or 32 lanes with two
// runs of 4 elements each.  The runs are laid so that a pair is always in one lane: lane l < R / 8 holds the elements
// [4 l, 4 l + 4) and [R / 2 + 4 l, R / 2 + 4 l + 4) of a head whose halves are paired, [8 l, 8 l + 8) where neighbours
// are, and every lane from R / 8 on holds [8 l, 8 l + 8), which stay.  Rotation then takes no exchange between lanes, and
// either way a lane needs cos and sin of the pairs [4 l, 4 l + 4): 16 bytes each.  Only the mean of squares crosses lanes.
// A CTA works on the heads of one token, so position, slot and angles are read once per thread and serve all its heads;
// the heads' loads go out before anything waits for the position.  Everything between load and store is fp32; the store
// rounds once.
#include <cuda_bf16.h>
#include <cuda_runtime.h>

#include "dvm_launch.h"
#include "dvm_serving.h"

namespace dvm {
namespace rotary {

constexpr int THREADS = 256;
constexpr int UNROLL = 3;  // heads a group loads before it works on the first

struct Args {
  const void *q, *k, *v, *wq, *wk;
  const float* angles;
  const int *positions, *slots;
  void *q_out, *k_out, *v_out;
  long long qs[2], ks[2], vs[2], qo[2], ko[3], vo[3];
  int tokens, hq, hk, D, rot, angle_rows, n_slots, page, chunks;
  int lanes;       // lanes of a group
  int vec_in, vec_out, vec_a;  // runs of 4 elements are aligned
  int norm, interleaved, paged, w_bf16;
  float eps;
};

// Four elements as they lie in memory, and as fp32.
template <class T> struct Run;
template <> struct Run<__nv_bfloat16> {
  uint2 w;
  __device__ __forceinline__ void load(const __nv_bfloat16* p, bool vec) {
    if (vec) {
      w = *(const uint2*)p;
    } else {
      const uint16_t* h = (const uint16_t*)p;
      w = make_uint2(h[0] | ((uint32_t)h[1] << 16), h[2] | ((uint32_t)h[3] << 16));
    }
  }
  __device__ __forceinline__ void get(float* x) const {
    x[0] = __uint_as_float(w.x << 16);
    x[1] = __uint_as_float(w.x & 0xffff0000u);
    x[2] = __uint_as_float(w.y << 16);
    x[3] = __uint_as_float(w.y & 0xffff0000u);
  }
};
template <> struct Run<float> {
  float4 w;
  __device__ __forceinline__ void load(const float* p, bool vec) { w = vec ? *(const float4*)p : make_float4(p[0], p[1], p[2], p[3]); }
  __device__ __forceinline__ void get(float* x) const { x[0] = w.x; x[1] = w.y; x[2] = w.z; x[3] = w.w; }
};
__device__ __forceinline__ void store4(__nv_bfloat16* p, bool vec, const float* x) {
  const __nv_bfloat162 a = __floats2bfloat162_rn(x[0], x[1]), b = __floats2bfloat162_rn(x[2], x[3]);
  if (vec) {
    *(uint2*)p = make_uint2(*(const uint32_t*)&a, *(const uint32_t*)&b);
  } else {
    p[0] = a.x; p[1] = a.y; p[2] = b.x; p[3] = b.y;
  }
}
__device__ __forceinline__ void store4(float* p, bool vec, const float* x) {
  if (vec) {
    *(float4*)p = make_float4(x[0], x[1], x[2], x[3]);
  } else {
#pragma unroll
    for (int i = 0; i < 4; ++i) p[i] = x[i];
  }
}

template <class TI, class TO>
__global__ void __launch_bounds__(THREADS, sizeof(TI) == 2 ? 4 : 3) dvm_rotary_kernel(const __grid_constant__ Args a) {
  const int L = a.lanes, group = threadIdx.x / L, lane = threadIdx.x & (L - 1), groups = THREADS / L;
  const bool live = 8 * lane < a.D, turned = 8 * lane < a.rot;
  const bool halves = turned && !a.interleaved;
  const int at0 = halves ? 4 * lane : 8 * lane, at1 = halves ? (a.rot >> 1) + 4 * lane : 8 * lane + 4;  // this lane's two runs
  const int heads = a.hq + a.hk * (a.paged ? 2 : 1);

  float wq[8], wk[8];
  if (a.norm && live) {
    if (a.w_bf16) {
      Run<__nv_bfloat16> r;
      r.load((const __nv_bfloat16*)a.wq + at0, false); r.get(wq);
      r.load((const __nv_bfloat16*)a.wq + at1, false); r.get(wq + 4);
      r.load((const __nv_bfloat16*)a.wk + at0, false); r.get(wk);
      r.load((const __nv_bfloat16*)a.wk + at1, false); r.get(wk + 4);
    } else {
      Run<float> r;
      r.load((const float*)a.wq + at0, false); r.get(wq);
      r.load((const float*)a.wq + at1, false); r.get(wq + 4);
      r.load((const float*)a.wk + at0, false); r.get(wk);
      r.load((const float*)a.wk + at1, false); r.get(wk + 4);
    }
  }
  const int per = (heads + a.chunks - 1) / a.chunks;
  const long long items = (long long)a.tokens * a.chunks;
  for (long long item = blockIdx.x; item < items; item += gridDim.x) {
    const int t = (int)(item / a.chunks), chunk = (int)(item - (long long)t * a.chunks);
    const int h_end = min(heads, (chunk + 1) * per);
    Run<TI> x[UNROLL][2];
    auto fetch = [&](int hb) {
#pragma unroll
      for (int u = 0; u < UNROLL; ++u) {
        const int h = hb + u * groups + group;
        if (h < h_end && live) {
          const TI* p = h < a.hq          ? (const TI*)a.q + t * a.qs[0] + h * a.qs[1]
                        : h < a.hq + a.hk ? (const TI*)a.k + t * a.ks[0] + (h - a.hq) * a.ks[1]
                                          : (const TI*)a.v + t * a.vs[0] + (h - a.hq - a.hk) * a.vs[1];
          x[u][0].load(p + at0, a.vec_in);
          x[u][1].load(p + at1, a.vec_in);
        }
      }
    };
    fetch(chunk * per);
    const int pos = a.positions[t];
    if (pos < 0 || pos >= a.angle_rows) continue;  // (the whole CTA: t is the same for all its threads)
    long long k_at = t * a.ko[0], v_at = 0;
    bool stored = true;
    if (a.paged) {
      const int slot = a.slots[t];
      stored = slot >= 0 && slot < a.n_slots;
      const int page = slot / a.page, off = slot - page * a.page;
      k_at = page * a.ko[0] + off * a.ko[1];
      v_at = page * a.vo[0] + off * a.vo[1];
    }
    float c[4], s[4];  // of the pairs [4 lane, 4 lane + 4)
    if (turned) {
      const float* row = a.angles + (long long)pos * a.rot + 4 * lane;
      Run<float> r;
      r.load(row, a.vec_a); r.get(c);
      r.load(row + (a.rot >> 1), a.vec_a); r.get(s);
    }
    for (int hb = chunk * per; hb < h_end; hb += groups * UNROLL) {
      if (hb != chunk * per) fetch(hb);
#pragma unroll
      for (int u = 0; u < UNROLL; ++u) {
        if (hb + u * groups >= h_end) break;  // (the same for the whole CTA: the shuffles below stay converged)
        const int h = hb + u * groups + group;
        const bool mine = h < h_end && live, is_q = h < a.hq, is_v = h >= a.hq + a.hk;
        float y[8] = {};
        if (mine) {
          x[u][0].get(y);
          x[u][1].get(y + 4);
        }
        if (a.norm) {
          float sum = 0.f;
#pragma unroll
          for (int i = 0; i < 8; ++i) sum = fmaf(y[i], y[i], sum);
          for (int d = L >> 1; d > 0; d >>= 1) sum += __shfl_xor_sync(0xffffffffu, sum, d);
          if (!is_v) {
            const float r = rsqrtf(sum / (float)a.D + a.eps);
#pragma unroll
            for (int i = 0; i < 8; ++i) y[i] = y[i] * r * (is_q ? wq[i] : wk[i]);
          }
        }
        if (!mine || (!is_q && !stored)) continue;
        if (turned && !is_v) {
          if (a.interleaved) {
#pragma unroll
            for (int i = 0; i < 4; ++i) {
              const float p = y[2 * i], q = y[2 * i + 1];
              y[2 * i] = p * c[i] - q * s[i];
              y[2 * i + 1] = q * c[i] + p * s[i];
            }
          } else {
#pragma unroll
            for (int i = 0; i < 4; ++i) {
              const float p = y[i], q = y[4 + i];
              y[i] = p * c[i] - q * s[i];
              y[4 + i] = q * c[i] + p * s[i];
            }
          }
        }
        TO* out = is_q   ? (TO*)a.q_out + t * a.qo[0] + h * a.qo[1]
                  : is_v ? (TO*)a.v_out + v_at + (h - a.hq - a.hk) * a.vo[2]
                         : (TO*)a.k_out + k_at + (h - a.hq) * (a.paged ? a.ko[2] : a.ko[1]);
        store4(out + at0, a.vec_out, y);
        store4(out + at1, a.vec_out, y + 4);
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
  // a run of 4 elements in one access: it starts a multiple of 4 elements into a row
  auto aligned = [](const void* p, const long long* s, int n, int64_t es) {
    bool ok = (uintptr_t)p % (4 * es) == 0;
    for (int i = 0; i < n; ++i) ok = ok && s[i] % 4 == 0;
    return ok;
  };
  for (int i = 0; i < 2; ++i) { a.qs[i] = d.q_stride[i]; a.ks[i] = d.k_stride[i]; a.vs[i] = d.v_stride[i]; a.qo[i] = d.q_out_stride[i]; a.ko[i] = d.k_out_stride[i]; }
  if (d.paged) for (int i = 0; i < 3; ++i) { a.ko[i] = d.k_cache_stride[i]; a.vo[i] = d.v_cache_stride[i]; }
  a.vec_in = aligned(a.q, a.qs, 2, ei) && aligned(a.k, a.ks, 2, ei) && (!d.paged || aligned(a.v, a.vs, 2, ei));
  a.vec_out = aligned(a.q_out, a.qo, 2, eo) && aligned(a.k_out, a.ko, d.paged ? 3 : 2, eo) && (!d.paged || aligned(a.v_out, a.vo, 3, eo));
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

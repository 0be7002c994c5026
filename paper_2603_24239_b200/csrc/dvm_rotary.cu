// Rotary meta-kernel: norms of the query and key heads, rotation by position, keys and values into the paged cache.
//
// One pass, bound by memory: a head of D elements is read once and written once, by a group of 8, 16 or 32 lanes with two
// runs of 4 elements each, so laid that a pair is always in one lane and that the lanes' runs lie side by side: lane
// l < R / 8 holds the elements [4 l, 4 l + 4) and [R / 2 + 4 l, R / 2 + 4 l + 4) of the part that turns, the lanes from
// R / 8 on hold the rest, which stays, in the same manner.  Rotation then takes no exchange between lanes, whether halves
// or neighbours are paired.  Only the mean of squares crosses lanes.  (8 elements in a row per lane where
// fp32 neighbours are paired, so that every access left out every other 16 bytes: 1531 tokens of 40 + 8 + 8 heads of 96 17.6 us
// on the device, 13.0 now, with data that stays in L2; 14.6 with three sets of it in turn.)
// A CTA keeps the same heads for all tokens it takes -- all of them, or a part where there are more than its groups can
// have in flight -- so what a thread reads and writes is found once and moves by a stride; position, slot and angles are
// read once per thread and token, and while one token is computed the heads and angles of the next are on their way, and
// the position and slot of the one after it.  Everything between load and store is fp32 (two elements to an
// instruction); the store rounds once.  With the head's place worked out anew for every token, the same kernel took 744
// instructions per warp and token and was bound by them: 80 us for 8192 tokens of 32 + 8 + 8 heads of 128.  With the next
// token's data in registers (one token ahead, two CTAs per SM) it was bound by what is in flight: 50 us.  Now each
// thread copies its own runs into shared memory (cp.async, DEPTH tokens ahead) and reads them from there: 41 us in calls in a
// row, 5.0 TB/s (37 us in a chain of captured launches, 39 in bursts); one token 1.8 us in such a chain.
#include <cuda_bf16.h>
#include <cuda_runtime.h>

#include "dvm_launch.h"
#include "dvm_serving.h"
#include "dvm_sm100.cuh"

namespace dvm {
namespace rotary {

using namespace sm100;

constexpr int THREADS = 256;   // at most
constexpr int DEPTH = 2;       // tokens on their way
constexpr int UNROLL = 3;      // heads of a group
// bytes of a thread: per token on its way two runs of each head, and cos and sin
template <class T> constexpr int BYTES = DEPTH * (UNROLL * 2 * 4 * (int)sizeof(T) + 32);

struct Args {
  const void *q, *k, *v, *wq, *wk;
  const float* angles;
  const int *positions, *slots;
  void *q_out, *k_out, *v_out;
  long long qs[2], ks[2], vs[2], qo[2], ko[3], vo[3];
  int tokens, hq, hk, D, rot, angle_rows, n_slots, page, page_log, chunks;  // page_log: -1 where page is no power of two
  int lanes;       // lanes of a group
  int vec;         // runs of 4 elements are aligned in every tensor
  int norm, interleaved, paged, w_bf16;
  float eps, inv_D;
};

__device__ __forceinline__ void copy8(uint32_t dst, const void* p) { asm volatile("cp.async.ca.shared.global [%0], [%1], 8;" ::"r"(dst), "l"(p) : "memory"); }

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
  static __device__ __forceinline__ void copy(uint32_t dst, const __nv_bfloat16* p) {
    copy8(dst, p);
  }
  __device__ __forceinline__ void get(float2* x) const {
    x[0] = make_float2(__uint_as_float(w.x << 16), __uint_as_float(w.x & 0xffff0000u));
    x[1] = make_float2(__uint_as_float(w.y << 16), __uint_as_float(w.y & 0xffff0000u));
  }
};
template <> struct Run<float> {
  float4 w;
  __device__ __forceinline__ void load(const float* p, bool vec) { w = vec ? *(const float4*)p : make_float4(p[0], p[1], p[2], p[3]); }
  static __device__ __forceinline__ void copy(uint32_t dst, const float* p) {
    asm volatile("cp.async.cg.shared.global [%0], [%1], 16;" ::"r"(dst), "l"(p) : "memory");
  }
  __device__ __forceinline__ void get(float2* x) const { x[0] = make_float2(w.x, w.y); x[1] = make_float2(w.z, w.w); }
};
__device__ __forceinline__ void store4(__nv_bfloat16* p, bool vec, const float2* x) {
  const __nv_bfloat162 a = __float22bfloat162_rn(x[0]), b = __float22bfloat162_rn(x[1]);
  if (vec) {
    *(uint2*)p = make_uint2(*(const uint32_t*)&a, *(const uint32_t*)&b);
  } else {
    p[0] = a.x; p[1] = a.y; p[2] = b.x; p[3] = b.y;
  }
}
__device__ __forceinline__ void store4(float* p, bool vec, const float2* x) {
  if (vec) {
    *(float4*)p = make_float4(x[0].x, x[0].y, x[1].x, x[1].y);
  } else {
    p[0] = x[0].x; p[1] = x[0].y; p[2] = x[1].x; p[3] = x[1].y;
  }
}

// LANES: lanes of a group, VEC: runs of 4 elements are aligned everywhere, INTER: neighbours are paired; 0, false, false: the
// kernel for the other layouts.
template <class TI, class TO, int LANES, bool VEC, bool INTER>
__global__ void __launch_bounds__(THREADS, VEC ? 3 : 2) dvm_rotary_kernel(const __grid_constant__ Args a) {
  constexpr int U = UNROLL;
  extern __shared__ __align__(16) uint8_t smem[];
  const int L = LANES ? LANES : a.lanes, group = threadIdx.x / L, lane = threadIdx.x & (L - 1), groups = blockDim.x / L;
  const bool live = 8 * lane < a.D, turned = 8 * lane < a.rot;
  // this lane's two runs, and where the cosines of their pairs are: two from c0 on, two from c1 on
  const int from = turned ? 0 : a.rot, width = turned ? a.rot : a.D - a.rot, nth = turned ? lane : lane - (a.rot >> 3);
  // bf16 neighbours stay in a row: their 8 elements are 16 bytes, and so are their cosines (40.2 us in two runs, 38.5 in one,
  // for the 8192 tokens above)
  constexpr bool IN_A_ROW = VEC && INTER && sizeof(TI) == 2 && sizeof(TO) == 2;
  const bool interleaved = VEC ? INTER : a.interleaved;
  const int at0 = IN_A_ROW && turned ? 8 * lane : from + 4 * nth, at1 = at0 + (IN_A_ROW && turned ? 4 : width >> 1);
  const bool apart = interleaved && !IN_A_ROW;
  const int c0 = apart ? 2 * lane : 4 * lane, c1 = apart ? (a.rot >> 2) + 2 * lane : 4 * lane + 2;
  const int heads = a.hq + a.hk * (a.paged ? 2 : 1);

  __shared__ float4 weight[2][2][32];  // [query, key][run][lane]
  // This thread's heads: chunk per + u groups + group, where they read and write for token 0, and what a token adds.
  enum { QUERY, KEY, VALUE, NONE };
  const int chunk = blockIdx.x % a.chunks, step = gridDim.x / a.chunks, per = (heads + a.chunks - 1) / a.chunks;
  long long t = blockIdx.x / a.chunks;
  const TI* src[U];
  long long add[U];
  TO* dst[U];
  int kind[U];
#pragma unroll
  for (int u = 0; u < U; ++u) {
    const int i = u * groups + group, h = chunk * per + i;
    kind[u] = i >= per || h >= heads || !live ? NONE : h < a.hq ? QUERY : h < a.hq + a.hk ? KEY : VALUE;
    const int hh = kind[u] == QUERY ? h : kind[u] == KEY ? h - a.hq : h - a.hq - a.hk;
    if (kind[u] == QUERY) {
      src[u] = (const TI*)a.q + hh * a.qs[1];
      add[u] = a.qs[0];
      dst[u] = (TO*)a.q_out + hh * a.qo[1];
    } else if (kind[u] == KEY) {
      src[u] = (const TI*)a.k + hh * a.ks[1];
      add[u] = a.ks[0];
      dst[u] = (TO*)a.k_out + hh * (a.paged ? a.ko[2] : a.ko[1]);
    } else {
      src[u] = (const TI*)a.v + hh * a.vs[1];
      add[u] = a.vs[0];
      dst[u] = (TO*)a.v_out + hh * a.vo[2];
    }
    src[u] += at0 + t * add[u];
    add[u] *= step;
    dst[u] += at0;
  }
  const int run = at1 - at0;
  grid_ready();  // (one token in a chain of launches 1.75 us, 2.17 without)
  grid_wait();

  struct Place { int pos, slot; };
  auto place_of = [&](long long t) -> Place {
    Place p = {-1, -1};
    if (t < a.tokens) {
      p.pos = a.positions[t];
      if (a.paged) p.slot = a.slots[t];
    }
    return p;
  };
  auto in_table = [&](Place p) -> bool { return p.pos >= 0 && p.pos < a.angle_rows; };  // (the same for the whole CTA)
  // Token i of this CTA goes through place i mod DEPTH of the thread's shared memory: 2 U runs, cos, sin.
  constexpr uint32_t RUN = 4 * sizeof(TI);
  const uint32_t place_bytes = blockDim.x * (2 * U * RUN + 32), mine = threadIdx.x * RUN, mine_cs = blockDim.x * 2 * U * RUN + threadIdx.x * 16;
  const uint32_t base = smem_u32(smem);
  auto fetch = [&](uint32_t place, long long t, Place p) {  // of the token that src points to
    if (VEC && t < a.tokens) {
#pragma unroll
      for (int u = 0; u < U; ++u)
        if (kind[u] != NONE) {
          Run<TI>::copy(base + place + mine + (2 * u) * blockDim.x * RUN, src[u]);
          Run<TI>::copy(base + place + mine + (2 * u + 1) * blockDim.x * RUN, src[u] + run);
        }
      if (turned && in_table(p)) {
        const float* row = a.angles + (long long)p.pos * a.rot;
        const uint32_t to = base + place + mine_cs;
#pragma unroll
        for (int i = 0; i < 2; ++i, row += a.rot >> 1) {  // cos, sin
          if (apart) {
            copy8(to + i * blockDim.x * 16, row + c0);
            copy8(to + i * blockDim.x * 16 + 8, row + c1);
          } else {
            Run<float>::copy(to + i * blockDim.x * 16, row + c0);
          }
        }
      }
    }
    asm volatile("cp.async.commit_group;" ::: "memory");
  };
  auto compute = [&](uint32_t place, long long t, Place p) {
    if (!in_table(p)) return;
    const uint8_t* const here = smem + place;
    Run<TI> x[U][2];
    Run<float> dc, ds;
    if (VEC) {
#pragma unroll
      for (int u = 0; u < U; ++u)
#pragma unroll
        for (int i = 0; i < 2; ++i) x[u][i] = *(const Run<TI>*)(here + mine + (2 * u + i) * blockDim.x * RUN);
      dc = *(const Run<float>*)(here + mine_cs);
      ds = *(const Run<float>*)(here + mine_cs + blockDim.x * 16);
    } else {
#pragma unroll
      for (int u = 0; u < U; ++u)
        if (kind[u] != NONE) {
          x[u][0].load(src[u], false);
          x[u][1].load(src[u] + run, false);
        }
      if (turned) {
        const float *row = a.angles + (long long)p.pos * a.rot, *sines = row + (a.rot >> 1);
        dc.w = make_float4(row[c0], row[c0 + 1], row[c1], row[c1 + 1]);
        ds.w = make_float4(sines[c0], sines[c0 + 1], sines[c1], sines[c1 + 1]);
      }
    }
    const long long q_at = t * a.qo[0];
    long long k_at = 0, v_at = 0;
    bool stored = true;
    if (a.paged) {
      stored = p.slot >= 0 && p.slot < a.n_slots;
      const int page = a.page_log >= 0 ? p.slot >> a.page_log : p.slot / a.page, off = p.slot - page * a.page;
      k_at = page * a.ko[0] + off * a.ko[1];
      v_at = page * a.vo[0] + off * a.vo[1];
    } else {
      k_at = t * a.ko[0];
    }
    float2 c[2], s[2], ns[2];
    dc.get(c);
    ds.get(s);
#pragma unroll
    for (int i = 0; i < 2; ++i) ns[i] = make_float2(-s[i].x, -s[i].y);
#pragma unroll
    for (int u = 0; u < U; ++u) {
      if (u * groups >= per) break;  // (the same for the whole CTA: the shuffles below stay converged)
      float2 y[4] = {};
      if (kind[u] != NONE) {
        x[u][0].get(y);
        x[u][1].get(y + 2);
      }
      if (a.norm) {
        float2 sq = mul2(y[0], y[0]);
#pragma unroll
        for (int i = 1; i < 4; ++i) sq = fma2(y[i], y[i], sq);
        float sum = sq.x + sq.y;
        if (LANES) {
#pragma unroll
          for (int e = LANES >> 1; e > 0; e >>= 1) sum += __shfl_xor_sync(0xffffffffu, sum, e);
        } else {
          for (int e = L >> 1; e > 0; e >>= 1) sum += __shfl_xor_sync(0xffffffffu, sum, e);
        }
        if (kind[u] <= KEY) {
          const float r = rsqrtf(sum * a.inv_D + a.eps);
          const float4 w0 = weight[kind[u]][0][lane], w1 = weight[kind[u]][1][lane];
          const float2 w[4] = {make_float2(w0.x, w0.y), make_float2(w0.z, w0.w), make_float2(w1.x, w1.y), make_float2(w1.z, w1.w)};
#pragma unroll
          for (int i = 0; i < 4; ++i) y[i] = mul2(mul2(y[i], make_float2(r, r)), w[i]);
        }
      }
      if (kind[u] == NONE || (kind[u] != QUERY && !stored)) continue;
      if (turned && kind[u] != VALUE) {
        if (interleaved) {  // y[i] is pair i
          const float cc[4] = {c[0].x, c[0].y, c[1].x, c[1].y}, ss[4] = {s[0].x, s[0].y, s[1].x, s[1].y};
#pragma unroll
          for (int i = 0; i < 4; ++i) y[i] = fma2(make_float2(-y[i].y, y[i].x), make_float2(ss[i], ss[i]), mul2(y[i], make_float2(cc[i], cc[i])));
        } else {              // y[i] and y[2 + i] are the halves of two pairs
#pragma unroll
          for (int i = 0; i < 2; ++i) {
            const float2 p0 = y[i], p1 = y[2 + i];
            y[i] = fma2(p1, ns[i], mul2(p0, c[i]));
            y[2 + i] = fma2(p0, s[i], mul2(p1, c[i]));
          }
        }
      }
      TO* const out = dst[u] + (kind[u] == QUERY ? q_at : kind[u] == KEY ? k_at : v_at);
      store4(out, VEC, y);
      store4(out + run, VEC, y + 2);
    }
  };
  // (with VEC src runs DEPTH tokens ahead of t)
  Place p[DEPTH + 1];
#pragma unroll
  for (int i = 0; i <= DEPTH; ++i) p[i] = place_of(t + i * step);
  auto advance = [&]() {
#pragma unroll
    for (int u = 0; u < U; ++u) src[u] += add[u];
  };
  if (VEC) {
#pragma unroll
    for (int i = 0; i < DEPTH; ++i) {
      fetch(i * place_bytes, t + i * step, p[i]);
      advance();
    }
  }
  // (the weights last: nothing but the first token's sums waits for them)
  for (int i = threadIdx.x; a.norm && i < 2 * L && live; i += blockDim.x) {  // (blockDim is a multiple of L: i has this lane)
    const void* w = i < L ? a.wq : a.wk;
    float v[8];
#pragma unroll
    for (int j = 0; j < 8; ++j) {
      const int e = (j < 4 ? at0 : at1) + (j & 3);
      v[j] = a.w_bf16 ? __bfloat162float(((const __nv_bfloat16*)w)[e]) : ((const float*)w)[e];
    }
    weight[i >= L][0][lane] = make_float4(v[0], v[1], v[2], v[3]);
    weight[i >= L][1][lane] = make_float4(v[4], v[5], v[6], v[7]);
  }
  __syncthreads();
  for (uint32_t place = 0; t < a.tokens; t += step) {
    const Place later = place_of(t + (DEPTH + 1) * step);
    if (VEC) asm volatile("cp.async.wait_group %0;" ::"n"(DEPTH - 1) : "memory");
    compute(place, t, p[0]);
    if (VEC) fetch(place, t + DEPTH * step, p[DEPTH]);
    advance();
    place = place == (DEPTH - 1) * place_bytes ? 0 : place + place_bytes;
#pragma unroll
    for (int i = 0; i < DEPTH; ++i) p[i] = p[i + 1];
    p[DEPTH] = later;
  }
  if (VEC) asm volatile("cp.async.wait_group 0;" ::: "memory");
}

template <class TI, class TO, bool INTER> auto aligned_kernel(int lanes) {
  return lanes == 8 ? dvm_rotary_kernel<TI, TO, 8, true, INTER> : lanes == 16 ? dvm_rotary_kernel<TI, TO, 16, true, INTER> : dvm_rotary_kernel<TI, TO, 32, true, INTER>;
}

template <class TI, class TO>
int launch(const Args& a, int grid, int threads, int device, cudaStream_t stream) {
  const int bytes = threads * BYTES<TI>;
  if (!a.vec) return dvm_launch_early(dvm_rotary_kernel<TI, TO, 0, false, false>, grid, threads, 0, stream, a);
  auto kernel = a.interleaved ? aligned_kernel<TI, TO, true>(a.lanes) : aligned_kernel<TI, TO, false>(a.lanes);
  static std::atomic<uint64_t> allowed[2][3];
  const int st = dvm_allow_smem((const void*)kernel, THREADS * BYTES<TI>, device, &allowed[a.interleaved][a.lanes / 16]);
  if (st != DVM_OK) return st;
  return dvm_launch_early(kernel, grid, threads, bytes, stream, a);
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
  a.vec = aligned(a.q, a.qs, 2, ei) && aligned(a.k, a.ks, 2, ei) && aligned(a.q_out, a.qo, 2, eo) && aligned(a.k_out, a.ko, d.paged ? 3 : 2, eo) &&
          ((uintptr_t)a.angles & 15) == 0 && (!d.paged || (aligned(a.v, a.vs, 2, ei) && aligned(a.v_out, a.vo, 3, eo)));
  a.tokens = (int)d.tokens; a.hq = (int)d.q_heads; a.hk = (int)d.kv_heads; a.D = (int)d.head_dim; a.rot = (int)d.rotary_dim;
  a.angle_rows = (int)d.angle_rows; a.n_slots = d.paged ? (int)(d.pages * d.page_size) : 0; a.page = d.paged ? (int)d.page_size : 1;
  a.norm = d.norm; a.interleaved = d.interleaved; a.paged = d.paged; a.w_bf16 = d.weight_dtype == DVM_BF16; a.eps = d.eps;
  a.lanes = d.head_dim <= 64 ? 8 : d.head_dim <= 128 ? 16 : 32;
  a.inv_D = 1.f / (float)d.head_dim;
  a.page_log = -1;
  for (int i = 0; i < 31; ++i) if (a.page == 1 << i) a.page_log = i;
  // A CTA takes as many heads of a token as its groups have places for, with no more threads than that takes; of few tokens,
  // fewer heads, until every SM has some.
  const int heads = a.hq + a.hk * (d.paged ? 2 : 1);
  int threads = 32;
  while (threads < THREADS && threads / a.lanes * UNROLL < heads) threads *= 2;
  const int groups = threads / a.lanes, least = (heads + groups * UNROLL - 1) / (groups * UNROLL), most = (heads + groups - 1) / groups;
  const int64_t resident = 3 * (THREADS / threads) * (int64_t)dev.sm_count, want = resident / d.tokens;
  a.chunks = (int)(want < least ? least : want < most ? want : most);
  const int64_t cap = resident / a.chunks < 1 ? 1 : resident / a.chunks;  // tokens at a time
  const int grid = (int)(d.tokens < cap ? d.tokens : cap) * a.chunks;
  if (d.dtype == DVM_BF16) return d.out_dtype == DVM_BF16 ? launch<__nv_bfloat16, __nv_bfloat16>(a, grid, threads, dev.device, stream) : launch<__nv_bfloat16, float>(a, grid, threads, dev.device, stream);
  return d.out_dtype == DVM_BF16 ? launch<float, __nv_bfloat16>(a, grid, threads, dev.device, stream) : launch<float, float>(a, grid, threads, dev.device, stream);
}

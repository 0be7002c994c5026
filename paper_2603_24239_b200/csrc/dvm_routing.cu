// Routing meta-kernel: scores of a token's experts, the best ones in exact order, their weights, and the plan: the tokens'
// rows, expert by expert.
//
// A warp takes a token, lane l its experts l, l + 32, ...  The chosen ones are found one by one: the largest key of the warp,
// keys being the values c as unsigned integers of the same order, and of equal ones the lowest index (two warp reductions
// a round).  Without a bias the order of c is the order of the logits, which need no rounding; with one, or for groups, c is
// rounded, so where two neighbours in the order (or the last group that stays and the first that does not) are nearer
// than the roundings could move them, the token is done again in 64 bits: some tokens in ten thousand.
//
// The plan is a counting sort without atomics whose order could change it.  Tokens go in rounds of 32, and a round's choices
// are a bit per token in a word per expert: a token's rank at its expert is the number of bits below its own, plus what
// earlier rounds of the chunk counted.  With up to 64 tokens one CTA does it all; else every CTA leaves its chunk's counts in
// the workspace and a second launch adds up those of the chunks before it.
#include <cuda_bf16.h>
#include <cuda_runtime.h>
#include <math.h>

#include "dvm_experts_launch.h"

namespace dvm {
namespace routing {

constexpr int WARPS = 16, THREADS = WARPS * 32, ROUND = DVM_ROUTE_ROUND, PER_WARP = ROUND / WARPS;
constexpr uint32_t ALL = 0xffffffffu;

struct Args {
  const void* logits;
  const float* bias;
  const int* positions;
  int *ids, *places, *starts;
  float* weights;
  uint32_t* counts;    // [chunks][experts / 2]: 16 bits each
  long long stride;
  int tokens, experts, top_k, groups, top_groups, chunks, rounds;
  int bf16, sigmoid, renormalise;
  float factor;
};

// Keys: 0 for what cannot be chosen, 1 for NaN, then the order of the values.
__device__ __forceinline__ uint32_t key_of(float x) {
  const uint32_t b = __float_as_uint(x + 0.f);   // (-0 is 0)
  return x != x ? 1u : b ^ ((uint32_t)((int)b >> 31) | 0x80000000u);
}
__device__ __forceinline__ float of_key(uint32_t k) { return __uint_as_float(k & 0x80000000u ? k ^ 0x80000000u : ~k); }
__device__ __forceinline__ float logit_at(const Args& a, long long t, int e) {
  return a.bf16 ? __bfloat162float(((const __nv_bfloat16*)a.logits)[t * a.stride + e]) : ((const float*)a.logits)[t * a.stride + e];
}
__device__ __forceinline__ float warp_max(float v) {
#pragma unroll
  for (int d = 16; d > 0; d >>= 1) v = fmaxf(v, __shfl_xor_sync(ALL, v, d));
  return v;
}
template <class T> __device__ __forceinline__ T warp_sum(T v) {
#pragma unroll
  for (int d = 16; d > 0; d >>= 1) v += __shfl_xor_sync(ALL, v, d);
  return v;
}

// How near two values c are when 32 bits may have swapped them: twice what each may be off, in units of 2^-24.  A sigmoid: one
// ulp of the exponential, a sum, a quotient: less than 6.  Of a softmax every score is at most 1 / sum; the exponential and its
// argument, up to 16 + 5 additions and the quotient are less than 28 of that.  The bias adds a rounding of c itself.
__device__ __forceinline__ float doubt(float unit, float c) { return 0x1p-23f * (unit + 2.f * fabsf(c)); }

// The token again in 64 bits; returns lane j's choice.
template <int V> __device__ __noinline__ int choose_exactly(const Args& a, long long t) {
  const int lane = threadIdx.x & 31, per = a.experts / a.groups;
  double v[V], sum = 0.0, top = -INFINITY;
  bool nan = false;
#pragma unroll
  for (int i = 0; i < V; ++i) {
    const int e = 32 * i + lane;
    v[i] = e < a.experts ? (double)logit_at(a, t, e) : -INFINITY;
    if (v[i] > top) top = v[i];
    nan |= v[i] != v[i];
  }
  if (!a.sigmoid) {
#pragma unroll
    for (int d = 16; d > 0; d >>= 1) top = fmax(top, __shfl_xor_sync(ALL, top, d));
    if (__any_sync(ALL, nan)) top = NAN;
  }
#pragma unroll
  for (int i = 0; i < V; ++i) {
    v[i] = a.sigmoid ? 1.0 / (1.0 + exp(-v[i])) : exp(v[i] - top);
    if (32 * i + lane < a.experts) sum += v[i];
  }
  if (!a.sigmoid) sum = warp_sum(sum);
#pragma unroll
  for (int i = 0; i < V; ++i) {
    const int e = 32 * i + lane;
    if (!a.sigmoid) v[i] /= sum;
    if (a.bias && e < a.experts) v[i] += (double)a.bias[e];
  }
  uint32_t stay = ALL;
  if (a.groups > 1) {
    double first = -INFINITY, second = -INFINITY;
    nan = false;
#pragma unroll
    for (int i = 0; i < V; ++i)
      for (int k = 0; k < 32; ++k) {
        const double x = __shfl_sync(ALL, v[i], k);
        const int e = 32 * i + k;
        if (e >= a.experts || e / per != lane) continue;
        nan |= x != x;
        if (x > first) { second = first; first = x; } else if (x > second) second = x;
      }
    const double mine = nan ? -INFINITY : per > 1 ? first + second : first;
    int before = 0;
    for (int g = 0; g < a.groups; ++g) {
      const double other = __shfl_sync(ALL, mine, g);
      const bool other_nan = __shfl_sync(ALL, (int)nan, g);
      const bool more = nan != other_nan ? nan : other > mine || (other == mine && g < lane);
      if (g != lane && (more || (nan && other_nan && g < lane))) ++before;
    }
    stay = __ballot_sync(ALL, lane < a.groups && before < a.top_groups);
  }
  uint32_t free = 0;   // bits of the experts of this lane that may be chosen
#pragma unroll
  for (int i = 0; i < V; ++i) {
    const int e = 32 * i + lane;
    if (e < a.experts && ((stay >> (a.groups > 1 ? e / per : 0)) & 1u)) free |= 1u << i;
  }
  int mine = -1;
  for (int j = 0; j < a.top_k; ++j) {
    int at = 0x7fffffff;     // this lane's best; NaN is worse than anything
    double best = 0.0;
#pragma unroll
    for (int i = 0; i < V; ++i)
      if ((free >> i) & 1u) {
        if (at == 0x7fffffff || v[i] > best || (best != best && v[i] == v[i])) { at = 32 * i + lane; best = v[i]; }
      }
#pragma unroll
    for (int d = 16; d > 0; d >>= 1) {
      const double o = __shfl_xor_sync(ALL, best, d);
      const int oa = __shfl_xor_sync(ALL, at, d);
      const bool tie = o == best || (o != o && best != best);
      const bool better = oa != 0x7fffffff && (at == 0x7fffffff || o > best || (best != best && o == o) || (tie && oa < at));
      if (better) { best = o; at = oa; }
    }
    if ((at & 31) == lane) free &= ~(1u << (at >> 5));
    if (lane == j) mine = at;
  }
  return mine;
}

// Lane j's choice of token t and its weight.  V: experts of a lane at most; c: this warp's row of shared memory.
template <int V> __device__ __forceinline__ int choose(const Args& a, long long t, float* c, float* weight) {
  const int lane = threadIdx.x & 31, per = a.experts / a.groups;
  const float inv_per = 1.f / per;
  float l[V], top = -INFINITY, sum = 0.f;
  bool nan = false;
#pragma unroll
  for (int i = 0; i < V; ++i) {
    const int e = 32 * i + lane;
    l[i] = e < a.experts ? logit_at(a, t, e) : -INFINITY;
    top = fmaxf(top, l[i]);
    nan |= l[i] != l[i];
  }
  uint32_t key[V];
  if (!a.sigmoid) {
    top = warp_max(top);
    if (__any_sync(ALL, nan)) top = NAN;
#pragma unroll
    for (int i = 0; i < V; ++i)
      if (32 * i + lane < a.experts) sum += expf(l[i] - top);
    sum = warp_sum(sum);
  }
  uint32_t stay = ALL;
  bool unsure = false;
  const float unit = a.sigmoid ? 6.f : 28.f / sum;
  if (a.bias || a.groups > 1) {
#pragma unroll
    for (int i = 0; i < V; ++i) {
      const int e = 32 * i + lane;
      float s = a.sigmoid ? 1.f / (1.f + expf(-l[i])) : expf(l[i] - top) / sum;
      if (a.bias && e < a.experts) s += a.bias[e];
      key[i] = e < a.experts ? key_of(a.bias ? s : l[i]) : 0u;
      if (a.groups > 1 && e < a.experts) c[e] = s;
    }
    if (a.groups > 1) {
      __syncwarp();
      float first = -INFINITY, second = -INFINITY;
      bool bad = false;
      if (lane < a.groups)
        for (int k = 0; k < per; ++k) {
          const float x = c[lane * per + k];
          bad |= x != x;
          second = fmaxf(second, fminf(first, x));
          first = fmaxf(first, x);
        }
      const uint32_t mine = lane < a.groups ? (bad ? 1u : key_of(per > 1 ? first + second : first)) : 0u;
      int before = 0;
      for (int g = 0; g < a.groups; ++g) {
        const uint32_t other = __shfl_sync(ALL, mine, g);
        before += other > mine || (other == mine && g < lane);
      }
      const bool in = lane < a.groups && before < a.top_groups;
      stay = __ballot_sync(ALL, in);
      if (a.top_groups < a.groups) {
        const uint32_t least = __reduce_min_sync(ALL, in ? mine : ALL), most = __reduce_max_sync(ALL, lane < a.groups && !in ? mine : 0u);
        if (most > 1u) {
          const float x = of_key(least), y = of_key(most);
          // (a sum of two values: both may be off, and their sum is rounded)
          unsure = x - y <= 2.f * doubt(unit, fmaxf(fabsf(x), fabsf(y)));
        }
      }
      __syncwarp();
    }
  } else {
#pragma unroll
    for (int i = 0; i < V; ++i) key[i] = 32 * i + lane < a.experts ? key_of(l[i]) : 0u;
  }
  if (a.groups > 1) {
#pragma unroll
    for (int i = 0; i < V; ++i)
      if (!((stay >> min((int)((32 * i + lane + 0.5f) * inv_per), 31)) & 1u)) key[i] = 0u;
  }
  // ---- the largest keys, one after another; with a bias one more, to see how near it is ----
  uint32_t mine_key = 0u, extra_key = 0u;
  int mine = -1, extra = 0;
  const int rounds = a.top_k + (a.bias ? 1 : 0);
  for (int j = 0; j < rounds; ++j) {
    uint32_t best = key[0];
    int at = lane;
#pragma unroll
    for (int i = 1; i < V; ++i)
      if (key[i] > best) { best = key[i]; at = 32 * i + lane; }
    const uint32_t most = __reduce_max_sync(ALL, best);
    if (most == 0u) break;   // (no further expert: only where one more than top_k was asked for)
    at = (int)__reduce_min_sync(ALL, best == most ? (uint32_t)at : ALL);
#pragma unroll
    for (int i = 0; i < V; ++i)
      if (at == 32 * i + lane) key[i] = 0u;
    if (j == a.top_k) { extra = at; extra_key = most; }
    else if (lane == j) { mine = at; mine_key = most; }
  }
  float mine_l = mine >= 0 ? logit_at(a, t, mine) : 0.f;
  if (a.bias) {
    const float b = mine >= 0 ? a.bias[mine] : 0.f;
    uint32_t next_key = __shfl_down_sync(ALL, mine_key, 1);
    float next_l = __shfl_down_sync(ALL, mine_l, 1), next_b = __shfl_down_sync(ALL, b, 1);
    if (lane == a.top_k - 1) { next_key = extra_key; next_l = logit_at(a, t, extra); next_b = a.bias[extra]; }
    if (lane < a.top_k && next_key > 1u && mine_key > 1u) {
      const float x = of_key(mine_key), y = of_key(next_key);
      // (the same logit and bias: the index decides, here as in 64 bits)
      if (x - y <= doubt(unit, fmaxf(fabsf(x), fabsf(y))) && !(mine_l == next_l && b == next_b)) unsure = true;
    }
  }
  if (__any_sync(ALL, unsure)) {
    mine = choose_exactly<V>(a, t);
    mine_l = mine >= 0 ? logit_at(a, t, mine) : 0.f;
  }
  float s = a.sigmoid ? 1.f / (1.f + expf(-mine_l)) : expf(mine_l - top) / sum;
  if (a.renormalise) {
    const float total = warp_sum(lane < a.top_k ? s : 0.f);
    s = s / total;
  }
  *weight = s * a.factor;
  return lane < a.top_k ? mine : -1;
}

__device__ __forceinline__ uint32_t warp_scan(uint32_t v) {  // inclusive
  const int lane = threadIdx.x & 31;
#pragma unroll
  for (int d = 1; d < 32; d <<= 1) {
    const uint32_t y = __shfl_up_sync(ALL, v, d);
    if (lane >= d) v += y;
  }
  return v;
}
// starts of the experts from their counts (thread e: expert e), by all threads of the CTA
__device__ __forceinline__ uint32_t block_scan(uint32_t count, uint32_t* warp_sums, uint32_t* total) {  // exclusive
  const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
  const uint32_t upto = warp_scan(count);
  if (lane == 31) warp_sums[warp] = upto;
  __syncthreads();
  uint32_t before = 0, all = 0;
#pragma unroll
  for (int x = 0; x < WARPS; ++x) {
    if (x < warp) before += warp_sums[x];
    all += warp_sums[x];
  }
  *total = all;
  return before + upto - count;
}

template <int V> __global__ void __launch_bounds__(THREADS) dvm_routing_kernel(const __grid_constant__ Args a) {
  __shared__ uint32_t chosen[DVM_MAX_EXPERTS], carry[DVM_MAX_EXPERTS], sums[WARPS];
  __shared__ float rows[WARPS][V * 32];
  const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
  for (int e = threadIdx.x; e < DVM_MAX_EXPERTS; e += THREADS) chosen[e] = carry[e] = 0u;
  grid_ready();
  grid_wait();
  __syncthreads();
  const long long first = (long long)blockIdx.x * a.rounds * ROUND;
  for (int r = 0; r < a.rounds && first + r * ROUND < a.tokens; ++r) {
    int mine[PER_WARP];
#pragma unroll
    for (int x = 0; x < PER_WARP; ++x) {
      const int in_round = x * WARPS + warp;
      const long long t = first + r * ROUND + in_round;
      mine[x] = -1;
      if (t >= a.tokens) continue;
      float weight = 0.f;
      if (!a.positions || a.positions[t] >= 0) mine[x] = choose<V>(a, t, rows[warp], &weight);
      if (mine[x] >= 0) atomicOr(&chosen[mine[x]], 1u << in_round);
      if (lane < a.top_k) {
        a.ids[t * a.top_k + lane] = mine[x];
        a.weights[t * a.top_k + lane] = weight;
      }
    }
    __syncthreads();
#pragma unroll
    for (int x = 0; x < PER_WARP; ++x) {
      const int in_round = x * WARPS + warp;
      const long long t = first + r * ROUND + in_round;
      if (t < a.tokens && lane < a.top_k)
        a.places[t * a.top_k + lane] = mine[x] < 0 ? -1 : (int)(carry[mine[x]] + __popc(chosen[mine[x]] & ((1u << in_round) - 1u)));
    }
    __syncthreads();
    for (int e = threadIdx.x; e < a.experts; e += THREADS) {
      carry[e] += __popc(chosen[e]);
      chosen[e] = 0u;
    }
    __syncthreads();
  }
  if (a.chunks > 1) {
    for (int e = 2 * threadIdx.x; e < a.experts; e += 2 * THREADS)
      a.counts[(long long)blockIdx.x * ((a.experts + 1) / 2) + e / 2] = carry[e] | (carry[e + 1] << 16);   // (an odd last one: carry[experts] is 0)
    return;
  }
  uint32_t total;
  const uint32_t start = block_scan((int)threadIdx.x < a.experts ? carry[threadIdx.x] : 0u, sums, &total);
  if ((int)threadIdx.x < a.experts) a.starts[threadIdx.x] = (int)start;
  if (threadIdx.x == 0) a.starts[a.experts] = (int)total;
  chosen[threadIdx.x] = start;
  __syncthreads();
  for (int i = threadIdx.x; i < a.tokens * a.top_k; i += THREADS) {
    const int e = a.ids[i];
    if (e >= 0) a.places[i] += (int)chosen[e];
  }
}

// The plan of several chunks: thread (s, p) adds up the counts of experts 2 p and 2 p + 1 over every s-th chunk.
__global__ void __launch_bounds__(THREADS) dvm_routing_plan_kernel(const __grid_constant__ Args a) {
  __shared__ uint32_t before[DVM_MAX_EXPERTS], all[DVM_MAX_EXPERTS], sums[WARPS];
  for (int e = threadIdx.x; e < DVM_MAX_EXPERTS; e += THREADS) before[e] = all[e] = 0u;
  grid_ready();
  grid_wait();
  __syncthreads();
  const int pairs = (a.experts + 1) / 2, slices = THREADS / pairs, p = threadIdx.x % pairs, s = threadIdx.x / pairs;
  if (s < slices) {
    uint32_t b0 = 0, b1 = 0, n0 = 0, n1 = 0;
#pragma unroll 8
    for (int c = s; c < a.chunks; c += slices) {
      const uint32_t v = a.counts[(long long)c * pairs + p];
      n0 += v & 0xffffu;
      n1 += v >> 16;
      if (c < (int)blockIdx.x) { b0 += v & 0xffffu; b1 += v >> 16; }
    }
    atomicAdd(&before[2 * p], b0);   // (whole numbers: any order gives the same)
    atomicAdd(&before[2 * p + 1], b1);
    atomicAdd(&all[2 * p], n0);
    atomicAdd(&all[2 * p + 1], n1);
  }
  __syncthreads();
  uint32_t total;
  const uint32_t start = block_scan((int)threadIdx.x < a.experts ? all[threadIdx.x] : 0u, sums, &total);
  if (blockIdx.x == 0) {
    if ((int)threadIdx.x < a.experts) a.starts[threadIdx.x] = (int)start;
    if (threadIdx.x == 0) a.starts[a.experts] = (int)total;
  }
  before[threadIdx.x] += start;
  __syncthreads();
  const long long chunk = (long long)a.rounds * ROUND * a.top_k, first = blockIdx.x * chunk;
  const long long last = min(first + chunk, (long long)a.tokens * a.top_k);
  for (long long i = first + threadIdx.x; i < last; i += THREADS) {
    const int e = a.ids[i];
    if (e >= 0) a.places[i] += (int)before[e];
  }
}
static_assert(THREADS >= DVM_MAX_EXPERTS, "a thread per expert");

}  // namespace routing
}  // namespace dvm

int dvm_launch_routing(const dvm_routing_desc& d, void* const* t, cudaStream_t stream) {
  using namespace dvm::routing;
  const RoutingSlots s = dvm_slots(d);
  Args a = {};
  a.logits = t[s.logits];
  a.bias = s.bias >= 0 ? (const float*)t[s.bias] : nullptr;
  a.positions = s.positions >= 0 ? (const int*)t[s.positions] : nullptr;
  a.ids = (int*)t[s.ids]; a.weights = (float*)t[s.weights]; a.places = (int*)t[s.places]; a.starts = (int*)t[s.starts];
  a.counts = (uint32_t*)t[s.ws];
  a.stride = d.logits_stride;
  a.tokens = (int)d.tokens; a.experts = (int)d.experts; a.top_k = d.top_k; a.groups = d.groups; a.top_groups = d.top_groups;
  a.chunks = (int)dvm_route_chunks(d); a.rounds = (int)dvm_route_rounds(d);
  a.bf16 = d.dtype == DVM_BF16; a.sigmoid = d.scoring == DVM_ROUTE_SIGMOID; a.renormalise = d.renormalise; a.factor = d.factor;
  auto launch = [&](auto kernel) { return dvm_launch_next(kernel, a.chunks, THREADS, 0, stream, a); };
  const int st = d.experts <= 64 ? launch(dvm_routing_kernel<2>) : d.experts <= 128 ? launch(dvm_routing_kernel<4>)
                 : d.experts <= 256 ? launch(dvm_routing_kernel<8>) : launch(dvm_routing_kernel<16>);
  if (st != DVM_OK || a.chunks == 1) return st;
  return dvm_launch_next(dvm_routing_plan_kernel, a.chunks, THREADS, 0, stream, a);
}

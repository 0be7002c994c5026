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
// earlier rounds of the chunk counted.  With up to 32 tokens one CTA does it all; else every CTA leaves its chunk's counts in
// the workspace and a second launch adds up those of the chunks before.
#include <cuda_bf16.h>
#include <cuda_runtime.h>
#include <math.h>

#include "dvm_experts_launch.h"

namespace dvm {
namespace routing {

constexpr int ROUND = DVM_ROUTE_ROUND, WARPS = ROUND, THREADS = WARPS * 32;   // a warp to a token of a round
constexpr int PLAN = 4, PLAN_THREADS = 512;                                    // of the second launch: chunks of a CTA
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
  int lanes;           // of a warp to a group: the largest power of two
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

// How near two values c are when 32 bits may have swapped them: twice what each may be off, in units of 2^-24.  A sigmoid: the
// exponential's error, 2 ulp and 1.2 per unit of its argument, times s (1 - s), a sum and a quotient (2 ulp): less than 10.  Of a
// softmax every score is at most 1 / sum; exponentials (at most 5), up to 16 + 5 additions and the quotient are less than 36
// of that.  The bias adds a rounding of c itself.
__device__ __forceinline__ float doubt(float unit, float c) { return 0x1p-23f * (unit + 2.f * fabsf(c)); }
// Score of a logit: 1 / (1 + exp(-l)), or exp(l - top) / sum.
__device__ __forceinline__ float score(const Args& a, float l, float top, float sum) {
  return a.sigmoid ? __fdividef(1.f, 1.f + __expf(-l)) : __fdividef(__expf(l - top), sum);
}

// The group of every expert of this lane (experts behind the last: group 32, which is none).
template <int V> __device__ __forceinline__ void groups_of(const Args& a, int (&group)[V]) {
  const float inv = (float)a.groups / (float)a.experts;
#pragma unroll
  for (int i = 0; i < V; ++i) {
    const int e = 32 * i + (threadIdx.x & 31);
    group[i] = e < a.experts ? (int)((e + 0.5f) * inv) : 32;   // (exact: e + 1/2 is half an expert away from any border, e < 512)
  }
}
// The two largest of two pairs, larger one first.
template <class T> __device__ __forceinline__ void merge2(T& first, T& second, T of, T os) {
  if (of > first) { second = first > os ? first : os; first = of; }
  else second = second > of ? second : of;
}

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
  int group[V];
  groups_of<V>(a, group);
  if (a.groups > 1) {
    double mine = -INFINITY;   // of group `lane`
    bool mine_nan = false;
    for (int g = 0; g < a.groups; ++g) {
      double first = -INFINITY, second = -INFINITY;
      bool bad = false;
#pragma unroll
      for (int i = 0; i < V; ++i)
        if (group[i] == g) { bad |= v[i] != v[i]; merge2(first, second, v[i], (double)-INFINITY); }
#pragma unroll
      for (int d = 16; d > 0; d >>= 1) {
        const double of = __shfl_xor_sync(ALL, first, d), os = __shfl_xor_sync(ALL, second, d);
        merge2(first, second, of, os);
      }
      bad = __any_sync(ALL, bad);
      if (lane == g) { mine = bad ? -INFINITY : per > 1 ? first + second : first; mine_nan = bad; }
    }
    int before = 0;
    for (int g = 0; g < a.groups; ++g) {
      const double other = __shfl_sync(ALL, mine, g);
      const bool other_nan = __shfl_sync(ALL, (int)mine_nan, g);
      const bool more = mine_nan != other_nan ? mine_nan : other > mine || ((other == mine || mine_nan) && g < lane);
      if (g != lane && more) ++before;
    }
    stay = __ballot_sync(ALL, lane < a.groups && before < a.top_groups);
  }
  uint32_t free = 0;   // bits of the experts of this lane that may be chosen
#pragma unroll
  for (int i = 0; i < V; ++i)
    if (group[i] < 32 && ((stay >> group[i]) & 1u)) free |= 1u << i;
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

// This lane's logits of a token.
template <int V> __device__ __forceinline__ void load_logits(const Args& a, long long t, float (&l)[V]) {
#pragma unroll
  for (int i = 0; i < V; ++i) {
    const int e = 32 * i + (threadIdx.x & 31);
    l[i] = e < a.experts ? logit_at(a, t, e) : -INFINITY;
  }
}

// The first `found` lanes hold the largest values of a token in nearly their order: the j-th in exact order goes to lane j.  (NaN
// keep their places: they are the last.)
template <int V> __device__ __noinline__ int order_exactly(const Args& a, const float (&l)[V], float top, float mine_l, float b, int mine, uint32_t key, int found) {
  const int lane = threadIdx.x & 31;
  double c;
  if (a.sigmoid) {
    c = 1.0 / (1.0 + exp(-(double)mine_l));
  } else {
    double sum = 0.0;
#pragma unroll
    for (int i = 0; i < V; ++i)
      if (32 * i + lane < a.experts) sum += exp((double)l[i] - top);
    c = exp((double)mine_l - top) / warp_sum(sum);
  }
  c += (double)b;
  int before = 0;
  for (int j = 0; j < found; ++j) {
    const double o = __shfl_sync(ALL, c, j);
    const int oi = __shfl_sync(ALL, mine, j);
    const bool o_nan = __shfl_sync(ALL, key, j) <= 1u, nan = key <= 1u;
    before += o_nan || nan ? j < lane : o > c || (o == c && oi < mine);
  }
  int result = -1;
  for (int j = 0; j < found; ++j) {
    const int place = __shfl_sync(ALL, before, j), e = __shfl_sync(ALL, mine, j);
    if (lane == place) result = e;
  }
  return lane < a.top_k ? result : -1;
}

// The largest of a lane's keys and its expert, of equal ones the lowest.
template <int V> __device__ __forceinline__ void largest(const uint32_t (&key)[V], uint32_t* best, int* at) {
  uint32_t k[V];
  int e[V];
#pragma unroll
  for (int i = 0; i < V; ++i) { k[i] = key[i]; e[i] = 32 * i + (threadIdx.x & 31); }
#pragma unroll
  for (int d = 1; d < V; d <<= 1)
#pragma unroll
    for (int i = 0; i < V; i += 2 * d)
      if (k[i + d] > k[i]) { k[i] = k[i + d]; e[i] = e[i + d]; }
  *best = k[0];
  *at = e[0];
}

// Lane j's choice of token t and its weight.  V: experts of a lane at most; l: this lane's logits; bias: all of them, in shared
// memory; row: this warp's row of shared memory.
template <int V> __device__ __forceinline__ int choose(const Args& a, long long t, const float (&l)[V], const float* bias, float* row, float* weight) {
  const int lane = threadIdx.x & 31;
  float top = -INFINITY, sum = 0.f;
  uint32_t key[V];
  if (!a.sigmoid) {
    bool nan = false;
#pragma unroll
    for (int i = 0; i < V; ++i) {
      top = fmaxf(top, l[i]);
      nan |= l[i] != l[i];
    }
    top = warp_max(top);
    if (__any_sync(ALL, nan)) top = NAN;
#pragma unroll
    for (int i = 0; i < V; ++i)
      if (32 * i + lane < a.experts) sum += __expf(l[i] - top);
    sum = warp_sum(sum);
  }
  bool unsure = false;
  const float unit = a.sigmoid ? 10.f : 36.f / sum;
  if (a.bias || a.groups > 1) {
#pragma unroll
    for (int i = 0; i < V; ++i) {
      const int e = 32 * i + lane;
      key[i] = 0u;
      if (e < a.experts) {
        const float c = score(a, l[i], top, sum) + (a.bias ? bias[e] : 0.f);
        key[i] = key_of(a.bias ? c : l[i]);
        if (a.groups > 1) row[e + (e >> 5)] = c;   // (a word left out of every 33: groups of 32 in different banks)
      }
    }
    if (a.groups > 1) {
      // every group by a.lanes lanes, which take its experts in turn and merge what they found
      __syncwarp();
      const int per = a.experts / a.groups, g = lane / a.lanes, sub = lane - g * a.lanes;
      float first = -INFINITY, second = -INFINITY;
      bool bad = false;
      if (g < a.groups)
        for (int k = sub; k < per; k += a.lanes) {
          const int e = g * per + k;
          const float x = row[e + (e >> 5)];
          bad |= x != x;
          second = fmaxf(second, fminf(first, x));
          first = fmaxf(first, x);
        }
      for (int d = a.lanes >> 1; d > 0; d >>= 1) {
        const float of = __shfl_xor_sync(ALL, first, d), os = __shfl_xor_sync(ALL, second, d);
        bad |= __shfl_xor_sync(ALL, (int)bad, d) != 0;
        second = fmaxf(fmaxf(second, os), fminf(first, of));
        first = fmaxf(first, of);
      }
      // (every lane of a group has its key; lanes of no group the lowest)
      const uint32_t mine = g < a.groups ? (bad ? 1u : key_of(per > 1 ? first + second : first)) : 0u;
      int before = 0;
      for (int o = 0; o < a.groups; ++o) {
        const uint32_t other = __shfl_sync(ALL, mine, o * a.lanes);
        before += other > mine || (other == mine && o < g);
      }
      const bool in = g < a.groups && before < a.top_groups;
      const uint32_t stay = __ballot_sync(ALL, in);
      if (a.top_groups < a.groups) {
        const uint32_t least = __reduce_min_sync(ALL, in ? mine : ALL), most = __reduce_max_sync(ALL, in ? 0u : mine);
        if (most > 1u) {
          const float x = of_key(least), y = of_key(most);
          // (a sum of two values: both may be off, and their sum is rounded)
          unsure = x - y <= 2.f * doubt(unit, fmaxf(fabsf(x), fabsf(y)));
        }
      }
      const float inv = (float)a.groups / (float)a.experts;   // (e + 1/2 is half an expert away from any border, e < 512)
#pragma unroll
      for (int i = 0; i < V; ++i)
        if (!((stay >> min((int)((32 * i + lane + 0.5f) * inv) * a.lanes, 31)) & 1u)) key[i] = 0u;
      __syncwarp();   // (the row is the next token's)
    }
  } else {
#pragma unroll
    for (int i = 0; i < V; ++i) key[i] = 32 * i + lane < a.experts ? key_of(l[i]) : 0u;
  }
  // ---- the largest keys, one after another; with a bias also those so near the last one that they may be above it ----
  uint32_t mine_key = 0u, last_key = 0u, best = 0u;
  int mine = -1, at = 0, found = 0;
  largest<V>(key, &best, &at);
  for (;;) {
    const uint32_t most = __reduce_max_sync(ALL, best);
    if (found >= a.top_k) {
      if (!a.bias || most <= 1u || last_key <= 1u || of_key(last_key) - of_key(most) > doubt(unit, fmaxf(fabsf(of_key(last_key)), fabsf(of_key(most))))) break;
      if (found == 32) { unsure = true; break; }
    }
    const int won = (int)__reduce_min_sync(ALL, best == most ? (uint32_t)at : ALL);
    if (lane == found) { mine = won; mine_key = most; }
    if (++found == a.top_k) last_key = most;
    if (lane == (won & 31)) {
#pragma unroll
      for (int i = 0; i < V; ++i)
        if (32 * i + lane == won) key[i] = 0u;
      largest<V>(key, &best, &at);
    }
    __syncwarp();
  }
  float mine_l = mine >= 0 ? logit_at(a, t, mine) : 0.f;
  if (a.bias) {
    const float b = mine >= 0 ? bias[mine] : 0.f;
    const uint32_t next_key = __shfl_down_sync(ALL, mine_key, 1);
    const float next_l = __shfl_down_sync(ALL, mine_l, 1), next_b = __shfl_down_sync(ALL, b, 1);
    bool near = false;
    if (lane < found - 1 && next_key > 1u && mine_key > 1u) {
      const float x = of_key(mine_key), y = of_key(next_key);
      // (the same logit and bias: the index decides, here as in 64 bits)
      near = x - y <= doubt(unit, fmaxf(fabsf(x), fabsf(y))) && !(mine_l == next_l && b == next_b);
    }
    if (__any_sync(ALL, near) && !__any_sync(ALL, unsure)) mine = order_exactly<V>(a, l, top, mine_l, b, mine, mine_key, found);
  }
  if (__any_sync(ALL, unsure)) mine = choose_exactly<V>(a, t);
  mine_l = mine >= 0 ? logit_at(a, t, mine) : 0.f;
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
template <int WARPS> __device__ __forceinline__ uint32_t block_scan(uint32_t count, uint32_t* warp_sums, uint32_t* total) {  // exclusive
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

template <int V> __global__ void __launch_bounds__(THREADS, 1) dvm_routing_kernel(const __grid_constant__ Args a) {
  __shared__ uint32_t chosen[DVM_MAX_EXPERTS], carry[DVM_MAX_EXPERTS], sums[WARPS];
  __shared__ float bias[DVM_MAX_EXPERTS];
  extern __shared__ float rows[];   // V * 33 to a warp, where there are groups
  const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
  for (int e = threadIdx.x; e < DVM_MAX_EXPERTS; e += THREADS) chosen[e] = carry[e] = 0u;
  grid_ready();
  grid_wait();
  if (a.bias)
    for (int e = threadIdx.x; e < a.experts; e += THREADS) bias[e] = a.bias[e];
  __syncthreads();
  const long long first = (long long)blockIdx.x * a.rounds * ROUND;
  for (int r = 0; r < a.rounds && first + r * ROUND < a.tokens; ++r) {
    const long long t = first + r * ROUND + warp;
    int mine = -1;
    if (t < a.tokens) {
      float l[V], weight = 0.f;
      load_logits<V>(a, t, l);
      if (!a.positions || a.positions[t] >= 0) mine = choose<V>(a, t, l, bias, rows + warp * (V * 33), &weight);
      if (mine >= 0) atomicOr(&chosen[mine], 1u << warp);
      if (lane < a.top_k) {
        a.ids[t * a.top_k + lane] = mine;
        a.weights[t * a.top_k + lane] = weight;
      }
    }
    __syncthreads();
    if (t < a.tokens && lane < a.top_k) a.places[t * a.top_k + lane] = mine < 0 ? -1 : (int)(carry[mine] + __popc(chosen[mine] & ((1u << warp) - 1u)));
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
  const uint32_t start = block_scan<WARPS>((int)threadIdx.x < a.experts ? carry[threadIdx.x] : 0u, sums, &total);
  if ((int)threadIdx.x < a.experts) a.starts[threadIdx.x] = (int)start;
  if (threadIdx.x == 0) a.starts[a.experts] = (int)total;
  if (threadIdx.x < DVM_MAX_EXPERTS) chosen[threadIdx.x] = start;
  __syncthreads();
  for (int i = threadIdx.x; i < a.tokens * a.top_k; i += THREADS) {
    const int e = a.ids[i];
    if (e >= 0) a.places[i] += (int)chosen[e];
  }
}

// The plan of several chunks, for PLAN of them: thread (s, p) adds up the counts of experts 2 p and 2 p + 1 over every s-th chunk.
// The CTA's own choices and counts are on their way meanwhile.
__global__ void __launch_bounds__(PLAN_THREADS) dvm_routing_plan_kernel(const __grid_constant__ Args a) {
  constexpr int EACH = 2;   // choices of a thread that are asked for early
  __shared__ uint32_t before[DVM_MAX_EXPERTS], all[DVM_MAX_EXPERTS], own[PLAN][DVM_MAX_EXPERTS], sums[PLAN_THREADS / 32];
  for (int e = threadIdx.x; e < DVM_MAX_EXPERTS; e += PLAN_THREADS) before[e] = all[e] = 0u;
  grid_ready();
  grid_wait();
  __syncthreads();
  const int pairs = (a.experts + 1) / 2, slices = PLAN_THREADS / pairs, p = threadIdx.x % pairs, s = threadIdx.x / pairs, mine = blockIdx.x * PLAN;
  const long long chunk = (long long)a.rounds * ROUND * a.top_k, first = mine * chunk, last = min(first + PLAN * chunk, (long long)a.tokens * a.top_k);
  int id[EACH], place[EACH];
#pragma unroll
  for (int x = 0; x < EACH; ++x) {
    const long long i = first + threadIdx.x + x * PLAN_THREADS;
    id[x] = i < last ? a.ids[i] : -1;
    place[x] = i < last ? a.places[i] : 0;
  }
  uint32_t mine_n[PLAN] = {};
  if (s == 0)
#pragma unroll
    for (int q = 0; q < PLAN; ++q)
      if (mine + q < a.chunks) mine_n[q] = a.counts[(long long)(mine + q) * pairs + p];
  if (s < slices) {
    uint32_t b0 = 0, b1 = 0, n0 = 0, n1 = 0;
#pragma unroll 16
    for (int c = s; c < a.chunks; c += slices) {
      const uint32_t v = a.counts[(long long)c * pairs + p];
      n0 += v & 0xffffu;
      n1 += v >> 16;
      if (c < mine) { b0 += v & 0xffffu; b1 += v >> 16; }
    }
    atomicAdd(&before[2 * p], b0);   // (whole numbers: any order gives the same)
    atomicAdd(&before[2 * p + 1], b1);
    atomicAdd(&all[2 * p], n0);
    atomicAdd(&all[2 * p + 1], n1);
  }
  __syncthreads();
  uint32_t total;
  const uint32_t start = block_scan<PLAN_THREADS / 32>((int)threadIdx.x < a.experts ? all[threadIdx.x] : 0u, sums, &total);
  if (blockIdx.x == 0) {
    if ((int)threadIdx.x < a.experts) a.starts[threadIdx.x] = (int)start;
    if (threadIdx.x == 0) a.starts[a.experts] = (int)total;
  }
  before[threadIdx.x] += start;
  __syncthreads();
  if (s == 0) {
    uint32_t at0 = before[2 * p], at1 = before[2 * p + 1];
#pragma unroll
    for (int q = 0; q < PLAN; ++q) {
      own[q][2 * p] = at0;
      own[q][2 * p + 1] = at1;
      at0 += mine_n[q] & 0xffffu;
      at1 += mine_n[q] >> 16;
    }
  }
  __syncthreads();
#pragma unroll
  for (int x = 0; x < EACH; ++x) {
    const long long i = first + threadIdx.x + x * PLAN_THREADS;
    if (id[x] >= 0) a.places[i] = place[x] + (int)own[(int)((i - first) / chunk)][id[x]];
  }
  for (long long i = first + threadIdx.x + EACH * PLAN_THREADS; i < last; i += PLAN_THREADS) {
    const int e = a.ids[i];
    if (e >= 0) a.places[i] += (int)own[(int)((i - first) / chunk)][e];
  }
}
static_assert(PLAN_THREADS >= DVM_MAX_EXPERTS, "a thread per expert");

template <int V> int launch(const Args& a, int device, cudaStream_t stream) {
  static std::atomic<uint64_t> allowed{0};
  constexpr int BYTES = WARPS * V * 33 * 4;
  const int st = dvm_allow_smem((const void*)dvm_routing_kernel<V>, BYTES, device, &allowed);
  return st != DVM_OK ? st : dvm_launch_next(dvm_routing_kernel<V>, a.chunks, THREADS, a.groups > 1 ? BYTES : 0, stream, a);
}

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
  a.lanes = 32;
  while (a.lanes * a.groups > 32) a.lanes >>= 1;
  DvmDeviceInfo dev;
  int st = dvm_device_state(&dev);
  if (st != DVM_OK) return st;
  st = d.experts <= 64 ? launch<2>(a, dev.device, stream) : d.experts <= 128 ? launch<4>(a, dev.device, stream) : d.experts <= 256 ? launch<8>(a, dev.device, stream)
       : launch<16>(a, dev.device, stream);
  if (st != DVM_OK || a.chunks == 1) return st;
  return dvm_launch_next(dvm_routing_plan_kernel, (a.chunks + PLAN - 1) / PLAN, PLAN_THREADS, 0, stream, a);
}

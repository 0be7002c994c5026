// Routing meta-kernel: scores of a token's experts, the best ones in exact order, their weights, and the plan: the tokens'
// rows, expert by expert.
//
// A warp takes a token, lane l its experts l, l + 32, ...  Keys are the values c as unsigned integers of the same order, with the
// lowest bits given to the place in the lane: each lane sorts its keys (a maximum and a minimum to a trade), then the chosen ones
// are found one by one: the largest head of the warp, of equal ones the lowest index (two warp reductions a round).
// That order is exact but where two neighbours in it -- the last one chosen and those behind it included -- are as near as
// the roundings of c and the bits left out could move them; those are put in order in 64 bits (without a bias by the logits, whose
// order is that of c): some tokens in a thousand.
//
// The plan is a counting sort without atomics whose order could change it.  Tokens go in rounds, a warp to each, and a round's
// choices are a bit per token in a word per expert: a token's rank at its expert is the number of bits below its own, plus what
// earlier rounds of the chunk counted.  Up to 128 tokens are dealt to the 8 CTAs of a cluster, which read one another's counts;
// else every CTA leaves its chunk's counts in the workspace, a byte each, and a second launch adds up those of the chunks before.
// 8191 tokens of 256 experts in 8 groups with a bias: 28 us (19 without both), 64 tokens 6.0 (4.2), one token of 64
// experts 3.8 in a chain of launches (two launches of CTAs of 16 tokens took 9.8 for 64; one CTA of 32 took 6.6 for 32, 5.8 now).  Bound by
// instructions: 2.1 us would read the logits, but a token costs 870 instructions without groups or bias (a load, a score, a sort of
// 8 keys and 8 rounds of two reductions) and 1530 with both, 13 and 20 us of the first launch.  A warp per token was taken over a
// CTA per token (whose barriers made 8191 tokens 96 us) and over a thread per token (64 tokens leave the GPU empty).  One token in
// a CTA that goes to 64 bits keeps the others waiting: with all of it done again there, groups included, 8191 tokens took 29 to 36
// us by what they held, now 27 to 31 (25.7 if none did).  Sorting by merges of odd and even places (38 instructions for 56) made
// no difference for 8 keys and lost registers for 16.  The second launch, 8 us, reads every chunk's counts per 4 chunks; 16 bytes
// to a load and additions of two counts to an instruction took it there from 20.
#include <cuda_bf16.h>
#include <cuda_runtime.h>
#include <math.h>

#include "dvm_experts_launch.h"

namespace dvm {
namespace routing {

constexpr int PLAN = 4, PLAN_THREADS = 512;   // of the second launch: chunks of a CTA
constexpr int JOINT = 8, JOINT_WARPS = DVM_ROUTE_ONE / JOINT;   // of the one launch for few tokens: CTAs of a cluster, warps of each
constexpr uint32_t ALL = 0xffffffffu;

struct Args {
  const void* logits;
  const float* bias;
  const int* positions;
  int *ids, *places, *starts;
  float* weights;
  uint32_t* counts;    // [chunks][experts, rounded up to 16]: 8 bits each
  long long stride;
  int tokens, experts, top_k, groups, top_groups, chunks, rounds;
  int bf16, sigmoid, renormalise;
  int lanes;           // of a warp to a group: the largest power of two
  int quads, quads_up; // of the second launch
  float factor;
};

// Keys: 0 for what cannot be chosen, NAN_KEY for NaN, then the order of the values.
constexpr uint32_t NAN_KEY = 16u;
__device__ __forceinline__ uint32_t key_of(float x) {
  const uint32_t b = __float_as_uint(x + 0.f);   // (-0 is 0)
  return x != x ? NAN_KEY : b ^ ((uint32_t)((int)b >> 31) | 0x80000000u);
}
// The same with the place i of V in the lane in its lowest bits, the first place the highest.
template <int V> __device__ __forceinline__ uint32_t key_at(uint32_t key, int i) { return (key & ~(uint32_t)(V - 1)) | (uint32_t)(V - 1 - i); }
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
// exponential's error, 4 (2 ulp) and 1.25 |x| of it (its argument and log2 e are rounded), times s (1 - s): at most 1.05; the sum
// before the reciprocal 1; the reciprocal 2 (1 ulp): less than 4.2.  Of a softmax every score is at most 1 / sum; exponentials (at most
// 5), up to 16 + 5 additions and the quotient are less than 36 of that.  The bias adds a rounding of c itself.
constexpr float SIGMOID_UNIT = 4.2f, SOFTMAX_UNIT = 36.f;
// Of two sums of two values, at most most in magnitudes: four values and both sums' roundings.
__device__ __forceinline__ float doubt_of_sums(float unit, float most) { return 0x1p-23f * 2.f * (unit + most); }
// ... and of two keys without their lowest bits, which are less than V units in the last place (of at most 2^-23 of the value).
// Values by logits are not rounded (unit 0).
template <int V> __device__ __forceinline__ bool near_keys(uint32_t more, uint32_t less, float unit) {
  if (less < 2 * NAN_KEY) return false;   // (NaN, or nothing)
  const float x = of_key(more & ~(uint32_t)(V - 1)), y = of_key(less & ~(uint32_t)(V - 1));
  return x - y <= fmaxf(fabsf(x), fabsf(y)) * ((V + 1) * 0x1p-23f) + 0x1p-23f * unit;   // (infinite minus infinite: not near, the index decides)
}
__device__ __forceinline__ float exp_near(float x) {
  float y;
  asm("ex2.approx.ftz.f32 %0, %1;" : "=f"(y) : "f"(x * 1.4426950408889634f));
  return y;
}
__device__ __forceinline__ float rcp_near(float x) {
  float y;
  asm("rcp.approx.ftz.f32 %0, %1;" : "=f"(y) : "f"(x));
  return y;
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

// c of this lane's experts in 64 bits.
template <int V> __device__ __noinline__ void scores_exactly(const Args& a, long long t, double* v) {
  const int lane = threadIdx.x & 31;
  double sum = 0.0, top = -INFINITY;
  bool nan = false;
#pragma unroll 1
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
#pragma unroll 1
  for (int i = 0; i < V; ++i) {
    v[i] = exp(a.sigmoid ? -v[i] : v[i] - top);
    if (a.sigmoid) v[i] = 1.0 / (1.0 + v[i]);
    if (32 * i + lane < a.experts) sum += v[i];
  }
  if (!a.sigmoid) sum = warp_sum(sum);
#pragma unroll 1
  for (int i = 0; i < V; ++i) {
    const int e = 32 * i + lane;
    if (!a.sigmoid) v[i] /= sum;
    if (a.bias && e < a.experts) v[i] += (double)a.bias[e];
  }
}
// Of the groups `open`, the `places` that count most, by their sums in 64 bits (which are numbers).
template <int V> __device__ __noinline__ uint32_t groups_exactly(const Args& a, long long t, uint32_t open, int places) {
  const int lane = threadIdx.x & 31, per = a.experts / a.groups;
  double v[V], mine = 0.0;   // mine: of group `lane`
  int group[V];
  scores_exactly<V>(a, t, v);
  groups_of<V>(a, group);
  for (uint32_t m = open; m; m &= m - 1u) {
    const int g = __ffs(m) - 1;
    double first = -INFINITY, second = -INFINITY;
#pragma unroll
    for (int i = 0; i < V; ++i)
      if (group[i] == g) merge2(first, second, v[i], (double)-INFINITY);
#pragma unroll
    for (int d = 16; d > 0; d >>= 1) {
      const double of = __shfl_xor_sync(ALL, first, d), os = __shfl_xor_sync(ALL, second, d);
      merge2(first, second, of, os);
    }
    if (lane == g) mine = per > 1 ? first + second : first;
  }
  int before = 0;
  for (uint32_t m = open; m; m &= m - 1u) {
    const int g = __ffs(m) - 1;
    const double other = __shfl_sync(ALL, mine, g);
    before += g != lane && (other > mine || (other == mine && g < lane));
  }
  return __ballot_sync(ALL, ((open >> lane) & 1u) && before < places);
}

// The token again in 64 bits; returns lane j's choice.
template <int V> __device__ __noinline__ int choose_exactly(const Args& a, long long t) {
  const int lane = threadIdx.x & 31, per = a.experts / a.groups;
  double v[V];
  scores_exactly<V>(a, t, v);
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
  if (!a.bias)   // ranked by the logits, which tell apart what scores of 64 bits do not
#pragma unroll
    for (int i = 0; i < V; ++i) v[i] = 32 * i + lane < a.experts ? (double)logit_at(a, t, 32 * i + lane) : -INFINITY;
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
  const int lane = threadIdx.x & 31;
  if (a.bf16) {
    const __nv_bfloat16* p = (const __nv_bfloat16*)a.logits + t * a.stride + lane;
#pragma unroll
    for (int i = 0; i < V; ++i) l[i] = 32 * i + lane < a.experts ? __bfloat162float(p[32 * i]) : -INFINITY;
  } else {
    const float* p = (const float*)a.logits + t * a.stride + lane;
#pragma unroll
    for (int i = 0; i < V; ++i) l[i] = 32 * i + lane < a.experts ? p[32 * i] : -INFINITY;
  }
}

// The first `found` lanes hold the largest values of a token in nearly their order: the j-th in exact order goes to lane j.  (NaN
// keep their places: they are the last.)
template <int V> __device__ __noinline__ int order_exactly(const Args& a, long long t, float top, float mine_l, float b, int mine, uint32_t key, int found) {
  const int lane = threadIdx.x & 31;
  double c = (double)mine_l;
  if (a.bias && a.sigmoid) {
    c = 1.0 / (1.0 + exp(-c)) + (double)b;
  } else if (a.bias) {
    double sum = 0.0;
#pragma unroll 1
    for (int i = lane; i < a.experts; i += 32) sum += exp((double)logit_at(a, t, i) - top);
    c = exp(c - top) / warp_sum(sum) + (double)b;
  }
  int before = 0;
  for (int j = 0; j < found; ++j) {
    const double o = __shfl_sync(ALL, c, j);
    const int oi = __shfl_sync(ALL, mine, j);
    const bool o_nan = __shfl_sync(ALL, key, j) < 2 * NAN_KEY, nan = key < 2 * NAN_KEY;
    before += o_nan || nan ? j < lane : o > c || (o == c && oi < mine);
  }
  int result = -1;
  for (int j = 0; j < found; ++j) {
    const int place = __shfl_sync(ALL, before, j), e = __shfl_sync(ALL, mine, j);
    if (lane == place) result = e;
  }
  return lane < a.top_k ? result : -1;
}

// The chosen scores over their sum, lane j's of logit l, where scores may lie below what fp32 holds: relative to the largest of them
// (m: its logit), which changes no quotient: exp(l - m) of a softmax; exp(-m) / (1 + exp(-l)) of a sigmoid, none of which is above
// 1/2 here.
__device__ __noinline__ float share_of_small(const Args& a, float l) {
  const bool chosen = (threadIdx.x & 31) < a.top_k;
  const float m = of_key(__reduce_max_sync(ALL, chosen ? key_of(l) : 0u));   // (-inf: 0 / 0)
  const float s = a.sigmoid ? expf(l - m) / (1.f + expf(l)) : expf(l - m);
  return s / warp_sum(chosen ? s : 0.f);
}

// A lane's keys in descending order.  Neighbours of every other pair trade places in turn.
template <int V> __device__ __forceinline__ void sort_keys(uint32_t (&key)[V]) {
#pragma unroll
  for (int round = 0; round < V; ++round)
#pragma unroll
    for (int i = round & 1; i + 1 < V; i += 2) {
      const uint32_t more = max(key[i], key[i + 1]);
      key[i + 1] = min(key[i], key[i + 1]);
      key[i] = more;
    }
}

// Lane j's choice of token t and its weight.  V: experts of a lane at most; SCORED: ranked by scores (there is a bias, or groups are
// compared), else by the logits, which have their order; l: this lane's logits; bias: all of them, in shared
// memory; row: this warp's row of shared memory.
template <int V, bool SCORED> __device__ __forceinline__ int choose(const Args& a, long long t, const float (&l)[V], const float* bias, float* row, float* weight) {
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
      if (32 * i + lane < a.experts) sum += exp_near(l[i] - top);
    sum = warp_sum(sum);
  }
  bool unsure = false;
  const float unit = a.sigmoid ? SIGMOID_UNIT : SOFTMAX_UNIT / sum;
  if (SCORED) {
    const float inv_sum = rcp_near(sum);
    float c[V];
    if (a.sigmoid) {
#pragma unroll
      for (int i = 0; i < V; ++i) c[i] = rcp_near(1.f + exp_near(-l[i]));
    } else {
#pragma unroll
      for (int i = 0; i < V; ++i) c[i] = exp_near(l[i] - top) * inv_sum;
    }
    if (a.bias) {
#pragma unroll
      for (int i = 0; i < V; ++i) {
        c[i] += bias[32 * i + lane];   // (of experts behind the last: anything)
        key[i] = 32 * i + lane < a.experts ? key_at<V>(key_of(c[i]), i) : 0u;
      }
    } else {
#pragma unroll
      for (int i = 0; i < V; ++i) key[i] = 32 * i + lane < a.experts ? key_at<V>(key_of(l[i]), i) : 0u;
    }
    if (a.groups > 1)
#pragma unroll
      for (int i = 0; i < V; ++i) row[33 * i + lane] = c[i];   // (a word left out of every 33: groups of 32 in different banks)
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
      const float size = per > 1 ? fabsf(first) + fabsf(second) : fabsf(first);
      // (every lane of a group has its key; lanes of no group the lowest)
      const uint32_t mine = g < a.groups ? (bad ? NAN_KEY : key_of(per > 1 ? first + second : first)) : 0u;
      int before = 0;
      for (int o = 0; o < a.groups; ++o) {
        const uint32_t other = __shfl_sync(ALL, mine, o * a.lanes);
        before += other > mine || (other == mine && o < g);
      }
      bool in = g < a.groups && before < a.top_groups;
      if (a.top_groups < a.groups) {
        const uint32_t least = __reduce_min_sync(ALL, in ? mine : ALL), most = __reduce_max_sync(ALL, in ? 0u : mine);
        const float sizes = __uint_as_float(__reduce_max_sync(ALL, __float_as_uint(g < a.groups && !bad && size < INFINITY ? size : 0.f)));
        const float x = of_key(least), y = of_key(most), far = doubt_of_sums(unit, sizes);
        if (most > NAN_KEY && x - y <= far) {
          // those that may lie on either side of the border
          const float sum = of_key(mine);
          const bool may = g < a.groups && mine > NAN_KEY && sum - y <= far && x - sum <= far;
          uint32_t open = 0u;
          int sure = 0;
          for (int o = 0; o < a.groups; ++o) {
            const bool o_may = __shfl_sync(ALL, (int)may, o * a.lanes) != 0, o_in = __shfl_sync(ALL, (int)in, o * a.lanes) != 0;
            open |= (uint32_t)o_may << o;
            sure += o_in && !o_may;
          }
          open = groups_exactly<V>(a, t, open, a.top_groups - sure);
          if (may) in = (open >> g) & 1u;
        }
      }
      const uint32_t stay = __ballot_sync(ALL, in);
      const float inv = (float)a.groups / (float)a.experts;   // (e + 1/2 is half an expert away from any border, e < 512)
#pragma unroll
      for (int i = 0; i < V; ++i)
        if (!((stay >> min((int)((32 * i + lane + 0.5f) * inv) * a.lanes, 31)) & 1u)) key[i] = 0u;
      __syncwarp();   // (the row is the next token's)
    }
  } else {
#pragma unroll
    for (int i = 0; i < V; ++i) key[i] = 32 * i + lane < a.experts ? key_at<V>(key_of(l[i]), i) : 0u;
  }
  // ---- the largest keys, one after another, and those behind the last one that may be above it ----
  const float rank_unit = SCORED && a.bias ? unit : 0.f;
  uint32_t mine_key = 0u, last_key = 0u;
  int mine = -1, found = 0;
  sort_keys<V>(key);
  for (;;) {
    const uint32_t most = __reduce_max_sync(ALL, key[0]);
    if (found >= a.top_k) {
      if (!near_keys<V>(last_key, most, rank_unit)) break;
      if (found == 32) { unsure = true; break; }
    }
    const uint32_t at = (V - 1 - (key[0] & (V - 1))) * 32u + lane;
    const int won = (int)__reduce_min_sync(ALL, key[0] == most ? at : ALL);
    if (lane == found) { mine = won; mine_key = most; }
    if (++found == a.top_k) last_key = most;
    if (at == (uint32_t)won) {   // (its lane goes on to its next)
#pragma unroll
      for (int i = 0; i + 1 < V; ++i) key[i] = key[i + 1];
      key[V - 1] = 0u;
    }
  }
  float mine_l = mine >= 0 ? logit_at(a, t, mine) : 0.f;
  const float b = SCORED && a.bias && mine >= 0 ? bias[mine] : 0.f;
  const uint32_t next_key = __shfl_down_sync(ALL, mine_key, 1);
  const float next_l = __shfl_down_sync(ALL, mine_l, 1), next_b = __shfl_down_sync(ALL, b, 1);
  // (the same logit and bias: the index decides, here as in 64 bits)
  const bool near = lane < found - 1 && near_keys<V>(mine_key, next_key, rank_unit) && !(mine_l == next_l && b == next_b);
  const bool redo = __any_sync(ALL, unsure);
  if (redo) mine = choose_exactly<V>(a, t);
  else if (__any_sync(ALL, near)) mine = order_exactly<V>(a, t, top, mine_l, b, mine, mine_key, found);
  if (redo || found > a.top_k || __any_sync(ALL, near)) mine_l = mine >= 0 ? logit_at(a, t, mine) : 0.f;
  float s = a.sigmoid ? 1.f / (1.f + expf(-mine_l)) : expf(mine_l - top) / sum;
  if (a.renormalise) {
    const float total = warp_sum(lane < a.top_k ? s : 0.f);
    // (2^-128 is lost of a sigmoid whose logit is below -88, 2^-150 of a softmax: nothing that counts, but in a small total)
    s = total < (a.sigmoid ? 0.25f : 0x1p-23f) ? share_of_small(a, mine_l) : s / total;
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

// A chunk of many tokens; its counts go to the second launch.
template <int V, bool SCORED> __global__ void __launch_bounds__(DVM_ROUTE_ROUND * 32, 2) dvm_routing_kernel(const __grid_constant__ Args a) {
  constexpr int WARPS = DVM_ROUTE_ROUND, THREADS = WARPS * 32;
  __shared__ uint32_t chosen[DVM_MAX_EXPERTS], carry[DVM_MAX_EXPERTS];
  __shared__ float bias[DVM_MAX_EXPERTS];
  extern __shared__ float rows[];   // V * 33 to a warp, where there are groups
  const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
  for (int e = threadIdx.x; e < DVM_MAX_EXPERTS; e += THREADS) chosen[e] = carry[e] = 0u;
  grid_ready();
  grid_wait();
  if (SCORED && a.bias)
    for (int e = threadIdx.x; e < a.experts; e += THREADS) bias[e] = a.bias[e];
  __syncthreads();
  const long long first = (long long)blockIdx.x * a.rounds * WARPS;
  for (int r = 0; r < a.rounds && first + r * WARPS < a.tokens; ++r) {
    const long long t = first + r * WARPS + warp;
    int mine = -1;
    if (t < a.tokens) {
      float l[V], weight = 0.f;
      load_logits<V>(a, t, l);
      if (!a.positions || a.positions[t] >= 0) mine = choose<V, SCORED>(a, t, l, bias, rows + warp * (V * 33), &weight);
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
  const int words = (a.experts + 15) / 16 * 4;   // (the counts of experts behind the last are 0)
  for (int q = threadIdx.x; q < words; q += THREADS)
    a.counts[(long long)blockIdx.x * words + q] = carry[4 * q] | (carry[4 * q + 1] << 8) | (carry[4 * q + 2] << 16) | (carry[4 * q + 3] << 24);
}

// Few tokens, in one launch: the CTAs of a cluster share them, a warp to each, and read one another's counts.
template <int V, bool SCORED> __global__ void __cluster_dims__(JOINT) __launch_bounds__(JOINT_WARPS * 32, 1) dvm_routing_joint_kernel(const __grid_constant__ Args a) {
  constexpr int THREADS = JOINT_WARPS * 32;
  __shared__ uint32_t chosen[DVM_MAX_EXPERTS], counts[DVM_MAX_EXPERTS], sums[JOINT_WARPS];
  __shared__ float bias[DVM_MAX_EXPERTS];
  extern __shared__ float rows[];   // V * 33 to a warp, where there are groups
  const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31, e = threadIdx.x;
  uint32_t rank;
  asm("mov.u32 %0, %%cluster_ctarank;" : "=r"(rank));
  chosen[e] = 0u;
  grid_ready();
  grid_wait();
  if (SCORED && a.bias && e < a.experts) bias[e] = a.bias[e];
  __syncthreads();
  const int per = (a.tokens + JOINT - 1) / JOINT, t = (int)rank * per + warp;
  const bool here = warp < per && t < a.tokens;
  int mine = -1;
  if (here) {
    float l[V], weight = 0.f;
    load_logits<V>(a, t, l);
    if (!a.positions || a.positions[t] >= 0) mine = choose<V, SCORED>(a, t, l, bias, rows + warp * (V * 33), &weight);
    if (mine >= 0) atomicOr(&chosen[mine], 1u << warp);
    if (lane < a.top_k) {
      a.ids[t * a.top_k + lane] = mine;
      a.weights[t * a.top_k + lane] = weight;
    }
  }
  __syncthreads();
  const uint32_t place = mine >= 0 ? __popc(chosen[mine] & ((1u << warp) - 1u)) : 0u;
  counts[e] = __popc(chosen[e]);
  asm volatile("barrier.cluster.arrive.release.aligned;\n\tbarrier.cluster.wait.acquire.aligned;" ::: "memory");
  uint32_t of_all = 0u, before = 0u;
  const uint32_t at = (uint32_t)__cvta_generic_to_shared(&counts[e]);
#pragma unroll
  for (uint32_t c = 0; c < JOINT; ++c) {
    uint32_t there, n;
    asm("mapa.shared::cluster.u32 %0, %1, %2;" : "=r"(there) : "r"(at), "r"(c));
    asm volatile("ld.shared::cluster.u32 %0, [%1];" : "=r"(n) : "r"(there) : "memory");
    of_all += n;
    before += c < rank ? n : 0u;
  }
  asm volatile("barrier.cluster.arrive.release.aligned;" ::: "memory");   // (no CTA goes before its counts have been read)
  uint32_t total;
  const uint32_t start = block_scan<JOINT_WARPS>(e < a.experts ? of_all : 0u, sums, &total);
  if (rank == 0) {
    if (e < a.experts) a.starts[e] = (int)start;
    if (e == 0) a.starts[a.experts] = (int)total;
  }
  chosen[e] = start + before;
  __syncthreads();
  if (here && lane < a.top_k) a.places[t * a.top_k + lane] = mine < 0 ? -1 : (int)(chosen[mine] + place);
  asm volatile("barrier.cluster.wait.acquire.aligned;" ::: "memory");
}
static_assert(JOINT_WARPS * 32 == DVM_MAX_EXPERTS, "a thread per expert");

// The plan of several chunks, for PLAN of them: thread (s, q) adds up the counts of experts 16 q ... 16 q + 15 (16 bytes) over
// every s-th chunk, two to a word; the threads of a warp that share q add theirs up by exchange, the warps by atomics in shared
// memory.  The CTA's own choices and counts are on their way meanwhile.
__global__ void __launch_bounds__(PLAN_THREADS) dvm_routing_plan_kernel(const __grid_constant__ Args a) {
  constexpr int EACH = 2, DEEP = 16;   // choices of a thread that are asked for early; chunks asked for together
  __shared__ uint32_t before[DVM_MAX_EXPERTS], all[DVM_MAX_EXPERTS], own[PLAN][DVM_MAX_EXPERTS], sums[PLAN_THREADS / 32];
  for (int e = threadIdx.x; e < DVM_MAX_EXPERTS; e += PLAN_THREADS) before[e] = all[e] = 0u;
  grid_ready();
  grid_wait();
  __syncthreads();
  // a.quads: 16s of experts, a.quads_up: the same rounded up to a power of two, 2 at least
  const int quads = a.quads, slices = PLAN_THREADS / a.quads_up, q = threadIdx.x & (a.quads_up - 1), s = threadIdx.x / a.quads_up, mine = blockIdx.x * PLAN;
  const int chunk = a.rounds * DVM_ROUTE_ROUND * a.top_k;
  const long long first = (long long)mine * chunk;
  const int choices = (int)min((long long)PLAN * chunk, (long long)a.tokens * a.top_k - first);
  const int* const ids = a.ids + first;
  int* const places = a.places + first;
  int id[EACH], place[EACH];
#pragma unroll
  for (int x = 0; x < EACH; ++x) {
    const int i = threadIdx.x + x * PLAN_THREADS;
    id[x] = i < choices ? ids[i] : -1;
    place[x] = i < choices ? places[i] : 0;
  }
  // thread e: the counts of expert e in the CTA's own chunks
  uint32_t mine_n[PLAN] = {};
  if ((int)threadIdx.x < a.experts)
#pragma unroll
    for (int x = 0; x < PLAN; ++x)
      if (mine + x < a.chunks) mine_n[x] = ((const uint8_t*)a.counts)[(long long)(mine + x) * (quads * 16) + threadIdx.x];
  const uint4* const counts = (const uint4*)a.counts + q;
  const int leader = (int)(threadIdx.x & ~31u) / a.quads_up;   // the first of the slices of this warp
  const int many = slices * DEEP * (a.quads_up / 2);   // 32 / quads_up lanes x DEEP x quads_up / 2 chunks x 255 < 2^16
  for (int c1 = s; c1 - s + leader < a.chunks; c1 += many) {   // (the lanes of a warp alike)
    uint32_t n[8] = {}, b[8] = {};   // word w of the 16 bytes: bytes 0 and 2 in [2 w], 1 and 3 in [2 w + 1]
    for (int c0 = c1; c0 - c1 < many && c0 - s + leader < a.chunks; c0 += slices * DEEP) {
      uint4 v[DEEP];
#pragma unroll
      for (int x = 0; x < DEEP; ++x) v[x] = q < quads && c0 + x * slices < a.chunks ? counts[(long long)(c0 + x * slices) * quads] : make_uint4(0u, 0u, 0u, 0u);
#pragma unroll
      for (int x = 0; x < DEEP; ++x) {
        const uint32_t w[4] = {v[x].x, v[x].y, v[x].z, v[x].w}, earlier = c0 + x * slices < mine ? 0x00ff00ffu : 0u;
#pragma unroll
        for (int k = 0; k < 4; ++k) {
          n[2 * k] += w[k] & 0x00ff00ffu;
          n[2 * k + 1] += (w[k] >> 8) & 0x00ff00ffu;
          b[2 * k] += w[k] & earlier;
          b[2 * k + 1] += (w[k] >> 8) & earlier;
        }
      }
    }
    for (int d = a.quads_up; d < 32; d <<= 1) {
#pragma unroll
      for (int k = 0; k < 8; ++k) {
        n[k] += __shfl_xor_sync(ALL, n[k], d);
        b[k] += __shfl_xor_sync(ALL, b[k], d);
      }
    }
    const int sharers = 32 / a.quads_up, turn = (threadIdx.x & 31) / a.quads_up;   // lanes of this warp with this q, and which of them this is
#pragma unroll
    for (int k = 0; k < 16; ++k) {
      const int shift = k & 2 ? 16 : 0, from = k / 4 * 2 + (k & 1);
      if ((k & (sharers - 1)) == turn && q < quads) {   // (whole numbers: any order gives the same)
        atomicAdd(&all[k * 32 + q], (n[from] >> shift) & 0xffffu);
        atomicAdd(&before[k * 32 + q], (b[from] >> shift) & 0xffffu);
      }
    }
  }
  __syncthreads();
  uint32_t total;
  const int slot = (threadIdx.x & 15) * 32 + (threadIdx.x >> 4);   // of expert threadIdx.x
  const uint32_t start = block_scan<PLAN_THREADS / 32>((int)threadIdx.x < a.experts ? all[slot] : 0u, sums, &total);
  if (blockIdx.x == 0) {
    if ((int)threadIdx.x < a.experts) a.starts[threadIdx.x] = (int)start;
    if (threadIdx.x == 0) a.starts[a.experts] = (int)total;
  }
  uint32_t at = before[slot] + start;
#pragma unroll
  for (int x = 0; x < PLAN; ++x) {
    own[x][threadIdx.x] = at;
    at += mine_n[x];
  }
  __syncthreads();
  auto chunk_of = [&](int i) {
    int x = 0;
#pragma unroll
    for (int k = 1; k < PLAN; ++k) x += i >= k * chunk;
    return x;
  };
#pragma unroll
  for (int x = 0; x < EACH; ++x) {
    const int i = threadIdx.x + x * PLAN_THREADS;
    if (id[x] >= 0) places[i] = place[x] + (int)own[chunk_of(i)][id[x]];
  }
  for (int i = threadIdx.x + EACH * PLAN_THREADS; i < choices; i += PLAN_THREADS) {
    const int e = ids[i];
    if (e >= 0) places[i] += (int)own[chunk_of(i)][e];
  }
}
static_assert(PLAN_THREADS == DVM_MAX_EXPERTS, "a thread per expert");

template <int V, bool SCORED> int launch(const Args& a, int device, cudaStream_t stream) {
  static std::atomic<uint64_t> allowed{0}, allowed_joint{0};
  const bool few = a.tokens <= DVM_ROUTE_ONE;
  const int bytes = (few ? JOINT_WARPS : DVM_ROUTE_ROUND) * V * 33 * 4, smem = a.groups > 1 ? bytes : 0;
  if (few) {
    const int st = dvm_allow_smem((const void*)dvm_routing_joint_kernel<V, SCORED>, bytes, device, &allowed_joint);
    return st != DVM_OK ? st : dvm_launch_next(dvm_routing_joint_kernel<V, SCORED>, JOINT, JOINT_WARPS * 32, smem, stream, a);
  }
  const int st = dvm_allow_smem((const void*)dvm_routing_kernel<V, SCORED>, bytes, device, &allowed);
  return st != DVM_OK ? st : dvm_launch_next(dvm_routing_kernel<V, SCORED>, a.chunks, DVM_ROUTE_ROUND * 32, smem, stream, a);
}
template <int V> int launch(const Args& a, int device, cudaStream_t stream) {
  return a.bias || a.groups > 1 ? launch<V, true>(a, device, stream) : launch<V, false>(a, device, stream);
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
  a.quads = (a.experts + 15) / 16;
  a.quads_up = 2;
  while (a.quads_up < a.quads) a.quads_up <<= 1;
  while (a.lanes * a.groups > 32) a.lanes >>= 1;
  DvmDeviceInfo dev;
  int st = dvm_device_state(&dev);
  if (st != DVM_OK) return st;
  st = d.experts <= 64 ? launch<2>(a, dev.device, stream) : d.experts <= 128 ? launch<4>(a, dev.device, stream) : d.experts <= 256 ? launch<8>(a, dev.device, stream)
       : launch<16>(a, dev.device, stream);
  if (st != DVM_OK || a.tokens <= DVM_ROUTE_ONE) return st;
  return dvm_launch_next(dvm_routing_plan_kernel, (a.chunks + PLAN - 1) / PLAN, PLAN_THREADS, 0, stream, a);
}

// Attention of prompts: many query rows per request, on the tensor cores.
//
// A CTA takes two tiles of 128 rows of one kv head: a row is a (token, query head of the group) pair, so heads that share
// keys share the loads, and 2 x floor(128 / group) tokens move through the cache together.  Per tile t of 64 tokens of the
// cache and row tile x:
//   S_x = Q_x K^T        tcgen05.mma, both operands in shared memory, S_x in tensor memory (64 fp32 columns)
//   P_x = 2^(c S_x - m)  128 threads, one row each: running maximum m and sum, no exchange between threads;
//                        P_x goes back to tensor memory as bf16, over the S_x it came from
//   O_x += P_x V         tcgen05.mma with P_x as the tensor-memory operand
// S_x has two places, t and t + 1 in turn: S_x(t + 1) is there before P_x(t) is done, so neither the tensor cores nor the
// threads wait for the other's whole latency.  (Tiles of 128 tokens leave room for one place only -- tensor memory is
// S_0, S_1, O_0, O_1 and full -- and then the threads waited 1850 of 4300 cycles per 128 tokens.)  One thread issues
// a row tile's products, PV_x(t) then QK_x(t + 2), and they complete in that order: QK_x(t + 2) overwrites P_x(t) after its
// use.  (One thread for both row tiles spent 830 of 2030 cycles per 64 tokens in waits that were over when they began.)
// O_x is rescaled by a new maximum only when that has grown by more than 2^8 (weights stay below 2^8, far from any bound
// of bf16 or fp32; the quotient at the end does not depend on the maximum that was used); then the row's thread waits for
// PV_x(t - 1).  Weights are rounded to bf16 for the second product, their sum is not.
//
// CTAs stay (one per SM) and take blocks of rows in turn, so that a block's start -- tensor memory, barriers, lengths,
// tables, queries, the first keys -- and its end hide behind its neighbours: started anew for each block they were 10,000
// cycles beside 2,000 for a tile.  Roles: warps 0-3 and 4-7 the rows of the two tiles, warps 8 and 9 issue their products,
// warp 10 fetches (a block's queries once the last score product of the block before has read its own, then keys and
// values in turn through a ring, page by page), warp 11 finds the blocks and hands them on.
//
// Tokens a row does not see get a score of -inf.  That is not enough for the second product, where 0 x NaN is NaN: in
// tiles with a mask the values that no row of the CTA sees are cleared in shared memory (they may be anything: the end of
// a page, pages given back), and if a value that some rows see and others do not is not finite, the CTA's rows are done
// again without tensor cores (attend_row), exactly.
//
// Bound by the chain that a row goes through at every tile -- scores, their maximum, the warp's vote, weights, their way to
// tensor memory, the products -- with two row tiles to hide each other's.  No unit is full: a tile of 64 tokens takes 2050
// cycles, its products 1240 of them when issued alone, its exponentials 900 at 16 a cycle; profiled on 2 prompts of 2048
// tokens, tensor cores 41 %, the exponentials' unit 36 %, issue 39 % of their peaks.  Calls in a row (bursts of a dozen after
// a pause): one prompt of 8192 tokens, 32 / 8 heads of 128: 553 to 569 us at the power cap (490), 970 to 1120 TFLOP/s; 32 / 32
// heads under a window of 1024: 214 to 222 us (195); 12 ragged prompts on cached ones, 40 / 8 heads of 96: 146 us (140); 8
// prompts of up to 1531 tokens, 16 / 4 heads of 64, window 128: 41 us.  A block's cache is walked by one CTA: few rows on a long
// cache leave most of the device idle (4 rows on 16384 tokens: 270 us).
//
// Every wait is bounded: it gives up when 2 s pass in which the CTA neither fetched a tile nor went on doing rows again (one
// warp, 32 rows, token after token: 134 ms on 8192 tokens, 2.5 s on 153600).  Then the CTA raises its abort flag, all roles
// leave, what is in flight is awaited, tensor memory is released and the status word reports DVM_ERR_DEVICE_TIMEOUT.
#include <cuda_bf16.h>
#include <cuda_runtime.h>

#include "dvm_attention.cuh"
#include "dvm_attention_launch.h"
#include "dvm_sm100.cuh"

namespace dvm {
namespace att {

using namespace sm100;

constexpr int PT = 128;                  // rows of a row tile
constexpr int KT = 64;                   // tokens of a cache tile
// Registers are dealt out by role: 384 threads are launched with 168 each, 64,512 in all; the two warpgroups that hold rows of
// scores go up to ROW_REGS, the third down to OTHER_REGS: 256 x 224 + 128 x 56 = 64,512.
constexpr int PROMPT_THREADS = 384;
constexpr int ROW_REGS = 224, OTHER_REGS = 56;
static_assert(256 * ROW_REGS + 128 * OTHER_REGS <= PROMPT_THREADS * 168, "an increase draws on the registers of the launch");
constexpr uint32_t Q_HALF = PT * 128;    // 64 elements of the rows: 16 KB
constexpr uint32_t KV_HALF = KT * 128;   // 64 elements of the tokens: 8 KB
constexpr int HOLES = 16;                // tiles whose missing pages are remembered: more than the ring is deep
constexpr int POLYNOMIAL_EVERY = 8;      // one pair of weights in so many is formed by ex2_by_polynomial
constexpr float GROWTH = 8.f;            // log2 of how far weights may grow before the sums are rescaled

template <int DP>  // head_dim rounded up to 64 or 128
struct PromptSmem {
  static constexpr uint32_t HALVES = DP / 64;
  static constexpr uint32_t Q_TILE = HALVES * Q_HALF;
  static constexpr uint32_t STAGE = HALVES * KV_HALF;            // keys or values of a tile
  static constexpr uint32_t STAGES = DP == 128 ? 10 : 16;
  static constexpr uint32_t RING = 2 * Q_TILE;                   // behind the queries of both row tiles
  static constexpr uint32_t BARS = RING + STAGES * STAGE;        // see the kernel
  static constexpr uint32_t WORDS = BARS + 16 * STAGES + 192;    // tensor memory address, abort, dirty[2][4], holes[], signs of work
  static constexpr uint32_t WORK = WORDS + 48 + 4 * HOLES;       // two descriptions of blocks, the answer of a cancelled launch
  static constexpr uint32_t BYTES = WORK + 2 * 64 + 16 + 1024;
  static_assert(WORK % 16 == 0, "an answer is 16 bytes, aligned");
  static_assert(STAGES / 2 + 3 <= HOLES, "a tile's holes are kept until its weights are done");
};

// kind::f16, bf16 x bf16 -> fp32, M = 128; A K-major; B K-major (keys) or N-major (values)
constexpr uint32_t IDESC_QK = (1u << 4) | (1u << 7) | (1u << 10) | ((uint32_t)(KT >> 3) << 17) | ((uint32_t)(PT >> 4) << 24);
template <int DP> constexpr uint32_t IDESC_PV = (1u << 4) | (1u << 7) | (1u << 10) | (1u << 16) | ((uint32_t)(DP >> 3) << 17) | ((uint32_t)(PT >> 4) << 24);
// 128-byte swizzle: 8-row groups 1024 bytes apart; for the values the 64-column halves are KV_HALF bytes apart
__device__ __forceinline__ uint32_t desc_lo(uint32_t addr, uint32_t leading) { return ((addr >> 4) & 0x3fff) | (leading << 16); }
__device__ __forceinline__ uint64_t desc_of(uint32_t lo) {
  return lo | ((uint64_t)(1024 >> 4) << 32) | ((uint64_t)1 << 46) | ((uint64_t)2 << 61);
}
__device__ __forceinline__ bool elect_one() {
  uint32_t p;
  asm volatile("{\n\t.reg .pred p;\n\telect.sync _|p, 0xffffffff;\n\tselp.u32 %0, 1, 0, p;\n\t}" : "=r"(p));
  return p != 0;
}
// D += A B with A in tensor memory
__device__ __forceinline__ void umma_bf16_ts(uint32_t d_tmem, uint32_t a_tmem, uint64_t bdesc, uint32_t idesc, uint32_t accumulate) {
  asm volatile("{\n\t.reg .pred p;\n\tsetp.ne.b32 p, %4, 0;\n\ttcgen05.mma.cta_group::1.kind::f16 [%0], [%1], %2, %3, p;\n\t}"
               ::"r"(d_tmem), "r"(a_tmem), "l"(bdesc), "r"(idesc), "r"(accumulate)
               : "memory");
}
__device__ __forceinline__ void tmem_load32(uint32_t taddr, float* v) {  // (the caller waits: tmem_load_wait)
  uint32_t* r = (uint32_t*)v;
  asm volatile(
      "tcgen05.ld.sync.aligned.32x32b.x32.b32 "
      "{%0, %1, %2, %3, %4, %5, %6, %7, %8, %9, %10, %11, %12, %13, %14, %15, "
      "%16, %17, %18, %19, %20, %21, %22, %23, %24, %25, %26, %27, %28, %29, %30, %31}, [%32];"
      : "=r"(r[0]), "=r"(r[1]), "=r"(r[2]), "=r"(r[3]), "=r"(r[4]), "=r"(r[5]), "=r"(r[6]), "=r"(r[7]),
        "=r"(r[8]), "=r"(r[9]), "=r"(r[10]), "=r"(r[11]), "=r"(r[12]), "=r"(r[13]), "=r"(r[14]), "=r"(r[15]),
        "=r"(r[16]), "=r"(r[17]), "=r"(r[18]), "=r"(r[19]), "=r"(r[20]), "=r"(r[21]), "=r"(r[22]), "=r"(r[23]),
        "=r"(r[24]), "=r"(r[25]), "=r"(r[26]), "=r"(r[27]), "=r"(r[28]), "=r"(r[29]), "=r"(r[30]), "=r"(r[31])
      : "r"(taddr)
      : "memory");
}
__device__ __forceinline__ void tmem_load_wait() { asm volatile("tcgen05.wait::ld.sync.aligned;" ::: "memory"); }
// ... and what was loaded is used behind the wait only (the wait itself names no registers)
__device__ __forceinline__ void tmem_landed(float* v) {
  tmem_load_wait();
  asm volatile("" : "+f"(v[0]), "+f"(v[1]), "+f"(v[2]), "+f"(v[3]), "+f"(v[4]), "+f"(v[5]), "+f"(v[6]), "+f"(v[7]), 
                    "+f"(v[8]), "+f"(v[9]), "+f"(v[10]), "+f"(v[11]), "+f"(v[12]), "+f"(v[13]), "+f"(v[14]), "+f"(v[15]), 
                    "+f"(v[16]), "+f"(v[17]), "+f"(v[18]), "+f"(v[19]), "+f"(v[20]), "+f"(v[21]), "+f"(v[22]), "+f"(v[23]), 
                    "+f"(v[24]), "+f"(v[25]), "+f"(v[26]), "+f"(v[27]), "+f"(v[28]), "+f"(v[29]), "+f"(v[30]), "+f"(v[31]));
}
__device__ __forceinline__ void tmem_store16(uint32_t taddr, const uint32_t* r) {
  asm volatile(
      "tcgen05.st.sync.aligned.32x32b.x16.b32 [%16], {%0, %1, %2, %3, %4, %5, %6, %7, %8, %9, %10, %11, %12, %13, %14, %15};"
      ::"r"(r[0]), "r"(r[1]), "r"(r[2]), "r"(r[3]), "r"(r[4]), "r"(r[5]), "r"(r[6]), "r"(r[7]),
        "r"(r[8]), "r"(r[9]), "r"(r[10]), "r"(r[11]), "r"(r[12]), "r"(r[13]), "r"(r[14]), "r"(r[15]), "r"(taddr)
      : "memory");
}
__device__ __forceinline__ float ex2(float x) {
  float y;
  asm("ex2.approx.ftz.f32 %0, %1;" : "=f"(y) : "f"(x));
  return y;
}
__device__ __forceinline__ float max_nan(float a, float b) {  // NaN if either is
  float d;
  asm("max.NaN.f32 %0, %1, %2;" : "=f"(d) : "f"(a), "f"(b));
  return d;
}
__device__ __forceinline__ float max_nan(float a, float b, float c) {
  float d;
  asm("max.NaN.f32 %0, %1, %2, %3;" : "=f"(d) : "f"(a), "f"(b), "f"(c));
  return d;
}
// 2^x without the special function unit, for part of the weights: the unit's 16 results a cycle are what the weights take
// longest for, while multiply-adds are to spare.  x = f + r with f the nearest integer (1.5 2^23 added and taken away) and
// |r| <= 1/2; 2^r by the polynomial of degree 5 with constant term 1 of least largest relative error, found by Remez exchange
// (9.15e-8; 1.7e-7 with coefficients and steps in fp32), so that x <= -127 gives exactly 0; f is added to the exponent
// field.  For x below 128.  A NaN gives 0: it comes only from a row's maximum of NaN or +inf, which makes the other weights
// and their sum NaN (see `top` below).
__device__ __forceinline__ float2 ex2_by_polynomial(float2 x) {
  const float2 big = make_float2(12582912.f, 12582912.f);
  x.x = fmaxf(x.x, -127.f);
  x.y = fmaxf(x.y, -127.f);
  const float2 t = add2(x, big);
  const float2 r = fma2(add2(t, make_float2(-12582912.f, -12582912.f)), make_float2(-1.f, -1.f), x);
  float2 p = make_float2(0.001326472731307149f, 0.001326472731307149f);
  p = fma2(p, r, make_float2(0.009671512991189957f, 0.009671512991189957f));
  p = fma2(p, r, make_float2(0.05550733581185341f, 0.05550733581185341f));
  p = fma2(p, r, make_float2(0.24022242426872253f, 0.24022242426872253f));
  p = fma2(p, r, make_float2(0.6931470036506653f, 0.6931470036506653f));
  p = fma2(p, r, make_float2(1.f, 1.f));
  return make_float2(__int_as_float(__float_as_int(p.x) + (__float_as_int(t.x) << 23)), __int_as_float(__float_as_int(p.y) + (__float_as_int(t.y) << 23)));
}
__device__ __forceinline__ uint32_t pack_bf16(float lo, float hi) {
  const __nv_bfloat162 h = __floats2bfloat162_rn(lo, hi);
  return *(const uint32_t*)&h;
}
// bits 0 .. n - 1
__device__ __forceinline__ uint32_t bits_below(int n) { return n <= 0 ? 0u : n >= 32 ? 0xffffffffu : (1u << n) - 1u; }

template <int DP>
__global__ void __launch_bounds__(PROMPT_THREADS, 1)
dvm_attention_prompt_kernel(const __grid_constant__ CUtensorMap tm_q, const __grid_constant__ CUtensorMap tm_k, const __grid_constant__ CUtensorMap tm_v,
                            const __grid_constant__ Args a) {
  using S = PromptSmem<DP>;
  extern __shared__ uint8_t smem_raw[];
  const uint32_t raw = smem_u32(smem_raw), base = (raw + 1023u) & ~1023u;
  uint8_t* const sm = smem_raw + (base - raw);
  const int warp = __shfl_sync(0xffffffffu, (int)(threadIdx.x >> 5), 0), lane = threadIdx.x & 31;  // (the warp's number: known to be uniform)
  // full[], empty[]: the ring; q, qe: queries there, queries read; s, p, o of row tile x and place b at 16 x + 8 b: scores,
  // weights, sums done; w, we: block descriptions; drain; c: an answer
  const uint32_t bar_full = base + S::BARS, bar_empty = bar_full + 8 * S::STAGES, bar_q = bar_empty + 8 * S::STAGES, bar_qe = bar_q + 8, bar_s = bar_q + 16,
                 bar_p = bar_s + 32, bar_o = bar_p + 32, bar_w = bar_o + 32, bar_we = bar_w + 16, bar_drain = bar_we + 16, bar_c = bar_drain + 16;
  volatile uint32_t* const words = (volatile uint32_t*)(sm + S::WORDS);
  volatile uint32_t* const abort_flag = words + 1;
  volatile uint32_t* const dirty = words + 2;  // [x][block mod 4]
  volatile uint32_t* const holes = words + 10;
  volatile uint32_t* const signs = words + 10 + HOLES;  // of work: tiles fetched, tokens that rows were done again with
  volatile int* const work = (volatile int*)(sm + S::WORK);
  const int tokens = PT / a.group;  // of a row tile
  const long long held = (long long)a.max_blocks << a.page_log;

  if (threadIdx.x == 0) {
    for (uint32_t s = 0; s < S::STAGES; ++s) {
      mbar_init(bar_full + 8 * s, 1);
      mbar_init(bar_empty + 8 * s, 2);  // (both row tiles are done with it)
    }
    mbar_init(bar_q, 1);
    mbar_init(bar_qe, 2);
    for (uint32_t x = 0; x < 2; ++x) {
      for (uint32_t b = 0; b < 2; ++b) {
        mbar_init(bar_s + 16 * x + 8 * b, 1);
        mbar_init(bar_p + 16 * x + 8 * b, 4);  // (one arrival per warp)
        mbar_init(bar_o + 16 * x + 8 * b, 1);
      }
      mbar_init(bar_w + 8 * x, 1);
      mbar_init(bar_we + 8 * x, 11);           // (every warp but the one that finds blocks)
      mbar_init(bar_drain + 8 * x, 1);
    }
    mbar_init(bar_c, 1);
    for (int i = 0; i < 8; ++i) dirty[i] = 0;
    *abort_flag = signs[0] = signs[1] = 0;
    asm volatile("fence.mbarrier_init.release.cluster;" ::: "memory");
  }
  if (warp == 9 && lane < 3) tma_prefetch(lane == 0 ? &tm_q : lane == 1 ? &tm_k : &tm_v);
  // Tensor memory too is asked for behind the wait only: the kernel before may still be about to ask for its own on this SM (one
  // that lets dependents start first), and would wait for what this CTA holds while this CTA waits for it.
  grid_wait();
  if (warp == 8) {
    asm volatile("tcgen05.alloc.cta_group::1.sync.aligned.shared::cta.b32 [%0], %1;" ::"r"(smem_u32((const void*)words)), "r"(512u) : "memory");
    asm volatile("tcgen05.relinquish_alloc_permit.cta_group::1.sync.aligned;" ::: "memory");
  }
  tc_fence_before();
  __syncthreads();
  tc_fence_after();
  const uint32_t tmem = words[0], tmem_o = tmem + 4 * KT;  // S_x at place b: 64 (2 x + b)

  // A block: up to 2 x tokens rows of query tokens of one request, for one kv head, described by 16 words of shared memory
  // that stay until every warp has let them go.  Tiles of the cache: [0, ns), then [first, ...); tokens that some row sees:
  // s < end and (s >= low or s < sinks); n0, n1: tiles that the row tiles walk; p_first: position of the first row's token.
  enum { B_REQUEST, B_KVH, B_ROW0, B_TOKENS, B_N0, B_N1, B_NS, B_FIRST, B_END, B_LOW, B_P_LO, B_P_HI };
  // the k-th block of this CTA, or none (also when a wait ran out)
  auto take = [&](int k) -> volatile const int* {
    const bool got = mbar_wait_flat(bar_w + 8 * (k & 1), (k >> 1) & 1, abort_flag, signs);
    volatile const int* const w = work + 16 * (k & 1);
    return __all_sync(0xffffffffu, got) && w[B_TOKENS] > 0 ? w : nullptr;
  };
  auto let_go = [&](int k) {
    __syncwarp();
    if (lane == 0) mbar_arrive(bar_we + 8 * (k & 1));
  };

  uint32_t issued = 0, f_stage = 0, f_phase = 0;  // the fetching warp's ring and queries, and the answers asked for, kept for the abort path
  int q_loads = 0, asked = 0;
  if (warp == 11) {
    asm volatile("setmaxnreg.dec.sync.aligned.u32 %0;" ::"n"(OTHER_REGS));
    // ---------------- blocks: those of all requests in a row, a request's last block first ----------------
    // (Up to 32 requests: the longest first, so that short blocks are left for the end: 12 ragged prompts 143 -> 135 us.  With
    // more of them the end is a small part, and sorting every 32 cost 592 short prompts 37.6 -> 39.7 us.)
    int chunk = -32, before = 0, all = 0, mine = 0, upto = 0, who = 0, sorted = -1;  // 32 requests, the blocks before them, theirs
    auto sum_up = [&](int v) -> int {
#pragma unroll
      for (int d = 1; d < 32; d <<= 1) {
        const int y = __shfl_up_sync(0xffffffffu, v, d);
        if (lane >= d) v += y;
      }
      return v;
    };
    // The grid has a CTA for every block.  One that runs takes its own, then those of CTAs that have not started, in their
    // order, by cancelling their launch: whoever is free takes the next, longest first, without a counter in memory.
    const uint32_t answer = base + S::WORK + 128;
    bool ok = true;
    long long id = blockIdx.x;
    for (int k = 0; ok;) {
      const long long block = id < 0 ? -1 : id / a.hk;
      bool any = id >= 0;
      if (any && block < before) chunk = -32, before = all = 0, sorted = -1;  // (an order that the hardware does not promise)
      while (any && block >= (long long)before + all) {
        before += all;
        chunk += 32;
        any = chunk < a.n;
        const int i = chunk + lane;
        mine = i < a.n ? (min(request_at(a, i).q_len, a.max_q) + 2 * tokens - 1) / (2 * tokens) : 0;
        who = i;
        upto = sum_up(mine);
        all = __shfl_sync(0xffffffffu, upto, 31);
      }
      if (any && a.n > 1 && a.n <= 32 && sorted != chunk) {
        sorted = chunk;
        const int i = chunk + lane, length = i < a.n ? (a.window ? min(a.lengths[i], a.window) : a.lengths[i]) : -1;
        int rank = 0, from = 0;
#pragma unroll
        for (int j = 0; j < 32; ++j) {
          const int other = __shfl_sync(0xffffffffu, length, j);
          rank += other > length || (other == length && j < lane);
        }
#pragma unroll
        for (int j = 0; j < 32; ++j) {
          const uint32_t is = __ballot_sync(0xffffffffu, rank == j);
          if (lane == j) from = __ffs(is) - 1;
        }
        mine = __shfl_sync(0xffffffffu, mine, from);
        who = chunk + from;
        upto = sum_up(mine);
      }
      const int at = (int)(block - before);
      const uint32_t owner = __ballot_sync(0xffffffffu, any && at >= upto - mine && at < upto);
      const int src = owner ? __ffs(owner) - 1 : 0;
      const int tok0 = __shfl_sync(0xffffffffu, upto - 1 - at, src) * 2 * tokens, request = __shfl_sync(0xffffffffu, who, src);
      const bool beyond = !owner && id >= 0;  // (the grid is sized for the most blocks that `rows` rows can make)
      if (!beyond) {
      ok = k < 2 || mbar_wait_flat(bar_we + 8 * (k & 1), ((k >> 1) & 1) ^ 1, abort_flag, signs);
      if (!__all_sync(0xffffffffu, ok)) break;
      if (lane == 0) {
        volatile int* const w = work + 16 * (k & 1);
        w[B_TOKENS] = 0;
        if (owner) {
          const Request rq = request_at(a, request);
          const int n_tok = min(2 * tokens, min(rq.q_len, a.max_q) - tok0);
          const long long p_first = rq.pos0 + tok0;
          const int end = (int)max(0ll, min(p_first + n_tok, held));
          const long long from = a.window ? max(0ll, p_first - a.window + 1) : 0;
          const int low = from <= a.sinks ? 0 : (int)min(from, 0x7fffffffll);
          const int ns = low ? (min(a.sinks, end) + KT - 1) / KT : 0, first = max(low / KT, ns);
          // tiles that row tile x walks: its list ends with its own last position
          auto tiles_of = [&](int x) -> int {
            const int n = min(tokens, n_tok - x * tokens);
            if (n <= 0) return 0;
            const int last = (int)((max(0ll, min(p_first + x * tokens + n, held)) + KT - 1) / KT);
            return last <= ns ? last : ns + max(0, last - first);
          };
          w[B_REQUEST] = request; w[B_KVH] = (int)(id - block * a.hk); w[B_ROW0] = rq.s0 + tok0; w[B_TOKENS] = n_tok;
          w[B_N0] = tiles_of(0); w[B_N1] = tiles_of(1); w[B_NS] = ns; w[B_FIRST] = first; w[B_END] = end; w[B_LOW] = low;
          w[B_P_LO] = (int)(uint32_t)p_first; w[B_P_HI] = (int)(p_first >> 32);
        }
        mbar_arrive(bar_w + 8 * (k & 1));
      }
      __syncwarp();
      if (!owner) break;
      ++k;
      }
      if (lane == 0) {
        mbar_expect_tx(bar_c, 16);
        asm volatile("clusterlaunchcontrol.try_cancel.async.shared::cta.mbarrier::complete_tx::bytes.b128 [%0], [%1];" ::"r"(answer), "r"(bar_c) : "memory");
      }
      __syncwarp();
      ok = __all_sync(0xffffffffu, mbar_wait_flat(bar_c, asked++ & 1, abort_flag, signs));
      uint32_t got = 0, cta = 0;
      asm volatile(
          "{\n\t.reg .pred p;\n\t.reg .b128 r;\n\tld.shared.b128 r, [%2];\n\tclusterlaunchcontrol.query_cancel.is_canceled.pred.b128 p, r;\n\t"
          "selp.u32 %0, 1, 0, p;\n\tmov.u32 %1, 0;\n\t@p clusterlaunchcontrol.query_cancel.get_first_ctaid::x.b32.b128 %1, r;\n\t}"
          : "=r"(got), "=r"(cta)
          : "r"(answer)
          : "memory");
      asm volatile("fence.proxy.async.shared::cta;" ::: "memory");  // (read before the next answer is written)
      __syncwarp();
      id = ok && got ? (long long)cta : -1;  // none left: the end is handed on like a block
    }
  } else if (warp == 10) {
    asm volatile("setmaxnreg.dec.sync.aligned.u32 %0;" ::"n"(OTHER_REGS));
    // ---------------- fetch ----------------
    const int copy_log = min(a.page_log, 6), copies = KT >> copy_log;
    bool ok = true;
    int seen = 0;  // tiles of the blocks before
    for (int k = 0; ok; ++k) {
      volatile const int* const w = take(k);
      if (!w) break;
      const int n_tok = w[B_TOKENS], n_tiles = max(w[B_N0], w[B_N1]), ns = w[B_NS], first = w[B_FIRST], end = w[B_END], low = w[B_LOW], kvh = w[B_KVH], row0 = w[B_ROW0];
      const int* table = a.table + (long long)w[B_REQUEST] * a.max_blocks;
      let_go(k);
      if (n_tiles == 0) continue;
      auto tile_at = [&](int j) -> int { return j < ns ? j : first + (j - ns); };
      auto page_of = [&](int j) -> int {  // of this lane's copy of tile j; -1 where it holds no token that some row sees
        if (lane >= copies || j >= n_tiles) return -1;
        const long long s = (long long)tile_at(j) * KT + ((long long)lane << copy_log);
        if (s >= end || (s + (1 << copy_log) <= low && s >= a.sinks)) return -1;
        const int page = table[s >> a.page_log];
        return page >= 0 && page < a.pages ? page : -1;
      };
      int page = page_of(0);
      ok = __all_sync(0xffffffffu, q_loads == 0 || mbar_wait_flat(bar_qe, (q_loads - 1) & 1, abort_flag, signs));
      if (!ok) break;
      if (lane == 0) {
        const int active = n_tok > tokens ? 2 : 1;
        mbar_expect_tx(bar_q, active * (uint32_t)(tokens * a.group) * 128 * S::HALVES);
        for (int x = 0; x < active; ++x)
          for (uint32_t h = 0; h < S::HALVES; ++h)
            tma_load_4d(base + x * S::Q_TILE + h * Q_HALF, &tm_q, bar_q, 64 * h, 0, kvh, row0 + x * tokens);
      }
      ++q_loads;
      __syncwarp();
      for (int j = 0; ok && j < n_tiles; ++j) {
        const int next = page_of(j + 1);  // (its latency hides behind the waits below)
        const uint32_t missing = __ballot_sync(0xffffffffu, lane < copies && page < 0);
        const int off = (int)(((long long)tile_at(j) * KT + ((long long)lane << copy_log)) & ((1ll << a.page_log) - 1));
#pragma unroll
        for (int kv = 0; kv < 2; ++kv) {
          ok = __all_sync(0xffffffffu, ok && mbar_wait_flat(bar_empty + 8 * f_stage, f_phase ^ 1, abort_flag, signs));
          if (!ok) break;
          const uint32_t full = bar_full + 8 * f_stage, at = base + S::RING + f_stage * S::STAGE;
          if (lane == 0) {
            if (kv == 0) {
              holes[(seen + j) % HOLES] = missing;
              signs[0] = (uint32_t)(seen + j);  // (a block of a very long cache: others wait for its end)
            }
            mbar_expect_tx(full, S::STAGE);
          }
          __syncwarp();
          if (lane < copies)
            for (uint32_t h = 0; h < S::HALVES; ++h)
              tma_load_4d(at + h * KV_HALF + ((uint32_t)lane << (copy_log + 7)), kv ? &tm_v : &tm_k, full, 64 * h, off, kvh, page);
          ++issued;
          if (++f_stage == S::STAGES) { f_stage = 0; f_phase ^= 1; }
        }
        page = next;
      }
      seen += n_tiles;
    }
    __syncwarp();
  } else if (warp >= 8) {
    asm volatile("setmaxnreg.dec.sync.aligned.u32 %0;" ::"n"(OTHER_REGS));
    // ---------------- products of one row tile ----------------
    // The whole warp walks, so that descriptors and barriers stay in uniform registers; one elected lane issues.  (Issued
    // from a branch of lane 0 alone, with the descriptors formed anew, a product took 70 to 100 cycles to issue, more than
    // it takes to run.)
    const int x = warp - 8;
    const bool leader = elect_one();
    bool ok = true;
    // the low words of the descriptors: a stage or a step of the inner dimension is an addition to them
    const uint32_t q_lo = desc_lo(base + x * S::Q_TILE, 1), k_lo = desc_lo(base + S::RING, 1), v_lo = desc_lo(base + S::RING, KV_HALF >> 4);
    const uint32_t d_s = tmem + 2 * KT * x, d_o = tmem_o + x * DP;
    uint32_t k_stage = 0, k_phase = 0, v_stage = 1, v_phase = 0;  // two walks over the ring, that of the keys two tiles ahead
    int g = 0, queries = 0;                                       // tiles of this row tile and blocks with tiles so far
    auto step = [](uint32_t& stage, uint32_t& phase) {
      stage += 2;
      if (stage >= S::STAGES) { stage -= S::STAGES; phase ^= 1; }
    };
    auto qk = [&](int b) {
      const uint32_t kl = k_lo + k_stage * (S::STAGE >> 4);
      if (leader) {
#pragma unroll
        for (uint32_t k = 0; k < DP / 16; ++k)
          umma_bf16(d_s + KT * b, desc_of(q_lo + (k >> 2) * (Q_HALF >> 4) + 2 * (k & 3)), desc_of(kl + (k >> 2) * (KV_HALF >> 4) + 2 * (k & 3)), IDESC_QK, k != 0);
        umma_commit(bar_s + 16 * x + 8 * b);
        umma_commit(bar_empty + 8 * k_stage);
      }
    };
    auto pv = [&](int b, uint32_t accumulate) {
      const uint32_t vl = v_lo + v_stage * (S::STAGE >> 4);
      if (leader) {
#pragma unroll
        for (uint32_t k = 0; k < KT / 16; ++k) umma_bf16_ts(d_o, d_s + KT * b + 8 * k, desc_of(vl + (2048 >> 4) * k), IDESC_PV<DP>, k != 0 ? 1u : accumulate);
        umma_commit(bar_o + 16 * x + 8 * b);
        umma_commit(bar_empty + 8 * v_stage);
      }
    };
    for (int k = 0; ok; ++k) {
      volatile const int* const w = take(k);
      if (!w) break;
      const int n_tiles = max(w[B_N0], w[B_N1]), nx = w[x ? B_N1 : B_N0];
      let_go(k);
      if (n_tiles == 0) continue;
      ok = __all_sync(0xffffffffu, mbar_wait_flat(bar_q, queries++ & 1, abort_flag, signs));
      auto scores = [&](int t) -> bool {  // QK(t), if this row tile walks that far; else the keys are let go unread
        if (!__all_sync(0xffffffffu, mbar_wait_flat(bar_full + 8 * k_stage, k_phase, abort_flag, signs))) return false;
        tc_fence_after();
        if (t < nx) qk((g + t) & 1);
        else if (leader) mbar_arrive(bar_empty + 8 * k_stage);
        if (leader && t + 1 == max(nx, 1)) {  // the queries have been read (or are not wanted)
          if (nx > 0) umma_commit(bar_qe);
          else mbar_arrive(bar_qe);
        }
        step(k_stage, k_phase);
        return true;
      };
      for (int t = 0; ok && t < min(2, n_tiles); ++t) ok = scores(t);
      for (int t = 0; ok && t < n_tiles; ++t) {
        const int b = (g + t) & 1;
        ok = mbar_wait_flat(bar_full + 8 * v_stage, v_phase, abort_flag, signs);
        if (t < nx) ok = ok && mbar_wait_flat(bar_p + 16 * x + 8 * b, ((g + t) >> 1) & 1, abort_flag, signs);
        ok = __all_sync(0xffffffffu, ok);
        if (!ok) break;
        tc_fence_after();
        if (t < nx) pv(b, t != 0);
        else if (leader) mbar_arrive(bar_empty + 8 * v_stage);
        step(v_stage, v_phase);
        if (t + 2 < n_tiles) ok = scores(t + 2);
      }
      g += nx;
    }
    __syncwarp();
  } else {
    asm volatile("setmaxnreg.inc.sync.aligned.u32 %0;" ::"n"(ROW_REGS));
    // ---------------- weights: one row per thread ----------------
    const int x = warp >> 2, row = (warp & 3) * 32 + lane;
    const int tok = row / a.group, head = row - tok * a.group;  // of the row tile; of the group
    const uint32_t lanes = (uint32_t)((warp & 3) * 32) << 16;
    const uint32_t t_o = tmem_o + x * DP + lanes;
    const float c = a.scale * 1.4426950408889634f;
    int g = 0, seen_tiles = 0;  // tiles of this row tile, of the CTA so far
    bool ok = true;
    for (int k = 0; ok; ++k) {
    volatile const int* const w = take(k);
    if (!w) break;
    const int n_rows = min(tokens, w[B_TOKENS] - x * tokens);   // tokens of this row tile
    const int nx = w[x ? B_N1 : B_N0], ns = w[B_NS], first = w[B_FIRST];
    auto position = [&]() -> long long {                        // of the row tile's first token
      return (long long)(((unsigned long long)(uint32_t)w[B_P_HI] << 32) | (uint32_t)w[B_P_LO]) + x * tokens;
    };
    const long long p0 = position();
    // this row sees the tokens up to hi_at that are from lo_at on or below the sinks; every row of the tile sees those up
    // to all_hi that are from all_lo on
    auto cut = [](long long v) -> int { return (int)max(-1ll, min(v, 0x7fffffffll)); };
    const int hi_at = cut(min(p0 + tok, held - 1)), lo_at = a.window ? max(0, cut(p0 + tok - a.window + 1)) : 0;
    const int all_hi = cut(min(p0, held - 1)), all_lo = a.window ? max(0, cut(p0 + n_rows - a.window)) : 0;
    // Rows of no query of this request -- other requests' queries, padding, what an earlier kernel left where no head of the group
    // falls -- have scores too, which are never stored.  They have no say in when their warp rescales its sums: answers would
    // depend on them in their last bits, and NaN among them would rescale at every tile (12 ragged prompts: 187 us, not 143).
    const bool live = tok < n_rows;
    float m = -INFINITY, l = 0.f;
    uint32_t any = 0;  // tokens that this row sees
    if (row == 0) dirty[4 * x + ((k + 2) & 3)] = 0;  // (block k - 2 is through in every warp, or k were not here; k + 2 not before all let k go)
    // The scores of tile t + 1 are on their way while the second half of tile t's weights is formed: the lower half goes to
    // the registers that tile t's lower half has left, the upper half to those of the tile before.
    float s_lo[32], s_hi[2][32];
    auto scores = [&](int t) -> bool {  // tile t's scores are in tensor memory
      const bool got = mbar_poll(bar_s + 16 * x + 8 * ((g + t) & 1), ((g + t) >> 1) & 1, abort_flag, signs);
      tc_fence_after();
      return __all_sync(0xffffffffu, got);
    };
    auto tile = [&](int t, float* hi_now, float* hi_next) -> bool {
      const int b = (g + t) & 1;
      const uint32_t t_s = tmem + KT * (2 * x + b) + lanes, t_next = tmem + KT * (2 * x + (b ^ 1)) + lanes;
      const int key0 = (t < ns ? t : first + (t - ns)) * KT;
      const uint32_t missing = holes[(seen_tiles + t) % HOLES];
      const bool whole = missing == 0 && key0 + KT - 1 <= all_hi && (key0 >= all_lo || key0 <= a.sinks - KT);
      uint32_t seen[2] = {0xffffffffu, 0xffffffffu};
      if (!whole) {
        // bit i of seen[w]: this row sees token key0 + 32 w + i
        const int hi = hi_at - key0, lo = lo_at - key0, sk = a.sinks - key0;
        const int copy_log = min(a.page_log, 6);
#pragma unroll
        for (int h = 0; h < 2; ++h) {
          seen[h] = bits_below(hi + 1 - 32 * h) & (~bits_below(lo - 32 * h) | bits_below(sk - 32 * h));
          if (missing) {
            uint32_t there = 0;
#pragma unroll
            for (int b = 0; b < 4; ++b)
              if (!((missing >> ((32 * h + 8 * b) >> copy_log)) & 1u)) there |= 0xffu << (8 * b);
            seen[h] &= there;
          }
        }
        // The values of this tile, two threads per token.  Hidden tokens meet weights of 0, which does it unless their values
        // are not finite: then they are cleared if no row of the CTA sees the token, else the block's rows are done again.
        const uint32_t vi = 2 * (seen_tiles + t) + 1;
        if (!__all_sync(0xffffffffu, mbar_wait_flat(bar_full + 8 * (vi % S::STAGES), (vi / S::STAGES) & 1, abort_flag, signs))) return false;
        const int vrow = row & (KT - 1);
        uint8_t* const v = sm + S::RING + (vi % S::STAGES) * S::STAGE + vrow * 128;
        auto chunk_of = [&](uint32_t i) -> uint4* {
          const uint32_t q = i + (row >> 6) * 4 * S::HALVES;
          return (uint4*)(v + (q >> 3) * KV_HALF + (((q & 7) ^ (row & 7)) << 4));
        };
        const __nv_bfloat162 zero = __float2bfloat162_rn(0.f);
        __nv_bfloat162 test = zero, test2 = zero;
#pragma unroll 2
        for (uint32_t i = 0; i < 4 * S::HALVES; ++i) {
          const uint4 u = *chunk_of(i);
          test = __hfma2(*(const __nv_bfloat162*)&u.x, zero, test);
          test2 = __hfma2(*(const __nv_bfloat162*)&u.y, zero, test2);
          test = __hfma2(*(const __nv_bfloat162*)&u.z, zero, test);
          test2 = __hfma2(*(const __nv_bfloat162*)&u.w, zero, test2);
        }
        test = __hadd2(test, test2);
        const bool wild = __isnan(__low2float(test)) || __isnan(__high2float(test));
        if (__any_sync(0xffffffffu, wild)) {
          const int at = key0 + vrow;
          if (wild) {
            if (at < w[B_END] && (at >= w[B_LOW] || at < a.sinks) && !((missing >> (vrow >> copy_log)) & 1u)) {
              dirty[4 * x + (k & 3)] = 1;
            } else {
#pragma unroll 1
              for (uint32_t i = 0; i < 4 * S::HALVES; ++i) *chunk_of(i) = make_uint4(0, 0, 0, 0);
            }
          }
          asm volatile("fence.proxy.async.shared::cta;" ::: "memory");
        }
      }
      any |= seen[0] | seen[1];
      auto hide = [&](float* s, uint32_t bits) {
#pragma unroll
        for (int i = 0; i < 32; ++i)
          if (!((bits >> i) & 1u)) s[i] = -INFINITY;
      };
      auto highest = [](const float* s, float top) -> float {
        float t0 = top, t1 = s[0], t2 = s[1], t3 = s[2];
#pragma unroll
        for (int i = 3; i < 31; i += 4) { t0 = max_nan(t0, s[i]); t1 = max_nan(t1, s[i + 1]); t2 = max_nan(t2, s[i + 2]); t3 = max_nan(t3, s[i + 3]); }
        return max_nan(max_nan(max_nan(t0, s[31]), t1), max_nan(t2, t3));
      };
      tmem_landed(s_lo);
      tmem_landed(hi_now);
      if (!whole) { hide(s_lo, seen[0]); hide(hi_now, seen[1]); }
      // a NaN score makes the maximum NaN and with it the weights of the row and their sum, as the quotient has it; +inf does too
      const float top = highest(hi_now, highest(s_lo, -INFINITY));
      const float m_new = max_nan(m, top);
      if (__any_sync(0xffffffffu, live && ((m_new - m) * c > GROWTH || m_new != m_new))) {  // (from -inf: yes, unless it stays there)
        const float keep = m_new == m ? 1.f : ex2((m - m_new) * c);
        l *= keep;
        m = m_new == INFINITY ? NAN : m_new;  // (inf - inf in the exponent: NaN, which not every weight's arithmetic would keep)
        if (t > 0) {
          // PV(t - 1) is done; PV(t) waits for this tile's weights
          if (!__all_sync(0xffffffffu, mbar_poll(bar_o + 16 * x + 8 * (b ^ 1), ((g + t - 1) >> 1) & 1, abort_flag, signs))) return false;
          tc_fence_after();
#pragma unroll
          for (int q = 0; q < DP / 32; ++q) {
            float o[32];
            tmem_load32(t_o + 32 * q, o);
            tmem_landed(o);
#pragma unroll
            for (int i = 0; i < 32; ++i) o[i] *= keep;
            tmem_st32(t_o + 32 * q, o);
          }
        }
      }
      const float off = m == -INFINITY ? 0.f : -m * c;
      float2 l01 = make_float2(0.f, 0.f), l23 = l01;
      const float2 cc = make_float2(c, c), oo = make_float2(off, off);
      auto weigh = [&](const float* s, int q) {  // 32 columns: weights, their sum, the bf16 ones to tensor memory
        uint32_t pk[16];
#pragma unroll
        for (int i = 0; i < 16; i += 2) {
          const float2 x0 = fma2(make_float2(s[2 * i], s[2 * i + 1]), cc, oo), x1 = fma2(make_float2(s[2 * i + 2], s[2 * i + 3]), cc, oo);
          const float2 w0 = make_float2(ex2(x0.x), ex2(x0.y));
          const float2 w1 = i % POLYNOMIAL_EVERY == 0 ? ex2_by_polynomial(x1) : make_float2(ex2(x1.x), ex2(x1.y));
          l01 = add2(l01, w0);
          l23 = add2(l23, w1);
          pk[i] = pack_bf16(w0.x, w0.y);
          pk[i + 1] = pack_bf16(w1.x, w1.y);
        }
        tmem_store16(t_s + 16 * q, pk);  // (over scores that have been read)
      };
      weigh(s_lo, 0);
      // the next scores, if they are there already; nothing waits for them before this tile's weights are handed over
      const bool more = t + 1 < nx;
      const bool early = more && __all_sync(0xffffffffu, mbar_test(bar_s + 16 * x + 8 * (b ^ 1), ((g + t + 1) >> 1) & 1));
      if (early) {
        tc_fence_after();
        tmem_load32(t_next, s_lo);
        tmem_load32(t_next + 32, hi_next);
      }
      weigh(hi_now, 1);
      l += (l01.x + l01.y) + (l23.x + l23.y);
      tmem_st_wait();
      tc_fence_before();
      __syncwarp();
      if (lane == 0) mbar_arrive(bar_p + 16 * x + 8 * b);
      if (more && !early) {
        if (!scores(t + 1)) return false;
        tmem_load32(t_next, s_lo);
        tmem_load32(t_next + 32, hi_next);
      }
      return true;
    };
    if (nx > 0) {
      ok = scores(0);
      if (ok) {
        tmem_load32(tmem + KT * (2 * x + (g & 1)) + lanes, s_lo);
        tmem_load32(tmem + KT * (2 * x + (g & 1)) + lanes + 32, s_hi[0]);
      }
      for (int t = 0; ok && t < nx; t += 2) {
        ok = tile(t, s_hi[0], s_hi[1]);
        if (ok && t + 1 < nx) ok = tile(t + 1, s_hi[1], s_hi[0]);
      }
    }
    const int last = g + nx - 1;
    if (ok && nx > 0) {
      ok = __all_sync(0xffffffffu, mbar_poll(bar_o + 16 * x + 8 * (last & 1), (last >> 1) & 1, abort_flag, signs));
      tc_fence_after();
    }
    if (ok && n_rows > 0) {
      const float inv = 1.f / l;  // (tokens, but every score -inf: 0 / 0)
      const long long at = (long long)(w[B_ROW0] + x * tokens + tok) * a.os[0] + (long long)(w[B_KVH] * a.group + head) * a.os[1];
#pragma unroll
      for (int q = 0; q < DP / 32; ++q) {
        float o[32];
        if (nx > 0) { tmem_load32(t_o + 32 * q, o); tmem_landed(o); }
#pragma unroll
        for (int i = 0; i < 32; ++i) o[i] = any ? o[i] * inv : 0.f;
        if (!live) continue;
        if (a.out_vec) {
          __nv_bfloat16* const out = (__nv_bfloat16*)a.out + at + 32 * q;
#pragma unroll
          for (int i = 0; i < 4; i += 2) {
            uint32_t u[8];
#pragma unroll
            for (int e = 0; e < 8; ++e) u[e] = pack_bf16(o[8 * i + 2 * e], o[8 * i + 2 * e + 1]);
            if (a.out_vec == 2) {  // a whole 32-byte sector at a time
              if (32 * q + 8 * i < a.D)
                asm volatile("st.global.v8.b32 [%0], {%1, %2, %3, %4, %5, %6, %7, %8};" ::"l"(out + 8 * i), "r"(u[0]), "r"(u[1]), "r"(u[2]), "r"(u[3]), "r"(u[4]),
                             "r"(u[5]), "r"(u[6]), "r"(u[7])
                             : "memory");
            } else {
              if (32 * q + 8 * i < a.D) *(uint4*)(out + 8 * i) = make_uint4(u[0], u[1], u[2], u[3]);
              if (32 * q + 8 * i + 8 < a.D) *(uint4*)(out + 8 * i + 8) = make_uint4(u[4], u[5], u[6], u[7]);
            }
          }
        } else {
#pragma unroll
          for (int i = 0; i < 32; ++i)
            if (32 * q + i < a.D) put(a.out, a.out_bf16, at + 32 * q + i, o[i]);
        }
      }
      tc_fence_before();  // (the next block's first product into O_x comes after this row's next arrival)
    }
    // A value that some of these rows see and others do not was not finite: this warp's rows again.  (Whoever found one
    // said so before its weights of that tile were handed over, without which the sums would not be done.)
    __syncwarp();
    if (ok && dirty[4 * x + (k & 3)])
      for (int r = (warp & 3) * 32; r < min((warp & 3) * 32 + 32, n_rows * a.group); ++r)
        attend_row<__nv_bfloat16>(a, w[B_REQUEST], position() + r / a.group, w[B_ROW0] + x * tokens + r / a.group, w[B_KVH] * a.group + r % a.group,
                                  (uint32_t*)signs + 1);
    g += nx;
    seen_tiles += max(w[B_N0], w[B_N1]);
    let_go(k);
    }
  }

  // ---------------- teardown ----------------
  tc_fence_before();
  __syncthreads();
  if (*abort_flag) {
    if (warp == 10 && lane == 0) {  // the latest fill of every stage, and the queries
      mbar_drain(bar_full, S::STAGES, issued, f_stage, f_phase, abort_flag);
      mbar_drain(bar_q, 1, q_loads, 0, q_loads & 1, abort_flag);
    }
    if (warp == 11 && lane == 0) mbar_drain(bar_c, 1, asked, 0, asked & 1, abort_flag);  // (a cancelled launch's answer)
    if ((warp == 8 || warp == 9) && elect_one()) {  // (the lanes that issued)
      umma_commit(bar_drain + 8 * (warp - 8));
      if (!mbar_try(bar_drain + 8 * (warp - 8), 0)) mbar_spin(bar_drain + 8 * (warp - 8), 0, abort_flag, DRAIN_NS, false);
    }
    if (threadIdx.x == 0) atomicMax(a.status, (unsigned int)ST_TIMEOUT);
    __syncthreads();
  }
  if (warp == 8) {
    tc_fence_after();
    asm volatile("tcgen05.dealloc.cta_group::1.sync.aligned.b32 %0, %1;" ::"r"(tmem), "r"(512u) : "memory");
  }
}

template <int DP>
int launch_prompt(const CUtensorMap& q, const CUtensorMap& k, const CUtensorMap& v, const Args& a, int grid, int device, cudaStream_t stream) {
  static std::atomic<uint64_t> allowed{0};
  const int st = dvm_allow_smem((const void*)dvm_attention_prompt_kernel<DP>, (int)PromptSmem<DP>::BYTES, device, &allowed);
  if (st != DVM_OK) return st;
  return dvm_launch_early(dvm_attention_prompt_kernel<DP>, grid, PROMPT_THREADS, PromptSmem<DP>::BYTES, stream, q, k, v, a);
}

}  // namespace att
}  // namespace dvm

int dvm_launch_attention_prompt(const dvm_attention_desc& d, const dvm::att::Args& a, int device, cudaStream_t stream) {
  using namespace dvm::att;
  const int tokens = PT / a.group;
  CUtensorMap q, k, v;
  int st = dvm_query_map(d, a.q, tokens, &q);
  if (st == DVM_OK) st = dvm_cache_map(d, d.k_stride, a.k, KT, &k);
  if (st == DVM_OK) st = dvm_cache_map(d, d.v_stride, a.v, KT, &v);
  if (st != DVM_OK) return st;
  // the most blocks of 2 x tokens query tokens that the requests can have
  const int64_t per = 2 * tokens, by_rows = (d.rows + d.requests * (per - 1)) / per, by_max = d.requests * ((d.max_q + per - 1) / per);
  const int64_t grid = (by_rows < by_max ? by_rows : by_max) * d.kv_heads;
  if (grid >= (1ll << 31)) return DVM_ERR_TOO_LARGE;
  return a.D <= 64 ? launch_prompt<64>(q, k, v, a, (int)grid, device, stream) : launch_prompt<128>(q, k, v, a, (int)grid, device, stream);
}

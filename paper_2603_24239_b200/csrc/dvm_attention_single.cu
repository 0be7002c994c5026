// Attention of single tokens: one query row per request over its paged cache.
//
//   out[h] = sum_s p_s v_s / sum_s p_s,   p_s = 2^(c q.k_s - m),  c = scale log2 e,  m the running maximum
//
// Bound by memory: every visible key and value is read once, 4 D flops per kv head and token against 4 D bytes times the
// group of query heads that share them.  So the work is cut by bytes: the tiles of DVM_ATT_TOKEN_TILE tokens of all
// (request, kv head) pairs form one line, and each of DVM_ATT_UNITS CTAs (two per SM) takes an equal range of it, whatever
// the lengths are -- they live on the device, so every CTA finds its range itself.  (One request alone: ranges begin where a
// head's tiles do, so that no CTA ends two pairs: 8000 tokens, 8 kv heads 16.5 -> 15.3 us, and 14.0 with no scan.)  A pair that lies in one range is
// finished there; the parts of one that spans several go to the workspace and a second kernel joins them (a dependent
// launch that starts while the first one drains).  The cut depends on the lengths alone: results do not vary.
//
// In a CTA one warp fetches tiles by TMA, page by page (128-byte swizzle, a ring of stages), and four warps take 16 tokens
// of each tile: scores and sums by mma.m16n8k16 with the query heads as the 16 rows (up to 16 share a kv head), fragments
// by ldmatrix.  Each warp keeps its own maximum, sum and output, so the warps only meet when a pair ends.  The tensor
// work is far below what the bytes take, which is why tcgen05 with its 128-row tiles and tensor-memory round trips is not
// used here.  64 requests of up to 8192 tokens, 64 / 8 heads of 128: 212 us, 6.2 TB/s; 32 requests of up to 16384 under a
// window of 4096, 32 / 32 heads: 330 us, 6.5 TB/s; one request of 8192, 32 / 8 heads: 14 us, of which the bytes take 5.
// Weights are rounded to bf16 for the second product, their sum is not: the error is that of one bf16
// rounding per weight, which averages out over the tokens.
//
// Tokens a row does not see: pages outside the pool, behind the last token or wholly hidden are never read (TMA fills
// zeros for a page index of -1); in pages that are partly visible the score becomes -inf and the value is cleared before
// the product, so nothing they hold, NaN included, reaches the result.
#include <cuda_bf16.h>
#include <cuda_runtime.h>
#include <float.h>

#include "dvm_attention.cuh"
#include "dvm_attention_launch.h"
#include "dvm_sm100.cuh"

namespace dvm {
namespace att {

using namespace sm100;

constexpr int TILE = DVM_ATT_TOKEN_TILE;
constexpr int WARPS = 4;                              // consumer warps, 16 tokens of a tile each
constexpr int THREADS = (WARPS + 1) * 32;
constexpr int MIN_TILES = 2;                          // a CTA's range is at least this long
static_assert(TILE == 16 * WARPS, "16 tokens per warp");

// The tiles of one request: sink tiles [0, ns), then tiles [first, last); visible tokens: s < end and (s >= low or s < sinks).
struct Span {
  long long end, low;
  int ns, first, count;  // count: tiles, at least one where the request has a row, else 0
};
__device__ __forceinline__ Span span_of(const Args& a, const Request& r) {
  Span p;
  const long long held = (long long)a.max_blocks << a.page_log;
  p.end = max(0ll, min(r.pos0 + 1, held));
  p.low = a.window ? max(0ll, r.pos0 - a.window + 1) : 0;
  if (p.low <= a.sinks) p.low = 0;
  p.ns = p.low ? (int)((min((long long)a.sinks, p.end) + TILE - 1) / TILE) : 0;
  p.first = max((int)min(p.low / TILE, 0x7fffffffll), p.ns);
  const int last = (int)((p.end + TILE - 1) / TILE);
  p.count = r.q_len > 0 ? max(1, p.ns + max(0, last - p.first)) : 0;
  return p;
}

// A CTA's walk over the line of tiles: a part [j0, j1) of the tiles of (request, kv head).
struct Walk {
  int request, kvh;
  Request r;
  Span p;
  long long base;   // place of the pair's first tile on the line
  int length;       // places of a pair on the line: its tiles; of one request alone, rounded up to whole ranges
  int j0, j1;
  __device__ __forceinline__ void load(const Args& a) { r = request_at(a, request); p = span_of(a, r); length = p.count; }
  __device__ __forceinline__ void cut(long long begin, long long stop) {
    j0 = (int)max(0ll, begin - base);
    j1 = (int)min((long long)p.count, stop - base);
  }
  __device__ __forceinline__ void next(const Args& a, long long begin, long long stop) {
    base += length;
    if (++kvh == a.hk) {
      kvh = 0;
      do { ++request; load(a); } while (p.count == 0);  // (only called while tiles are left: some later request has them)
    }
    cut(begin, stop);
  }
};

__device__ __forceinline__ void ldmatrix4(uint32_t addr, uint32_t (&r)[4]) {
  asm volatile("ldmatrix.sync.aligned.m8n8.x4.shared.b16 {%0, %1, %2, %3}, [%4];" : "=r"(r[0]), "=r"(r[1]), "=r"(r[2]), "=r"(r[3]) : "r"(addr) : "memory");
}
__device__ __forceinline__ void ldmatrix4_trans(uint32_t addr, uint32_t (&r)[4]) {
  asm volatile("ldmatrix.sync.aligned.m8n8.x4.trans.shared.b16 {%0, %1, %2, %3}, [%4];" : "=r"(r[0]), "=r"(r[1]), "=r"(r[2]), "=r"(r[3]) : "r"(addr) : "memory");
}
__device__ __forceinline__ void mma16816(float (&c)[4], const uint32_t (&a)[4], uint32_t b0, uint32_t b1) {
  asm volatile("mma.sync.aligned.m16n8k16.row.col.f32.bf16.bf16.f32 {%0, %1, %2, %3}, {%4, %5, %6, %7}, {%8, %9}, {%0, %1, %2, %3};"
               : "+f"(c[0]), "+f"(c[1]), "+f"(c[2]), "+f"(c[3])
               : "r"(a[0]), "r"(a[1]), "r"(a[2]), "r"(a[3]), "r"(b0), "r"(b1));
}
__device__ __forceinline__ uint32_t pack2(float lo, float hi) {
  const __nv_bfloat162 h = __floats2bfloat162_rn(lo, hi);
  return *(const uint32_t*)&h;
}
__device__ __forceinline__ void consumers_sync() { asm volatile("bar.sync 1, %0;" ::"n"(WARPS * 32) : "memory"); }

// The workspace: DVM_ATT_UNITS heads {request, first CTA, parts, slot of the first part}, then two slots of parts per CTA:
// slot 0 the part at the start of the CTA's range (the last one of a pair that began earlier, or the only one), slot 1 a
// later one.  With at most DVM_ATT_UNITS pairs there is a head per pair, written where the pair begins; with more, one per
// CTA, for the pair that continues beyond its range.
__device__ __forceinline__ int4* head_of(const Args& a, int i) { return (int4*)a.ws + i; }
__host__ __device__ __forceinline__ bool heads_by_pair(const Args& a) { return (long long)a.n * a.hk <= DVM_ATT_UNITS; }
__device__ __forceinline__ float* slot_of(const Args& a, int cta, int slot) {
  return a.ws + 4 * DVM_ATT_UNITS + ((long long)cta * 2 + slot) * a.group * (a.D + 2);
}

template <int DP>  // head_dim rounded up to 64 or 128
struct SingleSmem {
  static constexpr int HALVES = DP / 64;
  static constexpr uint32_t PART = TILE * 128;                 // 64 elements of every token of a tile
  static constexpr uint32_t STAGE = 2 * HALVES * PART;         // keys, then values
  static constexpr int STAGES = DP == 128 ? 3 : 6;
  static constexpr uint32_t SUM = STAGES * STAGE;              // [16][SUM_ROW] fp32: the warps' outputs added up
  static constexpr int SUM_ROW = DP + 8;                       // (the rows of a quarter warp lie in different banks)
  static constexpr uint32_t STATS = SUM + 16 * SUM_ROW * 4;    // [WARPS][16] maxima, [WARPS][16] sums, then [16] of each in all
  static constexpr uint32_t BARS = STATS + 2 * (WARPS + 1) * 16 * 4; // full[STAGES], empty[STAGES]
  static constexpr uint32_t BAD = BARS + 16 * STAGES;          // per stage: pages that hold nothing (a bit per copy)
  static constexpr uint32_t SCAN = BAD + 8 * STAGES;
  static constexpr uint32_t BYTES = SCAN + 16 * 8 + 16 + 1024; // 1024: alignment of the swizzled stages
};

template <int DP>
__global__ void __launch_bounds__(THREADS, 2)
dvm_attention_single_kernel(const __grid_constant__ CUtensorMap tm_k, const __grid_constant__ CUtensorMap tm_v, const __grid_constant__ Args a) {
  using S = SingleSmem<DP>;
  extern __shared__ uint8_t smem_raw[];
  const uint32_t raw = smem_u32(smem_raw), base = (raw + 1023u) & ~1023u;
  uint8_t* const sm = smem_raw + (base - raw);
  const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
  const uint32_t bar_full = base + S::BARS, bar_empty = bar_full + 8 * S::STAGES;
  volatile uint32_t* const bad = (volatile uint32_t*)(sm + S::BAD);
  long long* const scan = (long long*)(sm + S::SCAN);
  volatile uint32_t* const abort_flag = (volatile uint32_t*)(scan + 14);

  if (threadIdx.x == 0) {
    for (int s = 0; s < S::STAGES; ++s) {
      mbar_init(bar_full + 8 * s, 1);
      mbar_init(bar_empty + 8 * s, WARPS);
    }
    *abort_flag = 0;
    asm volatile("fence.mbarrier_init.release.cluster;" ::: "memory");
  }
  if (threadIdx.x == WARPS * 32) {
    tma_prefetch(&tm_k);
    tma_prefetch(&tm_v);
  }
  grid_ready();  // (the second kernel waits for this grid's end before it reads)
  grid_wait();

  Walk w;
  long long begin, stop;
  if (a.n == 1 && a.hk <= DVM_ATT_UNITS) {
    // ---- one request: every thread finds the range for itself ----
    w.request = 0;
    w.r = request_at(a, 0);
    w.p = span_of(a, w.r);
    const int count = w.p.count, units = DVM_ATT_UNITS / a.hk;  // per kv head
    const int chunk = max((count + units - 1) / units, MIN_TILES), ranges = (count + chunk - 1) / chunk;
    begin = (long long)blockIdx.x * chunk;
    stop = begin + chunk;
    w.kvh = ranges ? blockIdx.x / ranges : a.hk;
    if (w.kvh >= a.hk) return;
    w.length = ranges * chunk;
    w.base = (long long)w.kvh * w.length;
    if (threadIdx.x == 0) {
      scan[11] = chunk;
      scan[12] = stop;
    }
    __syncthreads();
  } else {
    // ---- thread t counts the tiles of requests [t per, (t + 1) per) ----
    const int per = (a.n + THREADS - 1) / THREADS;
    long long mine = 0;
    int count = 0;  // of the last one (with up to THREADS requests: the only one)
    for (int i = threadIdx.x * per; i < min(a.n, (int)(threadIdx.x + 1) * per); ++i) mine += count = span_of(a, request_at(a, i)).count;
    long long upto = mine;
#pragma unroll
    for (int d = 1; d < 32; d <<= 1) {
      const long long y = __shfl_up_sync(0xffffffffu, upto, d);
      if (lane >= d) upto += y;
    }
    if (lane == 31) scan[warp] = upto;
    __syncthreads();
    long long total = 0;
#pragma unroll
    for (int x = 0; x <= WARPS; ++x) {
      if (x < warp) upto += scan[x];
      total += scan[x];
    }
    total *= a.hk;
    const long long chunk = max((total + DVM_ATT_UNITS - 1) / DVM_ATT_UNITS, (long long)MIN_TILES);
    begin = min(total, blockIdx.x * chunk);
    stop = min(total, begin + chunk);
    if (begin == stop) {
      if (threadIdx.x == 0 && !heads_by_pair(a)) *head_of(a, blockIdx.x) = make_int4(0, 0, 0, 0);
      return;
    }
    // the thread whose requests hold tile `begin` walks to it
    const long long from = (upto - mine) * a.hk, to = upto * a.hk;
    if (begin >= from && begin < to) {
      long long at = from;
      for (int i = threadIdx.x * per;; ++i) {
        if (per > 1) count = span_of(a, request_at(a, i)).count;
        const long long after = at + (long long)count * a.hk;
        if (begin < after) {
          const long long kvh = (begin - at) / count;
          scan[8] = i;
          scan[9] = kvh;
          scan[10] = at + kvh * count;
          scan[11] = chunk;
          scan[12] = stop;
          break;
        }
        at = after;
      }
    }
    __syncthreads();
    w.request = (int)scan[8];
    w.kvh = (int)scan[9];
    w.base = scan[10];
    w.load(a);
  }
  w.cut(begin, stop);

  uint32_t f_stage = 0, f_phase = 0, issued = 0;  // the fetching warp's ring, kept for the abort path
  if (warp == WARPS) {
    // ---------------- one warp fetches: a copy of min(page, TILE) tokens per lane and 64 elements ----------------
    const int copy_log = min(a.page_log, 6), copies = TILE >> copy_log;
    bool ok = true;
    for (;;) {
      const int* table = a.table + (long long)w.request * a.max_blocks;
      auto page_of = [&](int j) -> int {  // of this lane's copy of tile j, -1 where it holds no visible token
        if (lane >= copies || j >= w.j1) return -1;
        const long long s = (long long)(j < w.p.ns ? j : w.p.first + (j - w.p.ns)) * TILE + ((long long)lane << copy_log);
        if (s >= w.p.end || (s + (1 << copy_log) <= w.p.low && s >= a.sinks)) return -1;
        const int page = table[s >> a.page_log];
        return page >= 0 && page < a.pages ? page : -1;
      };
      int page = page_of(w.j0);
      for (int j = w.j0; ok && j < w.j1; ++j) {
        const int page_next = page_of(j + 1);  // (its latency hides behind the wait below)
        ok = mbar_wait(bar_empty + 8 * f_stage, f_phase ^ 1, abort_flag);
        if (!__all_sync(0xffffffffu, ok)) { ok = false; break; }
        const uint32_t holes = __ballot_sync(0xffffffffu, lane < copies && page < 0);
        const uint32_t full = bar_full + 8 * f_stage, at = base + f_stage * S::STAGE;
        if (lane == 0) {
          bad[f_stage] = holes;
          mbar_expect_tx(full, S::STAGE);
        }
        __syncwarp();
        if (lane < copies) {
          const long long s = (long long)(j < w.p.ns ? j : w.p.first + (j - w.p.ns)) * TILE + ((long long)lane << copy_log);
          const int off = (int)(s & ((1ll << a.page_log) - 1));
#pragma unroll
          for (int h = 0; h < S::HALVES; ++h) {
            const uint32_t dst = at + h * S::PART + ((uint32_t)lane << (copy_log + 7));
            tma_load_4d(dst, &tm_k, full, 64 * h, off, w.kvh, page);
            tma_load_4d(dst + S::HALVES * S::PART, &tm_v, full, 64 * h, off, w.kvh, page);
          }
        }
        ++issued;
        if (++f_stage == S::STAGES) { f_stage = 0; f_phase ^= 1; }
        page = page_next;
      }
      if (!ok || w.base + w.length >= stop) break;
      w.next(a, begin, stop);
    }
    __syncwarp();
  } else {
    // ---------------- four warps: scores, weights, sums ----------------
    const int g = lane >> 2, t4 = lane & 3;  // this lane's rows (query heads) g, g + 8; columns 2 t4, 2 t4 + 1 of 8
    const float c = a.scale * 1.4426950408889634f;
    float* const sum = (float*)(sm + S::SUM);
    float* const stats = (float*)(sm + S::STATS);
    // ldmatrix rows of this lane: tokens for the keys (two 8 x 8 blocks of tokens, each of two 8-element columns) ...
    const int k_row = warp * 16 + (lane & 7) + ((lane >> 4) << 3), k_col = (lane >> 3) & 1;
    // ... and for the values, read transposed (two blocks of tokens of one column, then of the next)
    const int v_row = warp * 16 + (lane & 15), v_col = lane >> 4;
    int stage = 0;
    uint32_t phase = 0;
    bool ok = true;  // false: a wait ran out; the walk goes on without work, so that the warps still meet at every pair's end
    for (;;) {
      // the heads' rows of q as the A operand: k step x {row g, row g + 8} x {columns 2 t4, 2 t4 + 8}
      uint32_t qa[DP / 16][4];
      const __nv_bfloat16* q = (const __nv_bfloat16*)a.q + w.r.s0 * a.qs[0] + (long long)w.kvh * a.group * a.qs[1];
#pragma unroll
      for (int k = 0; k < DP / 16; ++k)
#pragma unroll
        for (int x = 0; x < 4; ++x) {
          const int head = g + 8 * (x & 1), d = 16 * k + 2 * t4 + 8 * (x >> 1);
          qa[k][x] = head < a.group && d < a.D ? *(const uint32_t*)(q + head * a.qs[1] + d) : 0u;
        }
      float o[DP / 8][4];
#pragma unroll
      for (int n = 0; n < DP / 8; ++n)
#pragma unroll
        for (int x = 0; x < 4; ++x) o[n][x] = 0.f;
      float m[2] = {-INFINITY, -INFINITY}, l[2] = {0.f, 0.f};
      uint32_t any = 0;  // tokens of this lane that the rows see

      for (int j = w.j0; j < w.j1; ++j) {
        ok = __all_sync(0xffffffffu, ok && mbar_wait(bar_full + 8 * stage, phase, abort_flag));
        if (!ok) break;
        const uint32_t ks = base + stage * S::STAGE, vs = ks + S::HALVES * S::PART;
        const uint32_t holes = bad[stage];
        float s[2][4] = {};
#pragma unroll
        for (int k = 0; k < DP / 16; ++k) {
          uint32_t b[4];
          const int col = 2 * (k & 3) + k_col;
          ldmatrix4(ks + (k >> 2) * S::PART + k_row * 128 + ((col ^ (k_row & 7)) << 4), b);
          mma16816(s[0], qa[k], b[0], b[1]);
          mma16816(s[1], qa[k], b[2], b[3]);
        }
        const long long s0 = (long long)(j < w.p.ns ? j : w.p.first + (j - w.p.ns)) * TILE;
        uint32_t keep[2] = {0xffffffffu, 0xffffffffu};  // per pair of this lane's tokens: the halves that are visible
        const bool whole = s0 + TILE <= w.p.end && (s0 >= w.p.low || s0 + TILE <= a.sinks) && holes == 0;
        if (!whole) {
          const int copy_log = min(a.page_log, 6);
#pragma unroll
          for (int n = 0; n < 2; ++n) {
            keep[n] = 0;
#pragma unroll
            for (int e = 0; e < 2; ++e) {
              const int at = warp * 16 + 8 * n + 2 * t4 + e;
              const long long tok = s0 + at;
              const bool seen = tok < w.p.end && (tok >= w.p.low || tok < a.sinks) && !((holes >> (at >> copy_log)) & 1u);
              if (seen) keep[n] |= 0xffffu << (16 * e);
              else s[n][e] = s[n][2 + e] = -INFINITY;
            }
          }
        }
        any |= keep[0] | keep[1];
        uint32_t p[4];
#pragma unroll
        for (int h = 0; h < 2; ++h) {  // rows g and g + 8
          float top = fmaxf(fmaxf(s[0][2 * h], s[0][2 * h + 1]), fmaxf(s[1][2 * h], s[1][2 * h + 1]));
          top = fmaxf(top, __shfl_xor_sync(0xffffffffu, top, 1));
          top = fmaxf(top, __shfl_xor_sync(0xffffffffu, top, 2));
          if (top > m[h]) {
            const float scale = exp2f((m[h] - top) * c);  // (0 for the first)
            l[h] *= scale;
#pragma unroll
            for (int n = 0; n < DP / 8; ++n) { o[n][2 * h] *= scale; o[n][2 * h + 1] *= scale; }
            m[h] = top;
          }
          const float off = m[h] == -INFINITY ? 0.f : -m[h] * c;
          const float w0 = exp2f(fmaf(s[0][2 * h], c, off)), w1 = exp2f(fmaf(s[0][2 * h + 1], c, off));
          const float w2 = exp2f(fmaf(s[1][2 * h], c, off)), w3 = exp2f(fmaf(s[1][2 * h + 1], c, off));
          l[h] += (w0 + w1) + (w2 + w3);
          p[h] = pack2(w0, w1);
          p[2 + h] = pack2(w2, w3);
        }
#pragma unroll
        for (int n = 0; n < DP / 16; ++n) {
          uint32_t b[4];
          const int col = 2 * (n & 3) + v_col;
          ldmatrix4_trans(vs + (n >> 2) * S::PART + v_row * 128 + ((col ^ (v_row & 7)) << 4), b);
          if (!whole) { b[0] &= keep[0]; b[1] &= keep[1]; b[2] &= keep[0]; b[3] &= keep[1]; }
          mma16816(o[2 * n], p, b[0], b[1]);
          mma16816(o[2 * n + 1], p, b[2], b[3]);
        }
        __syncwarp();
        if (lane == 0) mbar_arrive(bar_empty + 8 * stage);
        if (++stage == S::STAGES) { stage = 0; phase ^= 1; }
      }

      // ---- the pair's part is done: the four warps' results become one ----
      // From here on a maximum of -inf says that no token was seen; tokens whose scores are all -inf have the lowest finite one.
      any = __any_sync(0xffffffffu, any != 0);
#pragma unroll
      for (int h = 0; h < 2; ++h) {
        if (any) m[h] = fmaxf(m[h], -FLT_MAX);
        l[h] += __shfl_xor_sync(0xffffffffu, l[h], 1);
        l[h] += __shfl_xor_sync(0xffffffffu, l[h], 2);
        if (t4 == 0) {
          stats[warp * 16 + g + 8 * h] = m[h];
          stats[(WARPS + warp) * 16 + g + 8 * h] = l[h];
        }
      }
      consumers_sync();
      float f[2];
#pragma unroll
      for (int h = 0; h < 2; ++h) {
        float top = -INFINITY, all = 0.f;
#pragma unroll
        for (int x = 0; x < WARPS; ++x) top = fmaxf(top, stats[x * 16 + g + 8 * h]);
#pragma unroll
        for (int x = 0; x < WARPS; ++x) {
          const float e = top == -INFINITY ? 1.f : exp2f((stats[x * 16 + g + 8 * h] - top) * c);
          all = fmaf(stats[(WARPS + x) * 16 + g + 8 * h], e, all);
          if (x == warp) f[h] = e;
        }
        if (warp == 0 && t4 == 0) {
          stats[2 * WARPS * 16 + g + 8 * h] = top;
          stats[(2 * WARPS + 1) * 16 + g + 8 * h] = all;
        }
      }
      // each warp adds another quarter of the columns at a time: always in the same order
#pragma unroll 1
      for (int x = 0; x < WARPS; ++x) {
#pragma unroll
        for (int n = 0; n < DP / 8; ++n)
          if (n / (DP / 32) == ((warp + x) & 3)) {
#pragma unroll
            for (int h = 0; h < 2; ++h)
              if (g + 8 * h < a.group) {
                float2* at = (float2*)(sum + (g + 8 * h) * S::SUM_ROW + 8 * n + 2 * t4);
                float2 v = make_float2(o[n][2 * h] * f[h], o[n][2 * h + 1] * f[h]);
                if (x) { v.x += at->x; v.y += at->y; }
                *at = v;
              }
          }
        consumers_sync();
      }
      // (read again: kept in registers, they would cost the loop above its own)
      const long long chunk = ((volatile long long*)scan)[11], stop = ((volatile long long*)scan)[12], begin = blockIdx.x * chunk;
      const bool alone = w.j0 == 0 && w.j1 == w.p.count;
      const int slot = w.j0 == 0 && w.base > begin ? 1 : 0;
      float* const part = slot_of(a, blockIdx.x, slot);
      for (int head = warp; head < a.group; head += WARPS) {
        const float top = stats[2 * WARPS * 16 + head], all = stats[(2 * WARPS + 1) * 16 + head];
        const float by = top == -INFINITY ? 0.f : 1.f / all;  // (tokens, but every score -inf: 0 / 0)
        const long long at = w.r.s0 * a.os[0] + ((long long)w.kvh * a.group + head) * a.os[1];
#pragma unroll
        for (int e = 0; e < DP / 32; ++e) {
          const int d = lane + 32 * e;
          if (d < a.D) {
            const float v = sum[head * S::SUM_ROW + d];
            if (alone) put(a.out, a.out_bf16, at + d, v * by);
            else part[head * a.D + d] = v;
          }
        }
        if (!alone && lane == 0) {
          part[a.group * a.D + head] = top;
          part[a.group * (a.D + 1) + head] = all;
        }
      }
      const long long after = w.base + w.length;
      if (threadIdx.x == 0) {
        const bool by_pair = heads_by_pair(a);
        const int parts = w.j0 == 0 && after > stop ? (int)((after - 1) / chunk) - (int)blockIdx.x + 1 : 0;
        if (by_pair ? w.j0 == 0 : after >= stop)
          *head_of(a, by_pair ? w.request * a.hk + w.kvh : (int)blockIdx.x) = make_int4(w.request * a.hk + w.kvh, blockIdx.x, parts, slot);
      }
      if (after >= stop) break;
      consumers_sync();  // the sums and statistics have been read
      w.next(a, begin, stop);
    }
  }
  __syncthreads();
  if (*abort_flag) {  // whoever's wait ran out: the copies in flight land first
    if (threadIdx.x == WARPS * 32) mbar_drain(bar_full, S::STAGES, issued, f_stage, f_phase, abort_flag);
    if (threadIdx.x == 0) atomicMax(a.status, (unsigned int)ST_TIMEOUT);
  }
}

// Joins the parts of a pair that spans several ranges: one CTA per head (grid x) and query head of the pair (grid y).
// The parts' maxima and sums first, then every warp adds up every JOIN_WARPS-th part, then the warps' sums in their order.
constexpr int JOIN_WARPS = 8, AHEAD = 4;
__global__ void __launch_bounds__(JOIN_WARPS * 32) dvm_attention_join_kernel(const __grid_constant__ Args a) {
  __shared__ float weight[DVM_ATT_UNITS];
  __shared__ float stat[2][JOIN_WARPS];
  __shared__ float sums[JOIN_WARPS][128];
  const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31, h = blockIdx.y;
  grid_ready();
  grid_wait();
  const int4 head = *head_of(a, blockIdx.x);
  const bool by_pair = heads_by_pair(a);
  if (by_pair && request_at(a, blockIdx.x / a.hk).q_len == 0) return;  // (no row: no CTA wrote this head)
  const int parts = head.z;
  if (parts < 2) return;
  const float c = a.scale * 1.4426950408889634f;
  const int size = a.group * a.D;
  auto part = [&](int k) -> const float* { return slot_of(a, head.y + k, k ? 0 : head.w); };
  // Everything is asked for at once: statistics of part threadIdx.x, the first AHEAD outputs of this warp, the row's place.
  const int request = head.x / a.hk, kvh = head.x - request * a.hk;
  const long long row = request_at(a, request).s0;
  float m0 = -INFINITY, l0 = 0.f, first[AHEAD][4] = {};
  if ((int)threadIdx.x < parts) {
    const float* p = part(threadIdx.x) + size + h;
    m0 = p[0];
    l0 = p[a.group];
  }
#pragma unroll
  for (int x = 0; x < AHEAD; ++x) {
    const int k = warp + x * JOIN_WARPS;
    if (k < parts) {
      const float* p = part(k) + h * a.D;
#pragma unroll
      for (int e = 0; e < 4; ++e)
        if (lane + 32 * e < a.D) first[x][e] = p[lane + 32 * e];
    }
  }
  float m = m0, l = 0.f;
  for (int k = threadIdx.x + JOIN_WARPS * 32; k < parts; k += JOIN_WARPS * 32) m = fmaxf(m, part(k)[size + h]);
#pragma unroll
  for (int d = 16; d > 0; d >>= 1) m = fmaxf(m, __shfl_xor_sync(0xffffffffu, m, d));
  if (lane == 0) stat[0][warp] = m;
  __syncthreads();
#pragma unroll
  for (int x = 0; x < JOIN_WARPS; ++x) m = fmaxf(m, stat[0][x]);
  for (int k = threadIdx.x; k < parts; k += JOIN_WARPS * 32) {
    const bool other = k >= JOIN_WARPS * 32;
    const float mk = other ? part(k)[size + h] : m0, lk = other ? part(k)[size + a.group + h] : l0;
    weight[k] = mk == -INFINITY ? 0.f : exp2f((mk - m) * c);  // (a part that saw nothing is all zeros)
    l += lk * weight[k];
  }
#pragma unroll
  for (int d = 16; d > 0; d >>= 1) l += __shfl_xor_sync(0xffffffffu, l, d);
  if (lane == 0) stat[1][warp] = l;
  __syncthreads();
  float v[4] = {};
#pragma unroll
  for (int x = 0; x < AHEAD; ++x) {
    const int k = warp + x * JOIN_WARPS;
    if (k < parts)
#pragma unroll
      for (int e = 0; e < 4; ++e) v[e] = fmaf(first[x][e], weight[k], v[e]);
  }
#pragma unroll 4
  for (int k = warp + AHEAD * JOIN_WARPS; k < parts; k += JOIN_WARPS) {
    const float* p = part(k) + h * a.D;
    const float f = weight[k];
#pragma unroll
    for (int e = 0; e < 4; ++e)
      if (lane + 32 * e < a.D) v[e] = fmaf(p[lane + 32 * e], f, v[e]);
  }
#pragma unroll
  for (int e = 0; e < 4; ++e) sums[warp][lane + 32 * e] = v[e];
  __syncthreads();
  l = 0.f;
#pragma unroll
  for (int x = 0; x < JOIN_WARPS; ++x) l += stat[1][x];
  if (threadIdx.x < a.D) {
    float all = 0.f;
#pragma unroll
    for (int x = 0; x < JOIN_WARPS; ++x) all += sums[x][threadIdx.x];
    put(a.out, a.out_bf16, row * a.os[0] + ((long long)kvh * a.group + h) * a.os[1] + threadIdx.x, m == -INFINITY ? 0.f : all / l);
  }
}

template <int DP>
int launch_single(const CUtensorMap& k, const CUtensorMap& v, const Args& a, int device, cudaStream_t stream) {
  static std::atomic<uint64_t> allowed{0};
  const int st = dvm_allow_smem((const void*)dvm_attention_single_kernel<DP>, (int)SingleSmem<DP>::BYTES, device, &allowed);
  if (st != DVM_OK) return st;
  return dvm_launch_early(dvm_attention_single_kernel<DP>, DVM_ATT_UNITS, THREADS, SingleSmem<DP>::BYTES, stream, k, v, a);
}

}  // namespace att
}  // namespace dvm

int dvm_launch_attention_single(const dvm_attention_desc& d, const dvm::att::Args& a, int device, cudaStream_t stream) {
  using namespace dvm::att;
  CUtensorMap k, v;
  int st = dvm_cache_map(d, d.k_stride, a.k, TILE, &k);
  if (st == DVM_OK) st = dvm_cache_map(d, d.v_stride, a.v, TILE, &v);
  if (st == DVM_OK) st = a.D <= 64 ? launch_single<64>(k, v, a, device, stream) : launch_single<128>(k, v, a, device, stream);
  if (st != DVM_OK) return st;
  return dvm_launch_early(dvm_attention_join_kernel, dim3(heads_by_pair(a) ? a.n * a.hk : DVM_ATT_UNITS, a.group), JOIN_WARPS * 32, 0, stream, a);
}

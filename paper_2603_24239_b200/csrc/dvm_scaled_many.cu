// Scaled product for many rows to a weight.
//
//   out[r, n] = sum_b xs[r, b] ws[n / 128, b] D_b[r, n],   D_b = x[r, block b of k] w[n, block b of k]^T
//
// Bound by the products, 2 k flops to an output at twice the rate of bf16 (512 cycles for a k block of a tile of 128 x 256; the
// 48 KB it takes from L2 are 768 at 64 bytes a cycle), then by power.  CTAs, one per SM, take the tiles of all groups in turn
// (rows first, so that those at work share the weights' tiles in L2).  One thread fetches by TMA (a ring of stages of 128 of
// k); a warp issues the four products of a k block into one of two places in tensor memory; eight warps take them out --
// thread r holds row r and 128 of the columns, in registers -- and add them up with the row's scale times the weight's: 128
// multiply-adds a thread to a block, two to an instruction, 290 cycles of an SM, 500 with the loads from tensor memory.  Two
// warps copy the scales of four blocks at a time into shared memory, ahead of all that.  At a tile's end rows leave by TMA from
// shared memory, beside the next tile's sums; of a warp whose rows are not all the group's each thread stores its own.
// A place in tensor memory is taken for the products (512 cycles), their end's arrival (190), the loads and sums (500) and the
// way back (200), and there are two: 700 cycles a block, or L2's 768.  It takes 950 (4096 rows, 4096 to 5632: cycles of the SMs over
// their blocks) to 1000; which of the ends of tiles, where rows are packed, and of what else holds the other 200 is not known.  8192
// rows, 4096 to 11008: 360 us in bursts, 2.05 PFLOP/s (1.7 GHz), 407 to 417 in calls in a row at the power cap (1.42 GHz).
// (The compiler keeps some values of a tile in memory: 9 loads a warp and tile, none to a block, by the counters.)
// Built and not faster: pairs of CTAs (cta_group::2; half the weight's bytes from L2, but a commit to both CTAs and an arrival at
// the other take 800 cycles more); places of half the columns each (416 us: x is read from shared memory twice); 32 columns at a time from tensor memory
// (spilled registers: 430 to 520 us); all waits polled without sleep (no change).
#include "dvm_experts_launch.h"
#include "dvm_scaled.cuh"

namespace dvm {
namespace scaled {

constexpr int MANY_THREADS = 384, MANY_M = 128, MANY_N = 256, HALF = MANY_N / 2, MANY_STAGES = 3, AHEAD = 4;   // AHEAD: k blocks whose scales come together
constexpr int SUM_REGS = 232, OTHER_REGS = 40;   // of a thread of the eight warps, and of the others
static_assert(256 * SUM_REGS + 128 * OTHER_REGS <= MANY_THREADS * 168, "an increase draws on the registers of the launch");

struct ManySmem {
  static constexpr uint32_t X = MANY_M * BLOCK, W = MANY_N * BLOCK, STAGE = X + W;
  static constexpr uint32_t OUT_BOX = 32 * 128;                             // 32 rows of 128 bytes
  static constexpr uint32_t OUT = MANY_STAGES * STAGE;                      // 8 warps x 2 boxes
  static constexpr uint32_t XS = OUT + 8 * 2 * OUT_BOX;                     // [2][AHEAD][MANY_M] scales of x
  static constexpr uint32_t WS = XS + 2 * AHEAD * MANY_M * 4;               // [2][2 halves][AHEAD] scales of the weight
  static constexpr uint32_t BARS = WS + 2 * 2 * AHEAD * 4;                  // full[STAGES], done[STAGES], free[2], laid[2], read[2], last
  static constexpr uint32_t WORDS = BARS + 8 * (2 * MANY_STAGES + 7);       // abort flag, two counts of nothing, place of tensor memory
  static constexpr uint32_t LINE = (WORDS + 16 + 15) / 16 * 16;             // tiles before each group
  static constexpr uint32_t FIRST = LINE + (DVM_MAX_WEIGHT_GROUPS + 1 + MANY_THREADS / 32) * 8;   // first row of each group
  static constexpr uint32_t BYTES = FIRST + (DVM_MAX_WEIGHT_GROUPS + 1) * 4 + 1024;
  static_assert(BYTES <= 227 * 1024, "");
};

// 16 columns of this thread's lane of tensor memory: asked for, and there (the values must not be used in between)
__device__ __forceinline__ void tmem_ask(uint32_t taddr, uint32_t (&r)[16]) {
  asm volatile("tcgen05.ld.sync.aligned.32x32b.x16.b32 {%0, %1, %2, %3, %4, %5, %6, %7, %8, %9, %10, %11, %12, %13, %14, %15}, [%16];"
               : "=r"(r[0]), "=r"(r[1]), "=r"(r[2]), "=r"(r[3]), "=r"(r[4]), "=r"(r[5]), "=r"(r[6]), "=r"(r[7]), "=r"(r[8]), "=r"(r[9]), "=r"(r[10]), "=r"(r[11]),
                 "=r"(r[12]), "=r"(r[13]), "=r"(r[14]), "=r"(r[15])
               : "r"(taddr)
               : "memory");
}
__device__ __forceinline__ void tmem_have(uint32_t (&r)[16]) {
  asm volatile("tcgen05.wait::ld.sync.aligned;"
               : "+r"(r[0]), "+r"(r[1]), "+r"(r[2]), "+r"(r[3]), "+r"(r[4]), "+r"(r[5]), "+r"(r[6]), "+r"(r[7]), "+r"(r[8]), "+r"(r[9]), "+r"(r[10]), "+r"(r[11]),
                 "+r"(r[12]), "+r"(r[13]), "+r"(r[14]), "+r"(r[15])
               :
               : "memory");
}
__device__ __forceinline__ void add16(float2* acc, const uint32_t (&r)[16], float by) {
#pragma unroll
  for (int i = 0; i < 8; ++i) acc[i] = fma2(make_float2(__uint_as_float(r[2 * i]), __uint_as_float(r[2 * i + 1])), make_float2(by, by), acc[i]);
}
__device__ __forceinline__ void tma_store_2d(const CUtensorMap* map, uint32_t src, int x, int y) {
  asm volatile("cp.async.bulk.tensor.2d.global.shared::cta.tile.bulk_group [%0, {%2, %3}], [%1];" ::"l"(map), "r"(src), "r"(x), "r"(y) : "memory");
  asm volatile("cp.async.bulk.commit_group;" ::: "memory");
}

__device__ __forceinline__ void copy4(uint32_t dst, const float* p) { asm volatile("cp.async.ca.shared.global [%0], [%1], 4;" ::"r"(dst), "l"(p) : "memory"); }

// The tiles of a CTA, one after another.
struct Tiles {
  const long long* line;
  const int* first_of;
  long long t, tiles;
  int groups, g;
  int first, rows, n0;   // first row, rows, first column
  __device__ __forceinline__ bool at() {
    if (t >= tiles) return false;
    while (line[g + 1] <= t) ++g;
    const int from = first_of[g], all = first_of[g + 1] - from, down = (all + MANY_M - 1) / MANY_M, in_group = (int)(t - line[g]), nb = in_group / down;   // (all > 0: the group has tiles)
    const int into = (in_group - nb * down) * MANY_M;
    first = from + into;
    rows = min(MANY_M, all - into);
    n0 = nb * MANY_N;
    return true;
  }
  __device__ __forceinline__ bool next() {
    t += gridDim.x;
    return at();
  }
};

// 16 bytes of results of type T
template <class T> struct Out;
template <> struct Out<__nv_bfloat16> {
  static __device__ __forceinline__ uint4 pack(const float2* f) {
    uint32_t p[4];
#pragma unroll
    for (int k = 0; k < 4; ++k) {
      const __nv_bfloat162 b = __floats2bfloat162_rn(f[k].x, f[k].y);
      p[k] = *(const uint32_t*)&b;
    }
    return make_uint4(p[0], p[1], p[2], p[3]);
  }
};
template <> struct Out<float> {
  static __device__ __forceinline__ uint4 pack(const float2* f) {
    return make_uint4(__float_as_uint(f[0].x), __float_as_uint(f[0].y), __float_as_uint(f[1].x), __float_as_uint(f[1].y));
  }
};

template <class T>   // T: of the result
__global__ void __launch_bounds__(MANY_THREADS, 1)
dvm_scaled_many_kernel(const __grid_constant__ CUtensorMap tm_x, const __grid_constant__ CUtensorMap tm_w, const __grid_constant__ CUtensorMap tm_out,
                       const __grid_constant__ Args a) {
  using S = ManySmem;
  constexpr int PIECE = 16 / sizeof(T), PER_LINE = 128 / sizeof(T);   // results in 16 bytes, and in a line of a box
  extern __shared__ uint8_t smem_raw[];
  const uint32_t raw = smem_u32(smem_raw), base = (raw + 1023u) & ~1023u;
  uint8_t* const sm = smem_raw + (base - raw);
  const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
  // full: a stage has landed; done: its products have ended, which frees it; free: a place in tensor memory has been read; laid,
  // read: scales of AHEAD blocks
  const uint32_t bar_full = base + S::BARS, bar_done = bar_full + 8 * MANY_STAGES, bar_free = bar_done + 8 * MANY_STAGES, bar_laid = bar_free + 16, bar_read = bar_laid + 16,
                 bar_last = bar_read + 16;
  volatile uint32_t* const abort_flag = (volatile uint32_t*)(sm + S::WORDS);
  volatile uint32_t* const idle = abort_flag + 1;
  uint32_t* const tmem_slot = (uint32_t*)(sm + S::WORDS) + 3;
  long long* const line = (long long*)(sm + S::LINE);
  int* const first_of = (int*)(sm + S::FIRST);

  if (threadIdx.x == 0) {
    for (int s = 0; s < MANY_STAGES; ++s) { mbar_init(bar_full + 8 * s, 1); mbar_init(bar_done + 8 * s, 1); }
    for (int s = 0; s < 2; ++s) { mbar_init(bar_free + 8 * s, 8); mbar_init(bar_laid + 8 * s, 64); mbar_init(bar_read + 8 * s, 8); }
    mbar_init(bar_last, 1);
    abort_flag[0] = abort_flag[1] = abort_flag[2] = 0;
    asm volatile("fence.mbarrier_init.release.cluster;" ::: "memory");
    tma_prefetch(&tm_x);
    tma_prefetch(&tm_w);
    tma_prefetch(&tm_out);
  }
  grid_ready();
  grid_wait();
  if (warp == 1) {
    asm volatile("tcgen05.alloc.cta_group::1.sync.aligned.shared::cta.b32 [%0], 512;" ::"r"(smem_u32(tmem_slot)) : "memory");
    asm volatile("tcgen05.relinquish_alloc_permit.cta_group::1.sync.aligned;" ::: "memory");
  }
  for (int g = threadIdx.x; g <= a.groups; g += MANY_THREADS) first_of[g] = a.starts ? min(max(a.starts[g], 0), a.rows) : g ? a.rows : 0;
  lay_out<MANY_THREADS>(a, MANY_M, (a.n + MANY_N - 1) / MANY_N, line, line + a.groups + 1);
  tc_fence_before();
  __syncthreads();
  tc_fence_after();
  const uint32_t tmem = *(volatile uint32_t*)tmem_slot;
  Tiles tile = {line, first_of, blockIdx.x, line[a.groups], a.groups, 0, 0, 0, 0};

  uint32_t issued = 0, f_stage = 0, f_phase = 0;   // the fetching thread's ring, kept for the abort path
  if (warp == 0) {
    asm volatile("setmaxnreg.dec.sync.aligned.u32 %0;" ::"n"(OTHER_REGS));
    const bool leader = elect_one();
    bool ok = true;
    for (bool some = tile.at(); ok && some; some = tile.next())
      for (int kb = 0; kb < a.k_blocks; ++kb) {
        ok = __all_sync(ALL, mbar_wait_flat(bar_done + 8 * f_stage, f_phase ^ 1, abort_flag, idle));
        if (!ok) break;
        const uint32_t at = base + f_stage * S::STAGE, full = bar_full + 8 * f_stage;
        if (leader) {
          mbar_expect_tx(full, S::STAGE);
          tma_load_2d(at, &tm_x, full, kb * BLOCK, tile.first);
          tma_load_3d(at + S::X, &tm_w, full, kb * BLOCK, tile.n0, tile.g);
        }
        ++issued;
        if (++f_stage == MANY_STAGES) { f_stage = 0; f_phase ^= 1; }
      }
    __syncwarp();
  } else if (warp == 1) {
    asm volatile("setmaxnreg.dec.sync.aligned.u32 %0;" ::"n"(OTHER_REGS));
    const bool leader = elect_one();
    const uint32_t x0 = desc_lo(base), w0 = desc_lo(base + S::X);
    uint32_t stage = 0, phase = 0, buffer = 0, b_phase = 0;
    bool ok = true;
    for (bool some = tile.at(); ok && some; some = tile.next())
      for (int kb = 0; ok && kb < a.k_blocks; ++kb) {
        ok = __all_sync(ALL, mbar_wait_flat(bar_free + 8 * buffer, b_phase ^ 1, abort_flag, idle) && mbar_wait_flat(bar_full + 8 * stage, phase, abort_flag, idle));
        if (!ok) break;
        tc_fence_after();
        if (leader) {
          const uint32_t x = x0 + stage * (S::STAGE >> 4), w = w0 + stage * (S::STAGE >> 4);
#pragma unroll
          for (int k = 0; k < BLOCK / 32; ++k) umma_e4m3(tmem + buffer * MANY_N, desc_of(x + 2 * k), desc_of(w + 2 * k), IDESC<MANY_M, MANY_N>, k != 0);
          umma_commit(bar_done + 8 * stage);
        }
        if (++stage == MANY_STAGES) { stage = 0; phase ^= 1; }
        if (++buffer == 2) { buffer = 0; b_phase ^= 1; }
      }
    if (leader) {   // every product has ended before tensor memory is given back, whatever else ended early
      umma_commit(bar_last);
      mbar_spin(bar_last, 0, abort_flag, DRAIN_NS, false);
    }
    __syncwarp();
  } else if (warp < 4) {
    // ---------------- two warps fetch the scales: thread i those of rows i and i + 64 ----------------
    asm volatile("setmaxnreg.dec.sync.aligned.u32 %0;" ::"n"(OTHER_REGS));
    const int i = threadIdx.x - 64;
    uint32_t slot = 0, phase = 0;
    bool ok = true;
    for (bool some = tile.at(); ok && some; some = tile.next()) {
      const float* const xs0 = a.xs + (long long)(tile.first + min(i, tile.rows - 1)) * a.xs_stride;
      const float* const xs1 = a.xs + (long long)(tile.first + min(i + 64, tile.rows - 1)) * a.xs_stride;
      // threads 0 .. 2 AHEAD - 1: block i % AHEAD of half i / AHEAD
      const float* const ws = a.ws + ((long long)tile.g * a.n_blocks + min(tile.n0 / BLOCK + i / AHEAD, a.n_blocks - 1)) * a.k_blocks + i % AHEAD;
      for (int kb = 0; kb < a.k_blocks; kb += AHEAD) {
        ok = __all_sync(ALL, mbar_wait_flat(bar_read + 8 * slot, phase ^ 1, abort_flag, idle));
        if (!ok) break;
        const uint32_t x = base + S::XS + slot * (AHEAD * MANY_M * 4) + i * 4;
#pragma unroll
        for (int k = 0; k < AHEAD; ++k)
          if (kb + k < a.k_blocks) {
            copy4(x + k * (MANY_M * 4), xs0 + kb + k);
            copy4(x + k * (MANY_M * 4) + 256, xs1 + kb + k);
          }
        if (i < 2 * AHEAD && kb + i % AHEAD < a.k_blocks) copy4(base + S::WS + (slot * 2 * AHEAD + i) * 4, ws + kb);
        asm volatile("cp.async.mbarrier.arrive.noinc.shared::cta.b64 [%0];" ::"r"(bar_laid + 8 * slot) : "memory");
        if (++slot == 2) { slot = 0; phase ^= 1; }
      }
    }
    asm volatile("cp.async.wait_all;" ::: "memory");
  } else {
    asm volatile("setmaxnreg.inc.sync.aligned.u32 %0;" ::"n"(SUM_REGS));
    const int quarter = warp & 3, half = (warp - 4) >> 2, row = quarter * 32 + lane;
    const uint32_t mine = tmem + ((uint32_t)(quarter * 32) << 16) + half * HALF;
    const float* const xs = (const float*)(sm + S::XS) + row;
    const float* const ws = (const float*)(sm + S::WS) + half * AHEAD;
    uint32_t buffer = 0, stage = 0, phase = 0, slot = 0, s_phase = 0;
    bool ok = true;
    for (bool some = tile.at(); ok && some; some = tile.next()) {
      float2 acc[64];
#pragma unroll
      for (int i = 0; i < 64; ++i) acc[i] = make_float2(0.f, 0.f);
      float by[AHEAD];
      for (int kb = 0; kb < a.k_blocks; ++kb) {
        if (kb % AHEAD == 0) {
          ok = __all_sync(ALL, mbar_wait_flat(bar_laid + 8 * slot, s_phase, abort_flag, idle));
          if (!ok) break;
          const float4 w = *(const float4*)(ws + slot * 2 * AHEAD);
          const float* const x = xs + slot * AHEAD * MANY_M;
          by[0] = x[0] * w.x; by[1] = x[MANY_M] * w.y; by[2] = x[2 * MANY_M] * w.z; by[3] = x[3 * MANY_M] * w.w;
          __syncwarp();
          if (lane == 0) mbar_arrive(bar_read + 8 * slot);
          if (++slot == 2) { slot = 0; s_phase ^= 1; }
        }
        ok = __all_sync(ALL, mbar_wait_flat(bar_done + 8 * stage, phase, abort_flag, idle));
        if (!ok) break;
        if (++stage == MANY_STAGES) { stage = 0; phase ^= 1; }
        tc_fence_after();
        const uint32_t at = mine + buffer * MANY_N;
        uint32_t u[16], v[16];
        tmem_ask(at, u);
#pragma unroll
        for (int c = 0; c < 8; c += 2) {
          tmem_have(u);
          tmem_ask(at + 16 * c + 16, v);
          add16(acc + 8 * c, u, by[0]);
          tmem_have(v);
          if (c < 6) {
            tmem_ask(at + 16 * c + 32, u);
          } else {   // all has been read
            tc_fence_before();
            __syncwarp();
            if (lane == 0) mbar_arrive(bar_free + 8 * buffer);
          }
          add16(acc + 8 * c + 8, v, by[0]);
        }
        by[0] = by[1]; by[1] = by[2]; by[2] = by[3];
        buffer ^= 1;
      }
      if (!ok) break;
      // ---- results ----
      const int c0 = tile.n0 + half * HALF, cols = min(HALF, a.n - c0);   // (0 or less: this half lies behind the last column)
      if (a.out_tma && quarter * 32 + 32 <= tile.rows && cols > 0) {
        const uint32_t box = base + S::OUT + (warp - 4) * 2 * S::OUT_BOX;
        uint8_t* const my_line = sm + S::OUT + (warp - 4) * 2 * S::OUT_BOX + lane * 128;
        // all 32 rows of the warp: 128 bytes of each at a time into shared memory (pieces of 16 bytes swizzled by row), out by TMA
#pragma unroll
        for (int c = 0; c < HALF / PER_LINE; ++c) {
          // (of the two boxes the one that was stored first has been read)
          if (lane == 0) asm volatile("cp.async.bulk.wait_group.read 1;" ::: "memory");
          __syncwarp();
#pragma unroll
          for (int i = 0; i < 8; ++i) *(uint4*)(my_line + (c & 1) * S::OUT_BOX + ((i ^ (lane & 7)) << 4)) = Out<T>::pack(acc + (8 * c + i) * (PIECE / 2));
          asm volatile("fence.proxy.async.shared::cta;" ::: "memory");
          __syncwarp();
          if (lane == 0) tma_store_2d(&tm_out, box + (c & 1) * S::OUT_BOX, c0 + c * PER_LINE, tile.first + quarter * 32);
        }
      } else if (a.out_tma && cols == HALF) {
        if (row < tile.rows) {
          T* const out = (T*)a.out + (long long)(tile.first + row) * a.out_stride + c0;
#pragma unroll
          for (int i = 0; i < HALF / PIECE; ++i) *(uint4*)(out + i * PIECE) = Out<T>::pack(acc + i * (PIECE / 2));
        }
      } else if (cols > 0 && quarter * 32 < tile.rows) {
        // results that no copy out takes: the same lines through shared memory, so that a store has neighbours of one row
        const int rows = min(32, tile.rows - quarter * 32);
        uint8_t* const boxes = sm + S::OUT + (warp - 4) * 2 * S::OUT_BOX;
        T* const out = (T*)a.out + (long long)(tile.first + quarter * 32) * a.out_stride + c0;
        if (lane == 0) asm volatile("cp.async.bulk.wait_group.read 0;" ::: "memory");
        __syncwarp();
#pragma unroll
        for (int c = 0; c < HALF / PER_LINE; ++c) {
          uint8_t* const box = boxes + (c & 1) * S::OUT_BOX;
#pragma unroll
          for (int i = 0; i < 8; ++i) *(uint4*)(box + lane * 128 + ((i ^ (lane & 7)) << 4)) = Out<T>::pack(acc + (8 * c + i) * (PIECE / 2));
          __syncwarp();
          for (int r = 0; r < rows; ++r)
#pragma unroll
            for (int e = lane; e < PER_LINE; e += 32)
              if (c * PER_LINE + e < cols)
                out[r * a.out_stride + c * PER_LINE + e] = *(const T*)(box + r * 128 + (((e / PIECE) ^ (r & 7)) << 4) + e % PIECE * sizeof(T));
          __syncwarp();
        }
      }
    }
    if (lane == 0) asm volatile("cp.async.bulk.wait_group 0;" ::: "memory");
    __syncwarp();
  }
  tc_fence_before();
  __syncthreads();
  tc_fence_after();
  if (warp == 1) asm volatile("tcgen05.dealloc.cta_group::1.sync.aligned.b32 %0, 512;" ::"r"(tmem) : "memory");
  if (*abort_flag && threadIdx.x == 0) {   // whoever's wait ran out: the copies in flight land first
    mbar_drain(bar_full, MANY_STAGES, issued, f_stage, f_phase, abort_flag);
    atomicMax(a.status, (unsigned int)ST_TIMEOUT);
  }
}

}  // namespace scaled
}  // namespace dvm

namespace {
template <class T>
int launch(const CUtensorMap& x, const CUtensorMap& w, const CUtensorMap& out, const dvm::scaled::Args& a, int sm_count, int device, cudaStream_t stream) {
  using namespace dvm::scaled;
  static std::atomic<uint64_t> allowed{0};
  const int st = dvm_allow_smem((const void*)dvm_scaled_many_kernel<T>, (int)ManySmem::BYTES, device, &allowed);
  return st != DVM_OK ? st : dvm_launch_next(dvm_scaled_many_kernel<T>, sm_count, MANY_THREADS, ManySmem::BYTES, stream, x, w, out, a);
}
}  // namespace

int dvm_launch_scaled_many(const CUtensorMap& x, const CUtensorMap& w, const CUtensorMap& out, const dvm::scaled::Args& a, int sm_count, int device,
                           cudaStream_t stream) {
  return a.out_bf16 ? launch<__nv_bfloat16>(x, w, out, a, sm_count, device, stream) : launch<float>(x, w, out, a, sm_count, device, stream);
}

// Scaled product for few rows to a weight.
//
//   out[r, n] = sum_b xs[r, b] ws[n / 128, b] D_b[n, r],   D_b = w[n, block b of k] x[r, block b of k]^T
//
// Bound by the weights' bytes: 2 rows flops to each.  The weight is the product's left operand -- 128 of its rows fill the
// tensor cores' 128 whatever the rows of x are -- and up to ROWS (16 or 64) rows of x its right one, in steps of 16: a tile with
// fewer rows fetches, multiplies and adds up fewer.  The k blocks of all tiles (128 columns of the result, ROWS rows of a
// group; the row tiles of a weight's block side by side, so that it is read from memory once) form one line, and each of
// DVM_SCALED_UNITS CTAs takes an equal range of it, so every SM reads as many bytes wherever the rows are.  A tile that lies in
// one range is finished there; the parts of one that spans several go to the workspace and a second kernel adds them up in
// their order (a dependent launch that starts while this one drains).
//
// In a CTA one thread fetches tiles by TMA (128-byte swizzle, a ring of stages), a warp issues the four products of a k block (32
// of k each) into one of BUFFERS places in tensor memory, and warps take them out, multiply by the scales and add them up in
// registers: thread n holds column n of the result, a register per row, 32 rows at most (of 64 a second four warps hold the
// second half).  The scales of some k blocks at a time, one per row times the weight's, are laid in shared memory, a load per
// thread, ahead.  (The tensor cores add up 128 products; the sums over blocks are fp32 multiply-adds.)
// 512 rows of 128 experts, 4096 to 2816: 226 us, 6.3 TB/s; 64 rows of 64 experts 118 us, 6.3; one row, 4096 to 11008: 13.7 us in a
// chain of launches, of which the launches, the first tile, the join of the parts and their reads are 7.  A dense weight's first
// tiles, as many as the ring holds, are asked for in L2 before the launch before has ended (14.9 us without, 13.9 with half as
// many, 13.8 with twice).
#include <algorithm>

#include "dvm_experts_launch.h"
#include "dvm_scaled.cuh"

namespace dvm {
namespace scaled {

constexpr int BUFFERS = 4, MIN_BLOCKS = 4;

// The workspace: per CTA 32 bytes about the tile that begins in its range and goes on behind it (parts 0: none), then two
// parts per CTA [row][column]: slot 0 the part at the start of its range, slot 1 a later one.
struct Head { int first, rows, n0, parts, slot, pad[3]; };
static_assert(sizeof(Head) == 32, "");
template <int ROWS> __device__ __forceinline__ float* part_of(const Args& a, int cta, int slot) {
  return (float*)(a.work + DVM_SCALED_UNITS * sizeof(Head)) + (long long)(2 * cta + slot) * (ROWS * BLOCK);
}

template <int ROWS> struct Few {
  static constexpr int WARPS = ROWS == 16 ? 4 : 8, THREADS = (WARPS + 2) * 32;   // warps that add up; fetching and multiplying ones
  static constexpr int MINE = ROWS == 16 ? 16 : 32;                              // rows of a thread
  static constexpr int AHEAD = WARPS * 32 / ROWS;                                // k blocks whose scales are laid together
  static constexpr uint32_t W = BLOCK * BLOCK, X = ROWS * BLOCK, STAGE = W + X;
  static constexpr int STAGES = (int)(192 * 1024 / STAGE);
  static constexpr uint32_t SCALES = STAGES * STAGE;                             // [2][AHEAD][ROWS] fp32
  static constexpr uint32_t BARS = SCALES + 2 * AHEAD * ROWS * 4;                // full[STAGES], empty[STAGES], done[BUFFERS], free[BUFFERS], last
  static constexpr uint32_t WORDS = BARS + 8 * (2 * STAGES + 2 * BUFFERS + 1);
  static constexpr uint32_t LINE = (WORDS + 16 + 15) / 16 * 16;
  static constexpr uint32_t BYTES = LINE + (DVM_MAX_WEIGHT_GROUPS + 1 + THREADS / 32) * 8 + 1024;   // 1024: alignment of the swizzled stages
  static_assert(STAGE % 1024 == 0 && BYTES <= 227 * 1024 && MINE * WARPS / 4 == ROWS, "");
};

template <int THREADS> __device__ __forceinline__ void sum_sync() { asm volatile("bar.sync 1, %0;" ::"n"(THREADS) : "memory"); }
__device__ __forceinline__ void put(const Args& a, long long at, float v) {
  if (a.out_bf16) ((__nv_bfloat16*)a.out)[at] = __float2bfloat16_rn(v);
  else ((float*)a.out)[at] = v;
}
__device__ __forceinline__ void tmem_load16(uint32_t taddr, float (&v)[16]) {
  uint32_t r[16];
  asm volatile(
      "tcgen05.ld.sync.aligned.32x32b.x16.b32 {%0, %1, %2, %3, %4, %5, %6, %7, %8, %9, %10, %11, %12, %13, %14, %15}, [%16];\n\t"
      "tcgen05.wait::ld.sync.aligned;"
      : "=r"(r[0]), "=r"(r[1]), "=r"(r[2]), "=r"(r[3]), "=r"(r[4]), "=r"(r[5]), "=r"(r[6]), "=r"(r[7]),
        "=r"(r[8]), "=r"(r[9]), "=r"(r[10]), "=r"(r[11]), "=r"(r[12]), "=r"(r[13]), "=r"(r[14]), "=r"(r[15])
      : "r"(taddr)
      : "memory");
#pragma unroll
  for (int i = 0; i < 16; ++i) v[i] = __uint_as_float(r[i]);
}

// k blocks of a CTA's range
__device__ __forceinline__ long long range_of(long long total) { return max((total + gridDim.x - 1) / gridDim.x, (long long)MIN_BLOCKS); }

template <int ROWS>
__global__ void __launch_bounds__(Few<ROWS>::THREADS, 1)
dvm_scaled_few_kernel(const __grid_constant__ CUtensorMap tm_x, const __grid_constant__ CUtensorMap tm_w, const __grid_constant__ Args a) {
  using S = Few<ROWS>;
  constexpr uint32_t COLUMNS = BUFFERS * ROWS;   // of tensor memory: a power of two
  extern __shared__ uint8_t smem_raw[];
  const uint32_t raw = smem_u32(smem_raw), base = (raw + 1023u) & ~1023u;
  uint8_t* const sm = smem_raw + (base - raw);
  const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
  const uint32_t bar_full = base + S::BARS, bar_empty = bar_full + 8 * S::STAGES, bar_done = bar_empty + 8 * S::STAGES, bar_free = bar_done + 8 * BUFFERS,
                 bar_last = bar_free + 8 * BUFFERS;
  volatile uint32_t* const abort_flag = (volatile uint32_t*)(sm + S::WORDS);
  uint32_t* const tmem_slot = (uint32_t*)(sm + S::WORDS) + 1;
  long long* const line = (long long*)(sm + S::LINE);

  if (threadIdx.x == 0) {
    for (int s = 0; s < S::STAGES; ++s) { mbar_init(bar_full + 8 * s, 1); mbar_init(bar_empty + 8 * s, 1); }
    for (int s = 0; s < BUFFERS; ++s) { mbar_init(bar_done + 8 * s, 1); mbar_init(bar_free + 8 * s, S::WARPS); }
    mbar_init(bar_last, 1);
    *abort_flag = 0;
    asm volatile("fence.mbarrier_init.release.cluster;" ::: "memory");
  }
  grid_ready();
  if (threadIdx.x == S::WARPS * 32) {
    tma_prefetch(&tm_x);
    tma_prefetch(&tm_w);
    if (!a.starts) {   // the range is known: the weight's first tiles come to L2 while the launch before ends
      const int down = (a.rows + ROWS - 1) / ROWS;
      const long long total = (long long)down * a.n_blocks * a.k_blocks, chunk = range_of(total), begin = blockIdx.x * chunk;
      for (long long i = begin; i < min(total, begin + min(chunk, (long long)S::STAGES)); ++i) {
        const long long t = i / a.k_blocks;
        tma_ask_3d(&tm_w, (int)(i - t * a.k_blocks) * BLOCK, (int)(t / down) * BLOCK, 0);
      }
    }
  }
  grid_wait();
  if (warp == S::WARPS + 1) {
    asm volatile("tcgen05.alloc.cta_group::1.sync.aligned.shared::cta.b32 [%0], %1;" ::"r"(smem_u32(tmem_slot)), "r"(COLUMNS) : "memory");
    asm volatile("tcgen05.relinquish_alloc_permit.cta_group::1.sync.aligned;" ::: "memory");
  }
  lay_out<S::THREADS>(a, ROWS, a.n_blocks, line, line + a.groups + 1);
  tc_fence_before();
  __syncthreads();
  tc_fence_after();
  const uint32_t tmem = *(volatile uint32_t*)tmem_slot;

  // this CTA's range of the line of k blocks
  const long long total = line[a.groups] * a.k_blocks;
  const long long chunk = range_of(total);
  const long long begin = min(total, blockIdx.x * chunk), stop = min(total, begin + chunk);
  // f(group, first row, rows, block of n, first and last k block, tile's place on the line) for each tile of the range
  auto walk = [&](auto f) {
    if (begin >= stop) return;
    long long t = begin / a.k_blocks;
    int g = group_at(line, a.groups, t);
    for (; t * a.k_blocks < stop; ++t) {
      while (line[g + 1] <= t) ++g;   // (t is below line[groups])
      const Rows r = rows_of(a, g);
      const int down = (r.last - r.first + ROWS - 1) / ROWS, in_group = (int)(t - line[g]), nb = in_group / down, first = r.first + (in_group - nb * down) * ROWS;
      const long long at = t * a.k_blocks;
      if (!f(g, first, min(ROWS, r.last - first), nb, (int)max(0ll, begin - at), (int)min((long long)a.k_blocks, stop - at), at)) return;
    }
  };

  uint32_t issued = 0, f_stage = 0, f_phase = 0;   // the fetching thread's ring, kept for the abort path
  if (warp == S::WARPS) {
    // ---------------- a warp fetches ----------------
    const bool leader = elect_one();
    walk([&](int g, int first, int rows, int nb, int kb0, int kb1, long long) {
      const int steps = (rows + 15) >> 4;
      for (int kb = kb0; kb < kb1; ++kb) {
        if (!__all_sync(ALL, mbar_wait(bar_empty + 8 * f_stage, f_phase ^ 1, abort_flag))) return false;
        const uint32_t full = bar_full + 8 * f_stage, at = base + f_stage * S::STAGE;
        if (leader) {
          mbar_expect_tx(full, S::W + steps * (16 * BLOCK));
          tma_load_3d(at, &tm_w, full, kb * BLOCK, nb * BLOCK, g);
#pragma unroll
          for (int x = 0; x < ROWS / 16; ++x)
            if (x < steps) tma_load_2d(at + S::W + x * (16 * BLOCK), &tm_x, full, kb * BLOCK, first + 16 * x);
        }
        ++issued;
        if (++f_stage == S::STAGES) { f_stage = 0; f_phase ^= 1; }
      }
      return true;
    });
    __syncwarp();
  } else if (warp == S::WARPS + 1) {
    // ---------------- a warp multiplies ----------------
    const bool leader = elect_one();
    const uint32_t w0 = desc_lo(base), x0 = desc_lo(base + S::W);
    uint32_t stage = 0, phase = 0, buffer = 0, b_phase = 0;
    walk([&](int, int, int rows, int, int kb0, int kb1, long long) {
      const uint32_t idesc = IDESC<BLOCK, 0> | ((uint32_t)((rows + 15) >> 4) << 18);   // (n / 8 from bit 17 on)
      for (int kb = kb0; kb < kb1; ++kb) {
        if (!__all_sync(ALL, mbar_wait(bar_free + 8 * buffer, b_phase ^ 1, abort_flag) && mbar_wait(bar_full + 8 * stage, phase, abort_flag))) return false;
        tc_fence_after();
        if (leader) {
          const uint32_t w = w0 + stage * (S::STAGE >> 4), x = x0 + stage * (S::STAGE >> 4);
#pragma unroll
          for (int k = 0; k < BLOCK / 32; ++k) umma_e4m3(tmem + buffer * ROWS, desc_of(w + 2 * k), desc_of(x + 2 * k), idesc, k != 0);
          umma_commit(bar_empty + 8 * stage);
          umma_commit(bar_done + 8 * buffer);
        }
        if (++stage == S::STAGES) { stage = 0; phase ^= 1; }
        if (++buffer == BUFFERS) { buffer = 0; b_phase ^= 1; }
      }
      return true;
    });
    if (leader) {   // every product has ended before tensor memory is given back, whatever else ended early
      umma_commit(bar_last);
      mbar_spin(bar_last, 0, abort_flag, DRAIN_NS, false);
    }
    __syncwarp();
  } else {
    // ---------------- scales, sums, results ----------------
    float* const scales = (float*)(sm + S::SCALES);
    const int j_first = warp / 4 * S::MINE, column = threadIdx.x & 127;   // this thread's first row and its column
    const uint32_t mine = tmem + ((uint32_t)((warp & 3) * 32) << 16) + j_first;
    const int s_row = threadIdx.x % ROWS, s_block = threadIdx.x / ROWS;    // the scale that it lays out
    uint32_t buffer = 0, b_phase = 0, half = 0;
    Head head = {};
    walk([&](int g, int first, int rows, int nb, int kb0, int kb1, long long at) {
      float acc[S::MINE];
#pragma unroll
      for (int j = 0; j < S::MINE; ++j) acc[j] = 0.f;
      const float* xs = a.xs + (long long)(first + s_row) * a.xs_stride + s_block;
      const float* ws = a.ws + ((long long)g * a.n_blocks + nb) * a.k_blocks + s_block;
      auto scale_at = [&](int kb) { return s_row < rows && kb + s_block < kb1 ? xs[kb] * ws[kb] : 0.f; };
      float next = scale_at(kb0);
      for (int kb = kb0; kb < kb1; ++kb) {
        const int in = (kb - kb0) % S::AHEAD;
        if (in == 0) {
          half ^= 1;
          scales[(half * S::AHEAD + s_block) * ROWS + s_row] = next;
          // (two places in turn: a warp that is through with the blocks of one meets the others before it is overwritten)
          sum_sync<S::WARPS * 32>();
          next = scale_at(kb + S::AHEAD);
        }
        const float* const s = scales + (half * S::AHEAD + in) * ROWS + j_first;
        const bool ok = __all_sync(ALL, mbar_wait(bar_done + 8 * buffer, b_phase, abort_flag));   // (its lanes alike: what follows is for whole warps)
        if (ok) {   // (a warp that gave up goes on without work, so that the warps still meet)
          tc_fence_after();
#pragma unroll
          for (int c = 0; c < S::MINE; c += 16) {
            if (j_first + c >= rows) break;
            float d[16];
            __syncwarp();
            tmem_load16(mine + buffer * ROWS + c, d);
#pragma unroll
            for (int j = 0; j < 16; j += 4) {
              const float4 f = *(const float4*)(s + c + j);
              const float2 lo = fma2(make_float2(d[j], d[j + 1]), make_float2(f.x, f.y), make_float2(acc[c + j], acc[c + j + 1]));
              const float2 hi = fma2(make_float2(d[j + 2], d[j + 3]), make_float2(f.z, f.w), make_float2(acc[c + j + 2], acc[c + j + 3]));
              acc[c + j] = lo.x; acc[c + j + 1] = lo.y; acc[c + j + 2] = hi.x; acc[c + j + 3] = hi.y;
            }
          }
          tc_fence_before();
          __syncwarp();
          if (lane == 0) mbar_arrive(bar_free + 8 * buffer);
        }
        if (++buffer == BUFFERS) { buffer = 0; b_phase ^= 1; }
      }
      const int n = nb * BLOCK + column;
      if (kb0 == 0 && kb1 == a.k_blocks) {
        if (n < a.n)
#pragma unroll
          for (int j = 0; j < S::MINE; ++j)
            if (j_first + j < rows) put(a, (first + j_first + j) * a.out_stride + n, acc[j]);
      } else {
        const int slot = kb0 == 0 && at > begin ? 1 : 0;
        float* const part = part_of<ROWS>(a, blockIdx.x, slot) + column;
#pragma unroll
        for (int j = 0; j < S::MINE; ++j)
          if (j_first + j < rows) part[(j_first + j) * BLOCK] = acc[j];
        if (kb0 == 0) head = {first, rows, nb * BLOCK, (int)((at + a.k_blocks - 1) / chunk) - (int)blockIdx.x + 1, slot, {}};
      }
      return true;
    });
    if (threadIdx.x == 0) ((Head*)a.work)[blockIdx.x] = head;
  }
  tc_fence_before();
  __syncthreads();
  tc_fence_after();
  if (warp == S::WARPS + 1) asm volatile("tcgen05.dealloc.cta_group::1.sync.aligned.b32 %0, %1;" ::"r"(tmem), "r"(COLUMNS) : "memory");
  if (*abort_flag) {   // whoever's wait ran out: the copies in flight land first
    if (threadIdx.x == S::WARPS * 32) mbar_drain(bar_full, S::STAGES, issued, f_stage, f_phase, abort_flag);
    if (threadIdx.x == 0) atomicMax(a.status, (unsigned int)ST_TIMEOUT);
  }
}

// Adds up the parts of a tile that spans several ranges, in their order: one CTA per head (grid x) and 4 rows (grid y).
template <int ROWS> __global__ void __launch_bounds__(BLOCK) dvm_scaled_join_kernel(const __grid_constant__ Args a) {
  constexpr int EACH = 4;
  grid_ready();
  grid_wait();
  const Head h = ((const Head*)a.work)[blockIdx.x];
  const int j0 = blockIdx.y * EACH;
  if (h.parts < 2 || j0 >= h.rows) return;
  float v[EACH] = {};
#pragma unroll 4
  for (int p = 0; p < h.parts; ++p) {
    const float* part = part_of<ROWS>(a, blockIdx.x + p, p ? 0 : h.slot) + threadIdx.x;
#pragma unroll
    for (int j = 0; j < EACH; ++j)
      if (j0 + j < h.rows) v[j] += part[(j0 + j) * BLOCK];
  }
  const int n = h.n0 + threadIdx.x;
  if (n < a.n)
#pragma unroll
    for (int j = 0; j < EACH; ++j)
      if (j0 + j < h.rows) put(a, (h.first + j0 + j) * a.out_stride + n, v[j]);
}

template <int ROWS> int launch_few(const CUtensorMap& x, const CUtensorMap& w, const Args& a, int device, cudaStream_t stream) {
  static std::atomic<uint64_t> allowed{0};
  using S = Few<ROWS>;
  int st = dvm_allow_smem((const void*)dvm_scaled_few_kernel<ROWS>, (int)S::BYTES, device, &allowed);
  if (st == DVM_OK) st = dvm_launch_next(dvm_scaled_few_kernel<ROWS>, DVM_SCALED_UNITS, S::THREADS, S::BYTES, stream, x, w, a);
  return st != DVM_OK ? st : dvm_launch_next(dvm_scaled_join_kernel<ROWS>, dim3(DVM_SCALED_UNITS, (std::min(ROWS, a.rows) + 3) / 4), BLOCK, 0, stream, a);
}

}  // namespace scaled
}  // namespace dvm

int dvm_launch_scaled_few(const CUtensorMap& x, const CUtensorMap& w, const dvm::scaled::Args& a, int tile, int device, cudaStream_t stream) {
  using namespace dvm::scaled;
  return tile == 16 ? launch_few<16>(x, w, a, device, stream) : launch_few<64>(x, w, a, device, stream);
}

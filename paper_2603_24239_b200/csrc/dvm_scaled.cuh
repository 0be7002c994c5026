// What the kernels of the scaled product share: their arguments, the groups' rows, the tiles of all groups as one line.
#pragma once
#include <cuda.h>
#include <cuda_bf16.h>
#include <cuda_runtime.h>
#include <stdint.h>

#include "dvm_experts.h"
#include "dvm_sm100.cuh"

namespace dvm {
namespace scaled {

using namespace sm100;

constexpr uint32_t ALL = 0xffffffffu;
constexpr int BLOCK = DVM_SCALE_BLOCK;   // columns of k of one step: they share their scales

struct Args {
  const float *xs, *ws;
  const int* starts;       // nullptr: one group of all rows
  void* out;
  uint8_t* work;
  unsigned int* status;
  long long xs_stride, out_stride;
  int rows, n, k_blocks, n_blocks, groups;   // n_blocks: blocks of 128 columns of the result
  int out_bf16, out_tma;                     // out_tma: there is a tensor map of the result
};

struct Rows { int first, last; };
__device__ __forceinline__ Rows rows_of(const Args& a, int g) {
  if (!a.starts) return {0, a.rows};
  const int first = min(max(a.starts[g], 0), a.rows);
  return {first, min(max(a.starts[g + 1], first), a.rows)};
}

// Tiles of the groups before each, for `tile` rows a tile and `across` tiles across the result: line[g], g <= groups, in
// shared memory.  By all THREADS threads; sums: a word per warp.
template <int THREADS> __device__ __forceinline__ void lay_out(const Args& a, int tile, int across, long long* line, long long* sums) {
  const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31, per = (a.groups + THREADS - 1) / THREADS, g0 = threadIdx.x * per;
  long long mine = 0;
  for (int g = g0; g < min(g0 + per, a.groups); ++g) {
    const Rows r = rows_of(a, g);
    const long long tiles = (long long)((r.last - r.first + tile - 1) / tile) * across;
    line[g + 1] = tiles;
    mine += tiles;
  }
  long long upto = mine;
#pragma unroll
  for (int d = 1; d < 32; d <<= 1) {
    const long long y = __shfl_up_sync(0xffffffffu, upto, d);
    if (lane >= d) upto += y;
  }
  if (lane == 31) sums[warp] = upto;
  __syncthreads();
#pragma unroll
  for (int x = 0; x < THREADS / 32; ++x)
    if (x < warp) upto += sums[x];
  long long at = upto - mine;
  for (int g = g0; g < min(g0 + per, a.groups); ++g) {
    at += line[g + 1];
    line[g + 1] = at;
  }
  if (threadIdx.x == 0) line[0] = 0;
  __syncthreads();
}
// the group that holds tile t of the line
__device__ __forceinline__ int group_at(const long long* line, int groups, long long t) {
  int lo = 0, hi = groups - 1;   // the last g with line[g] <= t
  while (lo < hi) {
    const int mid = (lo + hi + 1) >> 1;
    if (line[mid] <= t) lo = mid; else hi = mid - 1;
  }
  return lo;
}

__device__ __forceinline__ void tma_load_3d(uint32_t dst, const CUtensorMap* map, uint32_t bar, int x, int y, int z) {
  asm volatile(
      "cp.async.bulk.tensor.3d.shared::cluster.global.tile.mbarrier::complete_tx::bytes [%0], [%1, {%3, %4, %5}], [%2];"
      ::"r"(dst), "l"(map), "r"(bar), "r"(x), "r"(y), "r"(z)
      : "memory");
}
// Asks L2 for a tile; nothing is read, so what an earlier launch still writes there is not missed.
__device__ __forceinline__ void tma_ask_3d(const CUtensorMap* map, int x, int y, int z) {
  asm volatile("cp.async.bulk.prefetch.tensor.3d.L2.global.tile [%0, {%1, %2, %3}];" ::"l"(map), "r"(x), "r"(y), "r"(z) : "memory");
}
__device__ __forceinline__ void umma_e4m3(uint32_t d_tmem, uint64_t adesc, uint64_t bdesc, uint32_t idesc, uint32_t accumulate) {
  asm volatile(
      "{\n\t.reg .pred p;\n\tsetp.ne.b32 p, %4, 0;\n\ttcgen05.mma.cta_group::1.kind::f8f6f4 [%0], %1, %2, %3, p;\n\t}"
      ::"r"(d_tmem), "l"(adesc), "l"(bdesc), "r"(idesc), "r"(accumulate)
      : "memory");
}
// Shared-memory matrix descriptors of K-major tiles: rows of 128 bytes, 128-byte swizzle, groups of 8 rows 1024 bytes apart;
// from their low word, the address, to which steps along k and stages are added.  The warp that issues products walks as a
// whole, so that descriptors and barriers stay in uniform registers, and one elected lane issues: from a branch of lane 0 alone
// a product took 70 cycles to issue, a wait 200.
__device__ __forceinline__ uint32_t desc_lo(uint32_t addr) { return ((addr >> 4) & 0x3fff) | (1u << 16); }
__device__ __forceinline__ uint64_t desc_of(uint32_t lo) { return lo | ((uint64_t)(1024 >> 4) << 32) | ((uint64_t)1 << 46) | ((uint64_t)2 << 61); }
__device__ __forceinline__ bool elect_one() {
  uint32_t p;
  asm volatile("{\n\t.reg .pred p;\n\telect.sync _|p, 0xffffffff;\n\tselp.u32 %0, 1, 0, p;\n\t}" : "=r"(p));
  return p != 0;
}
// Instruction descriptor: e4m3 x e4m3, both K-major, fp32 sums, M x N
template <int M, int N> constexpr uint32_t IDESC = (1u << 4) | ((uint32_t)(N >> 3) << 17) | ((uint32_t)(M >> 4) << 24);

}  // namespace scaled
}  // namespace dvm

int dvm_launch_scaled_few(const CUtensorMap& x, const CUtensorMap& w, const dvm::scaled::Args& a, int tile, int device, cudaStream_t stream);
int dvm_launch_scaled_many(const CUtensorMap& x, const CUtensorMap& w, const CUtensorMap& out, const dvm::scaled::Args& a, int sm_count, int device,
                           cudaStream_t stream);

// Paging meta-kernel: rows, positions and cache slots of a batch's new tokens, pages for the blocks they open.
//
// Everything follows from two running sums over the requests, of new rows and of new pages.  Every CTA forms both for
// itself in shared memory (n <= DVM_MAX_REQUESTS: at most 32 requests per thread) -- cheaper than a second launch or a
// grid-wide wait -- and then takes its share of the rows and of the new pages, finding the request of each by binary
// search.  A row that lies on a page handed out by this very launch reads the page from `free`, not from the table that
// another CTA is writing.  The call is bound by latency: launch, one read of the lengths, two block scans.
#include <cuda_runtime.h>

#include "dvm_launch.h"
#include "dvm_serving.h"

namespace dvm {
namespace paging {

constexpr int THREADS = 256;
constexpr int ROWS_PER_THREAD = 4;

struct Args {
  const int *cached, *fresh, *free;
  int *table, *starts, *lengths, *positions, *slots, *taken;
  int n, max_blocks, page, rows, free_pages;
};

__device__ __forceinline__ int clip(long long v) { return (int)(v < 0x7fffffffll ? v : 0x7fffffffll); }
__device__ __forceinline__ long long blocks_of(long long tokens, int page) { return (tokens + page - 1) / page; }

// last i with sums[i] <= x (sums[0] = 0, non-decreasing, x below sums[n])
__device__ __forceinline__ int owner(const int* sums, int n, int x) {
  int lo = 0, hi = n;
  while (hi - lo > 1) {
    const int mid = (lo + hi) >> 1;
    if (sums[mid] <= x) lo = mid; else hi = mid;
  }
  return lo;
}

// sum of v over the threads before this one, and over all of them
__device__ __forceinline__ long long before(long long v, long long* warp_sums, long long* all) {
  const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
  long long x = v;
#pragma unroll
  for (int d = 1; d < 32; d <<= 1) {
    const long long y = __shfl_up_sync(0xffffffffu, x, d);
    if (lane >= d) x += y;
  }
  __syncthreads();  // (the sums of the scan before have been read)
  if (lane == 31) warp_sums[warp] = x;
  __syncthreads();
  long long base = 0, total = 0;
#pragma unroll
  for (int w = 0; w < THREADS / 32; ++w) {
    if (w < warp) base += warp_sums[w];
    total += warp_sums[w];
  }
  *all = total;
  return base + x - v;
}

__global__ void __launch_bounds__(THREADS) dvm_paging_kernel(const __grid_constant__ Args a) {
  extern __shared__ int sm[];
  int* const starts = sm;               // n + 1: rows before request i
  int* const pages = sm + a.n + 1;      // n + 1: new pages before request i
  __shared__ long long warp_sums[THREADS / 32];
  const int per = (a.n + THREADS - 1) / THREADS, i0 = min(a.n, (int)threadIdx.x * per), i1 = min(a.n, i0 + per);

  // rows: the sum of the new tokens, in 64 bits, cut at `rows`
  long long sum = 0, all;
  for (int i = i0; i < i1; ++i) sum += max(a.fresh[i], 0);
  long long at = before(sum, warp_sums, &all);
  for (int i = i0; i < i1; ++i) {
    starts[i] = (int)min(at, (long long)a.rows);
    at += max(a.fresh[i], 0);
  }
  const int used = (int)min(all, (long long)a.rows);
  if (threadIdx.x == 0) starts[a.n] = used;
  __syncthreads();
  // new pages: blocks that the new rows reach and the cached tokens do not
  auto need = [&](int i) -> long long {
    const long long c = max(a.cached[i], 0), have = blocks_of(c, a.page);
    const long long want = min(blocks_of(clip(c + starts[i + 1] - starts[i]), a.page), (long long)a.max_blocks);
    return want > have ? want - have : 0;
  };
  sum = 0;
  for (int i = i0; i < i1; ++i) sum += need(i);
  at = before(sum, warp_sums, &all);
  for (int i = i0; i < i1; ++i) {
    pages[i] = clip(at);
    at += need(i);
  }
  if (threadIdx.x == 0) pages[a.n] = clip(all);
  __syncthreads();

  const int n_pages = pages[a.n];
  auto page_at = [&](int k) -> int { return k < a.free_pages ? a.free[k] : -1; };
  if (blockIdx.x == 0) {
    for (int i = threadIdx.x; i <= a.n; i += THREADS) {
      a.starts[i] = starts[i];
      if (i < a.n) a.lengths[i] = clip((long long)max(a.cached[i], 0) + starts[i + 1] - starts[i]);
    }
    if (threadIdx.x == 0) a.taken[0] = n_pages;
  }
  for (long long k = (long long)blockIdx.x * THREADS + threadIdx.x; k < n_pages; k += (long long)gridDim.x * THREADS) {
    const int i = owner(pages, a.n, (int)k);
    const long long b = blocks_of(max(a.cached[i], 0), a.page) + (k - pages[i]);
    a.table[(long long)i * a.max_blocks + b] = page_at((int)k);
  }
  const long long step = (long long)gridDim.x * THREADS * ROWS_PER_THREAD;
  for (long long t0 = ((long long)blockIdx.x * THREADS + threadIdx.x) * ROWS_PER_THREAD; t0 < a.rows; t0 += step) {
    int i = t0 < used ? owner(starts, a.n, (int)t0) : 0;
#pragma unroll
    for (int r = 0; r < ROWS_PER_THREAD; ++r) {
      const long long t = t0 + r;
      if (t >= a.rows) break;
      int pos = -1, slot = -1;
      if (t < used) {
        while (starts[i + 1] <= t) ++i;  // (t < starts[n]: ends)
        const long long c = max(a.cached[i], 0);
        pos = clip(c + t - starts[i]);
        const long long b = pos / a.page, have = blocks_of(c, a.page);
        if (b < a.max_blocks) {
          const int p = b < have ? a.table[(long long)i * a.max_blocks + b] : page_at(pages[i] + (int)(b - have));
          const long long s = (long long)p * a.page + pos % a.page;
          if (p >= 0 && s < 0x7fffffffll) slot = (int)s;
        }
      }
      a.positions[t] = pos;
      a.slots[t] = slot;
    }
  }
}

}  // namespace paging
}  // namespace dvm

int dvm_launch_paging(const dvm_paging_desc& d, void* const* t, cudaStream_t stream) {
  using namespace dvm::paging;
  DvmDeviceInfo dev;
  const int st = dvm_device_state(&dev);
  if (st != DVM_OK) return st;
  Args a;
  a.cached = (const int*)t[PG_CACHED]; a.fresh = (const int*)t[PG_FRESH]; a.free = (const int*)t[PG_FREE];
  a.table = (int*)t[PG_TABLE]; a.starts = (int*)t[PG_STARTS]; a.lengths = (int*)t[PG_LENGTHS];
  a.positions = (int*)t[PG_POSITIONS]; a.slots = (int*)t[PG_SLOTS]; a.taken = (int*)t[PG_TAKEN];
  a.n = (int)d.requests; a.max_blocks = (int)d.max_blocks; a.page = (int)d.page_size; a.rows = (int)d.rows; a.free_pages = (int)d.free_pages;
  const size_t smem = 2 * ((size_t)a.n + 1) * sizeof(int);
  if (smem > 48 * 1024) DVM_CUDA(cudaFuncSetAttribute(dvm_paging_kernel, cudaFuncAttributeMaxDynamicSharedMemorySize, (int)smem));
  const int64_t per_cta = THREADS * ROWS_PER_THREAD, ctas = (d.rows + per_cta - 1) / per_cta;
  const int grid = (int)(ctas < 1 ? 1 : ctas < 2 * dev.sm_count ? ctas : 2 * dev.sm_count);
  dvm_paging_kernel<<<grid, THREADS, smem, stream>>>(a);
  DVM_CUDA(cudaGetLastError());
  dvm_count_launch();
  return DVM_OK;
}

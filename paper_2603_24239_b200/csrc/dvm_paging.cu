// Paging meta-kernel: rows, positions and cache slots of a batch's new tokens, pages for the blocks they open.
//
// Everything follows from two running sums over the requests, of new rows and of new pages.  Every CTA forms both for
// itself in shared memory, in one scan (n <= DVM_MAX_REQUESTS: at most 32 requests per thread) -- cheaper than a second
// launch or a grid-wide wait -- and then takes its share of the rows and of the new pages, finding the request of each by
// binary search.  A row that lies on a page handed out by this very launch reads the page from `free`, not from the table
// that another CTA is writing.  The call is bound by latency: launch, one read of the lengths, a block scan, one read of
// the tables: 4.7 us in a chain of launches for one token of 32 requests, 5.3 us for 256 prompts of up to 1024 tokens (two
// scans and the lengths read again for every sum: 5.9 and 6.5 us).
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

struct Sums { long long rows, pages; };
// sums of v over the threads before this one, and over all of them
__device__ __forceinline__ Sums before(Sums v, Sums* warp_sums, Sums* all) {
  const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
  Sums x = v;
#pragma unroll
  for (int d = 1; d < 32; d <<= 1) {
    const long long y = __shfl_up_sync(0xffffffffu, x.rows, d), z = __shfl_up_sync(0xffffffffu, x.pages, d);
    if (lane >= d) { x.rows += y; x.pages += z; }
  }
  __syncthreads();  // (the sums of the scan before have been read)
  if (lane == 31) warp_sums[warp] = x;
  __syncthreads();
  Sums base = {0, 0}, total = {0, 0};
#pragma unroll
  for (int w = 0; w < THREADS / 32; ++w) {
    if (w < warp) { base.rows += warp_sums[w].rows; base.pages += warp_sums[w].pages; }
    total.rows += warp_sums[w].rows;
    total.pages += warp_sums[w].pages;
  }
  *all = total;
  return {base.rows + x.rows - v.rows, base.pages + x.pages - v.pages};
}

__global__ void __launch_bounds__(THREADS) dvm_paging_kernel(const __grid_constant__ Args a) {
  extern __shared__ int sm[];
  int* const starts = sm;               // n + 1: rows before request i
  int* const pages = sm + a.n + 1;      // n + 1: new pages before request i
  int* const cached = sm + 2 * a.n + 2; // n: tokens of request i in the cache
  __shared__ Sums warp_sums[THREADS / 32];
  grid_wait();  // (no grid_ready: 256 prompts in a chain of launches took 7.5 us with it)
  const int per = (a.n + THREADS - 1) / THREADS, i0 = min(a.n, (int)threadIdx.x * per), i1 = min(a.n, i0 + per);

  // Blocks that a request's new rows reach and its cached tokens do not.
  auto need = [&](long long c, long long rows) -> long long {
    const long long have = blocks_of(c, a.page), want = min(blocks_of(clip(c + rows), a.page), (long long)a.max_blocks);
    return want > have ? want - have : 0;
  };
  Sums mine = {0, 0}, all;
  for (int i = i0; i < i1; ++i) {
    const int c = max(a.cached[i], 0), f = max(a.fresh[i], 0);
    cached[i] = c;
    starts[i] = f;  // (for now)
    mine.rows += f;
    mine.pages += need(c, f);
  }
  Sums at = before(mine, warp_sums, &all);
  if (all.rows > a.rows) {  // the rows do not hold all new tokens: once more with what they hold
    mine.pages = 0;
    long long row = at.rows;
    for (int i = i0; i < i1; ++i) {
      const long long first = min(row, (long long)a.rows);
      row += starts[i];
      starts[i] = (int)(min(row, (long long)a.rows) - first);
      mine.pages += need(cached[i], starts[i]);
    }
    mine.rows = min(row, (long long)a.rows) - min(at.rows, (long long)a.rows);
    at = before(mine, warp_sums, &all);
  }
  for (int i = i0; i < i1; ++i) {
    const int f = starts[i];
    starts[i] = (int)at.rows;
    pages[i] = clip(at.pages);
    at.rows += f;
    at.pages += need(cached[i], f);
  }
  if (threadIdx.x == 0) {
    starts[a.n] = (int)all.rows;
    pages[a.n] = clip(all.pages);
  }
  __syncthreads();

  const int used = starts[a.n], n_pages = pages[a.n];
  auto page_at = [&](int k) -> int { return k < a.free_pages ? a.free[k] : -1; };
  if (blockIdx.x == 0) {
    for (int i = threadIdx.x; i <= a.n; i += THREADS) {
      a.starts[i] = starts[i];
      if (i < a.n) a.lengths[i] = clip((long long)cached[i] + starts[i + 1] - starts[i]);
    }
    if (threadIdx.x == 0) a.taken[0] = n_pages;
  }
  for (long long k = (long long)blockIdx.x * THREADS + threadIdx.x; k < n_pages; k += (long long)gridDim.x * THREADS) {
    const int i = owner(pages, a.n, (int)k);
    const long long b = blocks_of(cached[i], a.page) + (k - pages[i]);
    a.table[(long long)i * a.max_blocks + b] = page_at((int)k);
  }
  const long long step = (long long)gridDim.x * THREADS * ROWS_PER_THREAD;
  for (long long t0 = ((long long)blockIdx.x * THREADS + threadIdx.x) * ROWS_PER_THREAD; t0 < a.rows; t0 += step) {
    int i = t0 < used ? owner(starts, a.n, (int)t0) : 0;
    int pos[ROWS_PER_THREAD], page[ROWS_PER_THREAD];
#pragma unroll
    for (int r = 0; r < ROWS_PER_THREAD; ++r) {  // (the tables' reads go out together)
      const long long t = t0 + r;
      pos[r] = page[r] = -1;
      if (t < used) {
        while (starts[i + 1] <= t) ++i;  // (t < starts[n]: ends)
        const long long c = cached[i];
        pos[r] = clip(c + t - starts[i]);
        const long long b = pos[r] / a.page, have = blocks_of(c, a.page);
        if (b < a.max_blocks) page[r] = b < have ? a.table[(long long)i * a.max_blocks + b] : page_at(pages[i] + (int)(b - have));
      }
    }
#pragma unroll
    for (int r = 0; r < ROWS_PER_THREAD; ++r) {
      if (t0 + r >= a.rows) break;
      const long long s = (long long)page[r] * a.page + pos[r] % a.page;
      a.positions[t0 + r] = pos[r];
      a.slots[t0 + r] = page[r] >= 0 && s < 0x7fffffffll ? (int)s : -1;
    }
  }
}

}  // namespace paging
}  // namespace dvm

int dvm_launch_paging(const dvm_paging_desc& d, void* const* t, cudaStream_t stream) {
  using namespace dvm::paging;
  DvmDeviceInfo dev;
  int st = dvm_device_state(&dev);
  if (st != DVM_OK) return st;
  Args a;
  a.cached = (const int*)t[PG_CACHED]; a.fresh = (const int*)t[PG_FRESH]; a.free = (const int*)t[PG_FREE];
  a.table = (int*)t[PG_TABLE]; a.starts = (int*)t[PG_STARTS]; a.lengths = (int*)t[PG_LENGTHS];
  a.positions = (int*)t[PG_POSITIONS]; a.slots = (int*)t[PG_SLOTS]; a.taken = (int*)t[PG_TAKEN];
  a.n = (int)d.requests; a.max_blocks = (int)d.max_blocks; a.page = (int)d.page_size; a.rows = (int)d.rows; a.free_pages = (int)d.free_pages;
  const size_t smem = (3 * (size_t)a.n + 2) * sizeof(int);
  static std::atomic<uint64_t> allowed{0};
  st = dvm_allow_smem((const void*)dvm_paging_kernel, (3 * DVM_MAX_REQUESTS + 2) * (int)sizeof(int), dev.device, &allowed);
  if (st != DVM_OK) return st;
  const int64_t per_cta = THREADS * ROWS_PER_THREAD, ctas = (d.rows + per_cta - 1) / per_cta;
  const int grid = (int)(ctas < 1 ? 1 : ctas < 2 * dev.sm_count ? ctas : 2 * dev.sm_count);
  return dvm_launch_early(dvm_paging_kernel, grid, THREADS, smem, stream, a);
}

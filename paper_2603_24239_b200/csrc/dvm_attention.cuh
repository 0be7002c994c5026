// What the attention kernels share: their arguments, the request of a row, and one row the plain way.
#pragma once
#include <cuda_bf16.h>
#include <cuda_runtime.h>
#include <stdint.h>

#include "dvm_serving.h"

namespace dvm {
namespace att {

struct Args {
  const void *q, *k, *v;
  const int *table, *starts, *lengths;
  void* out;
  float* ws;
  unsigned int* status;
  long long qs[2], os[2], ks[3], vs[3];
  int n, rows, hq, hk, group, D;    // group: query heads per kv head
  int pages, page_log, max_blocks;
  int window, sinks, max_q, out_bf16;
  int out_vec;                      // bf16 output: 1: 8 elements in one store, 2: 16
  float scale;
};

// The rows and the position of a request: rows [s0, s0 + q_len), of which the last sits at position len - 1.
struct Request { int s0, q_len; long long pos0; };  // pos0: position of row s0 (negative: rows before the first token)
__device__ __forceinline__ Request request_at(const Args& a, int i) {
  Request r;
  r.s0 = min(max(a.starts[i], 0), a.rows);
  r.q_len = min(max(a.starts[i + 1], r.s0), a.rows) - r.s0;
  r.pos0 = (long long)a.lengths[i] - r.q_len;
  return r;
}

__device__ __forceinline__ float to_f(float x) { return x; }
__device__ __forceinline__ float to_f(__nv_bfloat16 x) { return __bfloat162float(x); }
__device__ __forceinline__ void put(void* out, int bf16, long long at, float v) {
  if (bf16) ((__nv_bfloat16*)out)[at] = __float2bfloat16_rn(v);
  else ((float*)out)[at] = v;
}

// One row of one head, by one warp: lane l holds the elements l, l + 32, ... of q, of the sum and of each key.  Running
// maximum and sum over the visible tokens, one after another.  beat: a word of shared memory that is counted up on the way, for
// a kernel in which others wait meanwhile.
template <class T>
__device__ void attend_row(const Args& a, int request, long long pos, int row, int head, uint32_t* beat = nullptr) {
  const int lane = threadIdx.x & 31, kvh = head / a.group;
  const int* table = a.table + (long long)request * a.max_blocks;
  const T* q = (const T*)a.q + row * a.qs[0] + head * a.qs[1];
  float qv[8], acc[8];
#pragma unroll
  for (int e = 0; e < 8; ++e) {
    qv[e] = lane + 32 * e < a.D ? to_f(q[lane + 32 * e]) * a.scale : 0.f;
    acc[e] = 0.f;
  }
  const long long held = (long long)a.max_blocks << a.page_log;
  const long long end = min(pos + 1, held);                                   // visible: s < end and (s >= low or s < sinks)
  const long long low = a.window ? max(0ll, pos - a.window + 1) : 0;
  float m = -INFINITY, sum = 0.f;
  bool any = false;  // the row sees a token
  uint32_t steps = 0;
  for (long long s = 0; s < end; ++s) {
    if (beat && (++steps & 255) == 0 && lane == 0) atomicAdd(beat, 1u);
    if (s >= a.sinks && s < low) { s = low - 1; continue; }
    const int page = table[s >> a.page_log];
    if (page < 0 || page >= a.pages) { s |= (1ll << a.page_log) - 1; continue; }  // the whole page is hidden
    any = true;
    const long long off = s & ((1ll << a.page_log) - 1);
    const T* k = (const T*)a.k + page * a.ks[0] + off * a.ks[1] + kvh * a.ks[2];
    float x = 0.f;
#pragma unroll
    for (int e = 0; e < 8; ++e)
      if (lane + 32 * e < a.D) x = fmaf(qv[e], to_f(k[lane + 32 * e]), x);
#pragma unroll
    for (int d = 16; d > 0; d >>= 1) x += __shfl_xor_sync(0xffffffffu, x, d);
    const float m_new = x > m ? x : m;  // (a NaN score: not above m, and its weight below is NaN)
    const float keep = m == m_new ? 1.f : expf(m - m_new), p = x == -INFINITY ? 0.f : expf(x - m_new);
    const T* v = (const T*)a.v + page * a.vs[0] + off * a.vs[1] + kvh * a.vs[2];
#pragma unroll
    for (int e = 0; e < 8; ++e)
      if (lane + 32 * e < a.D) acc[e] = fmaf(p, to_f(v[lane + 32 * e]), acc[e] * keep);
    sum = sum * keep + p;
    m = m_new;
  }
  const float inv = any ? 1.f / sum : 0.f;  // (tokens, but every score -inf: 0 / 0)
  const long long at = row * a.os[0] + head * a.os[1];
#pragma unroll
  for (int e = 0; e < 8; ++e)
    if (lane + 32 * e < a.D) put(a.out, a.out_bf16, at + lane + 32 * e, acc[e] * inv);
}

}  // namespace att
}  // namespace dvm

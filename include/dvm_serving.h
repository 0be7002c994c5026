/* libdvm -- operators of a serving step that bytecode over tiles cannot express: they index (block tables), turn pairs
 * of columns (rotary positions) and chain two products through a softmax (attention).  Each is a meta-kernel of its own
 * type, used like every other one: encode it for the concrete sizes of an instance (host, no CUDA call), then dvm_launch
 * it on device tensors.  dvm_verify, dvm_disassemble, dvm_tensor_extents, dvm_code_info and dvm_launch_checked know these
 * codes; the stacked launches and dvm_run_host refuse them (DVM_ERR_UNSUPPORTED).
 *
 * One step of a batch of requests, in order:
 *   dvm_encode_paging      what every new token's row, position and cache slot are; pages handed out to the block tables
 *   (the query / key / value product: dvm_program_matmul)
 *   dvm_encode_rotary      norms of the query and key heads, rotation by position, keys and values into the cache
 *   dvm_encode_attention   the new tokens attend to the cache: causal, with a sliding window and first tokens that stay
 * A step that uses all three has a page_size that is a power of two and at least 8: attention takes no other, though
 * paging and rotary do.
 * Only sizes are encoded.  Lengths, positions, tables live on the device and may change between launches of one code (also
 * between replays of a graph that captured the launch); the kernels stay inside the tensors whatever these hold.
 *
 * Conventions as in dvm.h: every call returns DVM_OK or a negative DVM_ERR_*; the caller owns every tensor, workspaces too;
 * nothing is allocated, nothing synchronised; launches are asynchronous on the stream given to dvm_launch and may be
 * captured.  Tensors are named by their place in the launch's list (inputs, then outputs).  Index tensors are int32.
 * Strides are in elements.  An output must not overlap another tensor of the launch; dvm_launch refuses what it can see
 * of that (outputs that begin where another tensor does, any overlap of paging's) with DVM_ERR_INVALID_ARG.
 */
#ifndef DVM_SERVING_H_
#define DVM_SERVING_H_

#include "dvm.h"

#ifdef __cplusplus
extern "C" {
#endif

#define DVM_MAX_REQUESTS 8192     /* requests of one batch */
#define DVM_SERVING_CODE_BYTES 512 /* a code buffer of this size holds any code of this header */

/* ---- paging: rows, positions and cache slots of a batch's new tokens; pages for them --------------------------------
 * n requests; request i holds c_i = max(cached[i], 0) tokens in the cache and brings f_i = max(fresh[i], 0) new ones.
 *   starts[i]      first row of request i: the sum of f_j over j < i, cut at `rows`; starts[n] rows are in use.  (Below,
 *                  f_i is what is left of it: starts[i + 1] - starts[i].)
 *   lengths[i]     c_i + f_i
 *   table[i, b]    page of the request's tokens [b P, (b + 1) P), P = page_size.  In: the pages of the blocks it holds
 *                  (b < ceil(c_i / P)).  Written: the blocks it gains, ceil(c_i / P) <= b < ceil(lengths[i] / P), b <
 *                  max_blocks; they take the entries of `free` in order, request by request, -1 once these run out.
 *                  Other entries are left as they were.
 *   positions[t]   position in its request of the token in row t; -1 in rows behind the last one
 *   slots[t]       table[i, position / P] P + position % P; -1 behind the last row, where there is no page (a
 *                  negative entry, a block beyond max_blocks) and for a slot beyond 2^31 - 2, which no cache has
 *   taken[0]       entries of `free` that were asked for: beyond free_pages, the batch did not fit
 * Tensors: cached [n], fresh [n], free [free_pages] -> table [n, max_blocks] (also read), starts [n + 1], lengths [n],
 * positions [rows], slots [rows], taken [1]; all int32, dense.  A position or length beyond 2^31 - 1 is cut there. */
typedef struct {
  int64_t requests;    /* n: 0 .. DVM_MAX_REQUESTS */
  int64_t max_blocks;  /* columns of the table */
  int64_t page_size;   /* P >= 1 */
  int64_t rows;
  int64_t free_pages;
} dvm_paging_desc;
int dvm_encode_paging(const dvm_paging_desc* d, void* code, size_t code_capacity, size_t* code_size);

/* ---- rotary: head norms, rotation by position, keys and values into the paged cache --------------------------------
 * For every row t with a position p = positions[t] in [0, angle_rows), and every query head and key head x of head_dim
 * elements:
 *   norm:    x_e = x_e / sqrt(mean(x^2) + eps) * w_e            (w: the query or the key weight; without `norm`: x as it is)
 *   rotate:  (x_i, x_j) = (x_i c - x_j s, x_j c + x_i s)        for the rotary_dim / 2 pairs k: (i, j) = (k, k +
 *            rotary_dim / 2), or (2 k, 2 k + 1) when `interleaved`; c = angles[p, k], s = angles[p, rotary_dim / 2 + k];
 *            elements from rotary_dim on stay
 * in fp32, rounded once when stored.  Query heads go to q_out[t]; with `paged`, key heads go to the cache at
 * slot = slots[t] (page slot / page_size, token slot % page_size) and the value heads, converted only, to the same place
 * of the value cache; a slot outside [0, pages * page_size) stores nothing.  Without `paged`, key heads go to k_out[t].
 * Rows whose position is outside [0, angle_rows) are left as they were everywhere.  Two rows must not share a slot.
 * Tensors: q [tokens, q_heads, head_dim], k, v [tokens, kv_heads, head_dim] (v: `paged` only), q weight, k weight
 * [head_dim] (`norm` only), angles [angle_rows, rotary_dim] fp32 dense, positions [tokens], slots [tokens] (`paged` only)
 * -> q_out, then k_cache, v_cache [pages, page_size, kv_heads, head_dim] or k_out [tokens, kv_heads, head_dim].
 * The last dimension of every tensor is adjacent.  q_out may be q itself (same pointer, strides and type), and k_out k.
 * DVM_ERR_UNSUPPORTED: head_dim not a multiple of 8 or above 256, rotary_dim not a multiple of 8. */
typedef struct {
  int64_t tokens, q_heads, kv_heads, head_dim;
  int64_t rotary_dim;                              /* 0 .. head_dim */
  int64_t angle_rows;
  int64_t pages, page_size;                        /* `paged` only */
  int64_t q_stride[2], k_stride[2], v_stride[2];   /* token, head */
  int64_t q_out_stride[2], k_out_stride[2];        /* token, head */
  int64_t k_cache_stride[3], v_cache_stride[3];    /* page, token, head */
  int32_t dtype, weight_dtype, out_dtype;          /* DVM_F32 or DVM_BF16: of q, k, v; of the weights; of the outputs */
  int32_t norm, interleaved, paged;                /* 0 / 1 */
  float eps;
} dvm_rotary_desc;
int dvm_encode_rotary(const dvm_rotary_desc* d, void* code, size_t code_capacity, size_t* code_size);

/* ---- attention over a paged cache: causal, sliding window, first tokens that stay visible ---------------------------
 * Request i owns the query rows starts[i] <= t < starts[i + 1] and the first lengths[i] tokens of its block table; its
 * last query row sits at position lengths[i] - 1.  Row t at position p sees the tokens s with
 *   s <= p,  s < max_blocks * page_size,  (window == 0 or s > p - window or s < sinks),
 *   and a page id table[i, s / page_size] inside [0, pages);
 * for query head h, with kv head h / (q_heads / kv_heads):
 *   out[t, h] = sum_s softmax_s(scale * q[t, h] . k[s]) v[s];   a row that sees nothing gives 0.
 * (Infinite scores as the quotient has them: one of +inf makes its row NaN, and so do scores that are all -inf.)
 * Tokens a row does not see have no influence on it, whatever the cache holds there.  Query rows outside every request
 * are left as they were in `out`, and so are a request's rows beyond the first max_q.
 * fp32 accumulation; the bf16 kernels round the unnormalised probabilities to bf16 for the second product.
 * Tensors: q [rows, q_heads, head_dim], k_cache, v_cache [pages, page_size, kv_heads, head_dim], table [requests,
 * max_blocks], starts [requests + 1], lengths [requests] -> out [rows, q_heads, head_dim], workspace.  The last dimension
 * of q, the caches and out is adjacent.  The workspace holds parts of long sequences within the launch and nothing
 * between launches: dvm_tensor_extents gives its bytes (16-byte aligned; any pointer, NULL too, where that is 0).
 * Launches that may run at the same time, in two captured graphs say, need workspaces of their own.
 * bf16 inputs with head_dim a multiple of 8 up to 128, strides that are multiples of 8 and pointers to 16 bytes run on
 * the tensor cores; other inputs on a kernel without them, which reads a row's tokens one after another (milliseconds).
 * Single tokens of up to 16 query heads per kv head share the device evenly whatever their lengths; otherwise one CTA walks
 * the cache for 2 floor(128 / heads per kv head) rows of one kv head, so few such rows on long caches leave most of it idle.
 * An infinite or NaN value that some rows of such a block see and others do not makes its rows take the slow way.
 * DVM_ERR_UNSUPPORTED: head_dim above 256; page_size not a power of two or below 8; more than 128 query heads per kv head. */
typedef struct {
  int64_t requests, rows, q_heads, kv_heads, head_dim;
  int64_t pages, page_size, max_blocks;
  int64_t window, sinks;                           /* window 0: every earlier token is visible */
  int64_t max_q;                                   /* most query rows of one request, >= 1; 1: the kernel for single tokens */
  int64_t q_stride[2], out_stride[2];              /* token, head */
  int64_t k_stride[3], v_stride[3];                /* page, token, head */
  int32_t dtype, out_dtype;                        /* DVM_F32 or DVM_BF16: of q and the caches; of out */
  float scale;                                     /* > 0 */
} dvm_attention_desc;
int dvm_encode_attention(const dvm_attention_desc* d, void* code, size_t code_capacity, size_t* code_size);

/* Which kernel the calling thread's last launch of an attention code ran on (for tests and tools): 0 without tensor
 * cores, 1 single tokens, 2 prompts.  DVM_ERR_INVALID_ARG before the thread's first. */
int dvm_last_attention_kernel(int* kernel);

#ifdef __cplusplus
}
#endif
#endif /* DVM_SERVING_H_ */

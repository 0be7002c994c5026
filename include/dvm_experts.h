/* libdvm -- operators of a layer of experts: a router picks some experts for every token, and the tokens' rows go through the
 * weights of theirs in 8-bit floating point.  Each is a meta-kernel of its own type, used like the operators of a serving
 * step (dvm_serving.h): encode it on the host for the sizes of an instance (no CUDA call), then dvm_launch it on device
 * tensors.  dvm_verify, dvm_disassemble, dvm_tensor_extents, dvm_code_info and dvm_launch_checked know these codes; the
 * stacked launches and dvm_run_host refuse them (DVM_ERR_UNSUPPORTED).
 *
 * A layer of experts, in order (positions as dvm_encode_paging gives them):
 *   (router logits: dvm_program_matmul)
 *   dvm_encode_routing         experts and weights of every token; the plan: the tokens' rows, expert by expert
 *   dvm_encode_quantize        activations as 8-bit codes, each token's to the rows of its experts
 *   dvm_encode_scaled_matmul   those rows by the gate and up weights of their expert
 *   dvm_encode_quantize        silu(gate) * up as 8-bit codes
 *   dvm_encode_scaled_matmul   by the down weights
 *   dvm_encode_combine         each token's results added up by weight, to the residual stream
 * Dense layers take the quantizer and the product alone.  The plan stays on the device and may change between launches of
 * one code (also between replays of a graph that captured the launch); the kernels stay inside the tensors whatever it holds.
 *
 * Conventions as in dvm_serving.h: every call returns DVM_OK or a negative DVM_ERR_*; the caller owns every tensor, the
 * workspaces too, which hold nothing between launches (launches that may run at the same time need workspaces of their
 * own); nothing is allocated, nothing synchronised; launches are asynchronous on the stream given to dvm_launch and may be
 * captured.  Tensors are named by their place in the launch's list (inputs, then outputs, then a workspace).  Index tensors
 * are int32, dense.  Strides are in elements; the last dimension is adjacent.  An output must not overlap another tensor of
 * the launch (dvm_launch refuses outputs that begin where another tensor does with DVM_ERR_INVALID_ARG).
 *
 * 8-bit values: a matrix is held as codes (e4m3: sign, 4 bits of exponent, 3 of mantissa, largest value 448, no infinities)
 * with an fp32 scale for each block of 128 columns of a row, or of 128 rows and 128 columns; blocks at the end may be
 * smaller.  A value is its code's value times its block's scale.
 */
#ifndef DVM_EXPERTS_H_
#define DVM_EXPERTS_H_

#include "dvm.h"

#ifdef __cplusplus
extern "C" {
#endif

#define DVM_MAX_EXPERTS 512         /* experts of one router */
#define DVM_MAX_TOP_K 32            /* experts of one token */
#define DVM_MAX_WEIGHT_GROUPS 1024  /* weights of one scaled product */
#define DVM_SCALE_BLOCK 128         /* columns (and rows of a weight) that share a scale */
#define DVM_EXPERTS_CODE_BYTES 512  /* a code buffer of this size holds any code of this header */

/* ---- routing: experts of every token, their weights, and the tokens' rows expert by expert --------------------------
 * For token t with logits l_e:
 *   s_e = softmax over e of l, or sigmoid(l_e)
 *   c_e = s_e + bias[e]                       (without `biased`: s_e)
 *   with groups > 1: the experts form `groups` groups of neighbours; a group counts the sum of its two largest c (its only
 *   one, where a group is one expert); the top_groups groups that count most stay, of equal ones the first
 *   ids[t, 0 .. top_k)    the experts of the largest c among those, largest first, of equal ones the lowest index
 *   weights[t, j]         s of expert ids[t, j]; with `renormalise` divided by the sum over j (the quotient itself, also of scores
 *                         that are below fp32's range: only where all of them are those of -inf is it 0 / 0, NaN); times `factor`
 * The order is that of exact values: where 32 bits cannot tell two apart, they are computed in 64.  Without `biased` experts (not
 * groups) are ordered by their logits, whose order is that of the scores.  A NaN counts less than anything else.  Under softmax a
 * NaN or +inf logit, or logits of -inf alone, make all of the token's scores and weights NaN: groups, and biased experts, are then
 * taken by index, others by their logits.
 * The plan, over all (t, j):
 *   starts[e]     first row of expert e: rows starts[e] <= r < starts[e + 1] are its tokens, in their order;
 *                 starts[experts] rows are in use
 *   places[t, j]  row of token t at its expert ids[t, j]
 * With `masked`, tokens of negative positions[t] (rows behind the last one of a padded batch) take no part: ids -1,
 * weights 0, places -1.
 * Tensors: logits [tokens, experts], bias [experts] fp32 (`biased` only), positions [tokens] (`masked` only) -> ids, weights
 * (fp32), places [tokens, top_k], starts [experts + 1], workspace (dvm_tensor_extents gives its bytes; 16-byte aligned; any
 * pointer, NULL too, where that is 0).
 * DVM_ERR_TOO_LARGE: more experts or top_k than above, more than 32 groups or 2^23 tokens. */
enum { DVM_ROUTE_SOFTMAX = 0, DVM_ROUTE_SIGMOID = 1 };
typedef struct {
  int64_t tokens, experts;
  int64_t logits_stride;           /* token */
  int32_t dtype;                   /* DVM_F32 or DVM_BF16: of the logits */
  int32_t scoring;                 /* DVM_ROUTE_* */
  int32_t top_k, groups, top_groups;
  int32_t biased, masked, renormalise;  /* 0 / 1 */
  float factor;
} dvm_routing_desc;
int dvm_encode_routing(const dvm_routing_desc* d, void* code, size_t code_capacity, size_t* code_size);

/* ---- quantize: rows, gated pairs of rows or weights as 8-bit codes with scales ---------------------------------------
 * v = x, or with `gated` v[t, c] = silu(x[t, c]) * x[t, cols + c], silu(z) = z / (1 + exp(-z)).  For each block:
 *   scale = max(max |v| / 448, 2^-126)        rounded to fp32
 *   code  = the e4m3 value nearest to the quotient v / scale, of two the even one
 * (not of a rounded quotient, so the codes of an input are the same everywhere; with `gated` v is taken to 2^-40 where that
 * decides, silu(z) counts as zero where exp(-z) passes 2^126 -- z below -87.3365 --, v of 2^128 and more is an infinity, and the
 * scale may be that of a value less than 2^-15 below the largest.)
 * A block that holds an infinity or a NaN has the scale NaN and codes of zero.
 * block_rows 1: a scale for 128 columns of a row; 128: for 128 x 128 (weights; neither gated nor with copies).
 * copies = 0: row t of x is row t of the codes (out_rows = rows).  copies > 0: it is written to the rows places[t, j], 0 <= j <
 * copies, where these are in [0, out_rows), and nowhere else; no two places may be the same; other rows stay as they were.
 * Tensors: x [rows, cols] or [rows, 2 cols], places [rows, copies] (copies > 0 only) -> codes [out_rows, cols], scales
 * [out_rows / block_rows rounded up, cols / 128 rounded up] fp32.
 * codes start at a multiple of 16 bytes, and codes_stride is one; x may lie anywhere (16-byte aligned rows are read faster).
 * DVM_ERR_UNSUPPORTED: cols or codes_stride not a multiple of 16. */
typedef struct {
  int64_t rows, cols, out_rows;
  int64_t x_stride, codes_stride, scales_stride;  /* row */
  int32_t dtype;                                  /* DVM_F32 or DVM_BF16: of x */
  int32_t gated;                                  /* 0 / 1 */
  int32_t copies;                                 /* 0 .. DVM_MAX_TOP_K */
  int32_t block_rows;                             /* 1 or 128 */
} dvm_quantize_desc;
int dvm_encode_quantize(const dvm_quantize_desc* d, void* code, size_t code_capacity, size_t* code_size);

/* ---- scaled matmul: product of 8-bit matrices with a scale per block, one weight or one per group of rows --------------
 *   out[r, n] = sum over blocks b of x_scales[r, b] w_scales[g, n / 128, b] (sum over k in b of x[r, k] w[g, n, k])
 * fp32 accumulation, rounded once when stored.  The two scales are multiplied first, in fp32: a product below 2^-126 has fewer
 * bits than others, one of 2^128 and more is infinite.  With `grouped`, g is the group with starts[g] <= r < starts[g + 1] (starts as
 * routing gives them: ascending; values outside [0, rows] are cut); rows of no group stay as they were.  Without, groups is
 * 1 and every row meets that weight.
 * Tensors: x codes [rows, k], x_scales [rows, k / 128 rounded up] fp32, w codes [groups, n, k], w_scales [groups, n / 128, k /
 * 128, rounded up] fp32 dense, starts [groups + 1] (`grouped` only) -> out [rows, n], workspace (dvm_tensor_extents gives
 * its bytes; 16-byte aligned; any pointer, NULL too, where that is 0).
 * The products run on the tensor cores.  x and w start at multiples of 16 bytes (DVM_ERR_INVALID_ARG at launch otherwise).
 * Which of a row's partial sums are added first may depend on the numbers of rows of all groups, never on what they hold:
 * the same sizes and starts give the same bits.
 * DVM_ERR_UNSUPPORTED: k or a stride of x or w not a multiple of 16.  DVM_ERR_TOO_LARGE: more groups than above, or more than 2^31 -
 * 256 rows or columns of the result. */
typedef struct {
  int64_t rows, n, k, groups;
  int64_t x_stride, x_scales_stride, out_stride;  /* row */
  int64_t w_stride[2];                            /* group, row */
  int32_t out_dtype;                              /* DVM_F32 or DVM_BF16 */
  int32_t grouped;                                /* 0 / 1 */
} dvm_scaled_matmul_desc;
int dvm_encode_scaled_matmul(const dvm_scaled_matmul_desc* d, void* code, size_t code_capacity, size_t* code_size);

/* Rows of the tiles that the calling thread's last launch of a scaled product worked on (for tests and tools): 16 or 64 in the
 * kernel for few rows, 128 in the one for many.  DVM_ERR_INVALID_ARG before the thread's first. */
int dvm_last_scaled_matmul_tile(int* rows);

/* ---- combine: every token's rows added up by weight -------------------------------------------------------------------
 *   out[t] = base[t] + sum over j of weights[t, j] y[places[t, j]]          (without `based`: no base[t])
 * over the j whose place is in [0, rows), in their order, in fp32, rounded once when stored.  Tokens without any such place
 * stay as they were in `out`.
 * Tensors: y [rows, cols], places [tokens, top_k], weights [tokens, top_k] fp32, base [tokens, cols] (`based` only) -> out
 * [tokens, cols].  y, base and out have one type.  out may be base itself (same pointer and stride). */
typedef struct {
  int64_t tokens, top_k, rows, cols;
  int64_t y_stride, base_stride, out_stride;      /* row */
  int32_t dtype;                                  /* DVM_F32 or DVM_BF16 */
  int32_t based;                                  /* 0 / 1 */
} dvm_combine_desc;
int dvm_encode_combine(const dvm_combine_desc* d, void* code, size_t code_capacity, size_t* code_size);

#ifdef __cplusplus
}
#endif
#endif /* DVM_EXPERTS_H_ */

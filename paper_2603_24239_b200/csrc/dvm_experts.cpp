// Host half of the operators of a layer of experts (routing, quantize, scaled matmul, combine): encode, verify, dump, tensor
// extents.  Pure CPU: no CUDA call, no allocation.
#include "dvm_experts.h"

#include <math.h>
#include <stdio.h>

#include "dvm_describe.h"

namespace {

int check(const dvm_routing_desc& d) {
  if (!dim_ok(d.tokens) || !dim_ok(d.experts, 1) || d.top_k < 1 || d.groups < 1 || d.top_groups < 1 || !float_type(d.dtype)) return DVM_ERR_INVALID_ARG;
  if ((d.biased | d.masked | d.renormalise) & ~1 || (d.scoring != DVM_ROUTE_SOFTMAX && d.scoring != DVM_ROUTE_SIGMOID) || !isfinite(d.factor)) return DVM_ERR_INVALID_ARG;
  if (d.experts > DVM_MAX_EXPERTS || d.top_k > DVM_MAX_TOP_K || d.groups > 32 || d.tokens > (1 << 23)) return DVM_ERR_TOO_LARGE;
  if (d.experts % d.groups || d.top_groups > d.groups) return DVM_ERR_SHAPE_MISMATCH;
  if (d.top_k > d.top_groups * (d.experts / d.groups)) return DVM_ERR_SHAPE_MISMATCH;
  const int64_t size[1] = {d.tokens}, stride[1] = {d.logits_stride};
  return extent(size, stride, 1, d.experts, es_of(d.dtype)) < 0 ? DVM_ERR_INVALID_ARG : DVM_OK;
}

int check(const dvm_quantize_desc& d) {
  if (!dim_ok(d.rows) || !dim_ok(d.cols, 1) || !dim_ok(d.out_rows) || !float_type(d.dtype) || (d.gated & ~1)) return DVM_ERR_INVALID_ARG;
  if (d.copies < 0 || (d.block_rows != 1 && d.block_rows != DVM_SCALE_BLOCK) || (d.block_rows != 1 && (d.gated || d.copies))) return DVM_ERR_INVALID_ARG;
  if (d.copies > DVM_MAX_TOP_K) return DVM_ERR_TOO_LARGE;
  if (!d.copies && d.out_rows != d.rows) return DVM_ERR_SHAPE_MISMATCH;
  if (d.cols % 16 || (d.out_rows > 1 && d.codes_stride % 16)) return DVM_ERR_UNSUPPORTED;
  const int64_t r[1] = {d.rows}, o[1] = {d.out_rows}, b[1] = {dvm_up(d.out_rows, d.block_rows)}, kb = dvm_up(d.cols, DVM_SCALE_BLOCK);
  if (extent(r, &d.x_stride, 1, d.cols * (1 + d.gated), es_of(d.dtype)) < 0 || extent(o, &d.codes_stride, 1, d.cols, 1) < 0 ||
      extent(b, &d.scales_stride, 1, kb, 4) < 0 || !distinct(o, &d.codes_stride, 1, d.cols) || !distinct(b, &d.scales_stride, 1, kb))
    return DVM_ERR_INVALID_ARG;
  return DVM_OK;
}

int check(const dvm_scaled_matmul_desc& d) {
  if (!dim_ok(d.rows) || !dim_ok(d.n, 1) || !dim_ok(d.k, 1) || !dim_ok(d.groups, 1) || !float_type(d.out_dtype) || (d.grouped & ~1)) return DVM_ERR_INVALID_ARG;
  if (!d.grouped && d.groups != 1) return DVM_ERR_SHAPE_MISMATCH;
  // (the kernels add a tile's rows or columns, 256 at most, less one to these in 32 bits)
  if (d.groups > DVM_MAX_WEIGHT_GROUPS || d.rows > kMaxDim - 255 || d.n > kMaxDim - 255) return DVM_ERR_TOO_LARGE;
  const int64_t r[1] = {d.rows}, w[2] = {d.groups, d.n}, kb = dvm_up(d.k, DVM_SCALE_BLOCK), nb = dvm_up(d.n, DVM_SCALE_BLOCK);
  if (extent(r, &d.x_stride, 1, d.k, 1) < 0 || extent(r, &d.x_scales_stride, 1, kb, 4) < 0 || extent(w, d.w_stride, 2, d.k, 1) < 0 ||
      extent(r, &d.out_stride, 1, d.n, es_of(d.out_dtype)) < 0 || !distinct(r, &d.out_stride, 1, d.n) || (__int128)d.groups * nb * kb * 4 > kMaxBytes)
    return DVM_ERR_INVALID_ARG;
  // (the strides of tile copies are multiples of 16 bytes below 2^40, and not 0)
  auto ok = [](int64_t size, int64_t stride) { return size <= 1 || (stride > 0 && stride % 16 == 0 && stride < (1ll << 39)); };
  if (d.k % 16 || !ok(d.rows, d.x_stride) || !ok(d.groups, d.w_stride[0]) || !ok(d.n, d.w_stride[1])) return DVM_ERR_UNSUPPORTED;
  return DVM_OK;
}

int check(const dvm_combine_desc& d) {
  if (!dim_ok(d.tokens) || !dim_ok(d.top_k, 1) || !dim_ok(d.rows) || !dim_ok(d.cols, 1) || !float_type(d.dtype) || (d.based & ~1)) return DVM_ERR_INVALID_ARG;
  if (d.top_k > DVM_MAX_TOP_K) return DVM_ERR_TOO_LARGE;
  const int64_t t[1] = {d.tokens}, r[1] = {d.rows}, es = es_of(d.dtype);
  if (extent(r, &d.y_stride, 1, d.cols, es) < 0 || (d.based && extent(t, &d.base_stride, 1, d.cols, es) < 0) || extent(t, &d.out_stride, 1, d.cols, es) < 0 ||
      !distinct(t, &d.out_stride, 1, d.cols))
    return DVM_ERR_INVALID_ARG;
  return DVM_OK;
}

// Pieces of work, 0 for an instance that launches nothing.
int64_t tiles_of(const dvm_routing_desc& d) { return 1 + d.tokens / DVM_ROUTE_ONE; }  // (no tokens: starts are still written)
int64_t tiles_of(const dvm_quantize_desc& d) { return d.out_rows ? d.rows : 0; }
int64_t tiles_of(const dvm_scaled_matmul_desc& d) { return d.rows; }
int64_t tiles_of(const dvm_combine_desc& d) { return d.rows ? d.tokens : 0; }

uint32_t type_of(const dvm_routing_desc&) { return DVM_KERNEL_ROUTING; }
uint32_t type_of(const dvm_quantize_desc&) { return DVM_KERNEL_QUANTIZE; }
uint32_t type_of(const dvm_scaled_matmul_desc&) { return DVM_KERNEL_SCALED_MATMUL; }
uint32_t type_of(const dvm_combine_desc&) { return DVM_KERNEL_COMBINE; }

template <class D> int encode(const D* d, void* code, size_t cap, size_t* size) {
  if (!d || !size) return DVM_ERR_INVALID_ARG;
  const int st = check(*d);
  if (st != DVM_OK) return st;
  const auto s = dvm_slots(*d);
  return dvm_emit_descriptor<DVM_EXPERTS_CODE_BYTES>(*d, type_of(*d), s.n_in, s.n - s.n_in, tiles_of(*d), code, cap, size);
}

template <class D> int verify(const uint32_t* w, size_t n_words, size_t desc_bytes) {
  D d;
  if (desc_bytes < sizeof d) return DVM_ERR_BAD_CODE;
  dvm_descriptor(w, &d);
  if (check(d) != DVM_OK) return DVM_ERR_BAD_CODE;
  const auto s = dvm_slots(d);
  return dvm_descriptor_well_formed<D>(w, n_words, s.n, s.n_in, tiles_of(d)) ? DVM_OK : DVM_ERR_BAD_CODE;
}

void extents(const dvm_routing_desc& d, int64_t* b) {
  const RoutingSlots s = dvm_slots(d);
  const int64_t t[1] = {d.tokens};
  b[s.logits] = extent(t, &d.logits_stride, 1, d.experts, es_of(d.dtype));
  if (d.biased) b[s.bias] = d.experts * 4;
  if (d.masked) b[s.positions] = d.tokens * 4;
  b[s.ids] = b[s.weights] = b[s.places] = d.tokens * d.top_k * 4;
  b[s.starts] = (d.experts + 1) * 4;
  b[s.ws] = dvm_routing_workspace(d);
}
void extents(const dvm_quantize_desc& d, int64_t* b) {
  const QuantizeSlots s = dvm_slots(d);
  const int64_t r[1] = {d.rows}, o[1] = {d.out_rows}, br[1] = {dvm_up(d.out_rows, d.block_rows)};
  b[s.x] = extent(r, &d.x_stride, 1, d.cols * (1 + d.gated), es_of(d.dtype));
  if (d.copies) b[s.places] = d.rows * d.copies * 4;
  b[s.codes] = extent(o, &d.codes_stride, 1, d.cols, 1);
  b[s.scales] = extent(br, &d.scales_stride, 1, dvm_up(d.cols, DVM_SCALE_BLOCK), 4);
}
void extents(const dvm_scaled_matmul_desc& d, int64_t* b) {
  const ScaledSlots s = dvm_slots(d);
  const int64_t r[1] = {d.rows}, w[2] = {d.groups, d.n}, kb = dvm_up(d.k, DVM_SCALE_BLOCK), nb = dvm_up(d.n, DVM_SCALE_BLOCK);
  b[s.x] = extent(r, &d.x_stride, 1, d.k, 1);
  b[s.xs] = extent(r, &d.x_scales_stride, 1, kb, 4);
  b[s.w] = extent(w, d.w_stride, 2, d.k, 1);
  b[s.ws] = d.groups * nb * kb * 4;
  if (d.grouped) b[s.starts] = (d.groups + 1) * 4;
  b[s.out] = extent(r, &d.out_stride, 1, d.n, es_of(d.out_dtype));
  b[s.work] = dvm_scaled_workspace(d);
}
void extents(const dvm_combine_desc& d, int64_t* b) {
  const CombineSlots s = dvm_slots(d);
  const int64_t t[1] = {d.tokens}, r[1] = {d.rows}, es = es_of(d.dtype);
  b[s.y] = extent(r, &d.y_stride, 1, d.cols, es);
  b[s.places] = b[s.weights] = d.tokens * d.top_k * 4;
  if (d.based) b[s.base] = extent(t, &d.base_stride, 1, d.cols, es);
  b[s.out] = extent(t, &d.out_stride, 1, d.cols, es);
}

const char* name_of(int dtype) { return dtype == DVM_BF16 ? "bf16" : "f32"; }
int dump(const dvm_routing_desc& d, char* buf, size_t cap) {
  return snprintf(buf, cap, "kernel routing  tokens %lld  experts %lld  top_k %d  groups %d of %d  %s%s%s%s  factor %g  %s\n", (long long)d.tokens, (long long)d.experts,
                  d.top_k, d.top_groups, d.groups, d.scoring == DVM_ROUTE_SOFTMAX ? "softmax" : "sigmoid", d.biased ? "  biased" : "", d.masked ? "  masked" : "",
                  d.renormalise ? "  renormalise" : "", d.factor, name_of(d.dtype));
}
int dump(const dvm_quantize_desc& d, char* buf, size_t cap) {
  return snprintf(buf, cap, "kernel quantize  rows %lld  cols %lld  out_rows %lld  copies %d  block %d x %d%s  %s -> e4m3\n", (long long)d.rows, (long long)d.cols,
                  (long long)d.out_rows, d.copies, d.block_rows, DVM_SCALE_BLOCK, d.gated ? "  gated" : "", name_of(d.dtype));
}
int dump(const dvm_scaled_matmul_desc& d, char* buf, size_t cap) {
  return snprintf(buf, cap, "kernel scaled_matmul  rows %lld  n %lld  k %lld  groups %lld%s  tile rows %d  e4m3 -> %s\n", (long long)d.rows, (long long)d.n, (long long)d.k,
                  (long long)d.groups, d.grouped ? "  grouped" : "", dvm_scaled_tile(d), name_of(d.out_dtype));
}
int dump(const dvm_combine_desc& d, char* buf, size_t cap) {
  return snprintf(buf, cap, "kernel combine  tokens %lld  top_k %lld  rows %lld  cols %lld%s  %s\n", (long long)d.tokens, (long long)d.top_k, (long long)d.rows,
                  (long long)d.cols, d.based ? "  based" : "", name_of(d.dtype));
}

// f(descriptor) for the descriptor of a verified code
template <class F> void with_descriptor(const uint32_t* w, F f) {
  switch (w[DVM_H_KERNEL_TYPE]) {
    case DVM_KERNEL_ROUTING: { dvm_routing_desc d; f(dvm_descriptor(w, &d)); break; }
    case DVM_KERNEL_QUANTIZE: { dvm_quantize_desc d; f(dvm_descriptor(w, &d)); break; }
    case DVM_KERNEL_SCALED_MATMUL: { dvm_scaled_matmul_desc d; f(dvm_descriptor(w, &d)); break; }
    default: { dvm_combine_desc d; f(dvm_descriptor(w, &d)); }
  }
}

}  // namespace

RoutingSlots dvm_slots(const dvm_routing_desc& d) {
  RoutingSlots s;
  int n = 0;
  s.logits = n++;
  s.bias = d.biased ? n++ : -1;
  s.positions = d.masked ? n++ : -1;
  s.n_in = n;
  s.ids = n++;
  s.weights = n++;
  s.places = n++;
  s.starts = n++;
  s.ws = n++;
  s.n = n;
  return s;
}
QuantizeSlots dvm_slots(const dvm_quantize_desc& d) {
  QuantizeSlots s;
  int n = 0;
  s.x = n++;
  s.places = d.copies ? n++ : -1;
  s.n_in = n;
  s.codes = n++;
  s.scales = n++;
  s.n = n;
  return s;
}
ScaledSlots dvm_slots(const dvm_scaled_matmul_desc& d) {
  ScaledSlots s;
  int n = 0;
  s.x = n++;
  s.xs = n++;
  s.w = n++;
  s.ws = n++;
  s.starts = d.grouped ? n++ : -1;
  s.n_in = n;
  s.out = n++;
  s.work = n++;
  s.n = n;
  return s;
}
CombineSlots dvm_slots(const dvm_combine_desc& d) {
  CombineSlots s;
  int n = 0;
  s.y = n++;
  s.places = n++;
  s.weights = n++;
  s.base = d.based ? n++ : -1;
  s.n_in = n;
  s.out = n++;
  s.n = n;
  return s;
}

// Which kernel takes a scaled product, by the rows of a group if they were dealt out evenly and by the tiles that gives.
//  16  the weights' bytes are all that counts: up to 12 rows to a group (of 128 experts, 4096 to 2816, drawn evenly, so that they have
//      more and fewer: 8 rows on average 235 us, 250 in tiles of 64, 280 in the kernel for many; 12: 253, 276, 285; 13: 262, 279, 294;
//      14: 283, 279, 293; 16: 317, 286, 285; of 64, 2048 to 4096: 12: 97, 109, 105; 14: 110, 110, 109; 16: 116, 112, 110; groups of just
//      16: 245, 258, 276, of just 20: 401, 290, 281), or up to 32 where the tiles do not fill the device (32 rows, 4096 to 4096: 9.9,
//      10.0, 17.7)
//  64  more rows, and still no more tiles than CTAs (128 rows, 4096 to 4096: 20.8, 13.0, 18.9; 256: 37, 18.4, 19.1)
//  else the kernel for many (128 rows, 4096 to 11008: 50, 26, 19.6; 2048 rows of 64 experts, 4096 to 2816: 256, 169, 157; 512 of
//      8, 2048 to 4096: 49, 30, 17.7)
int dvm_scaled_tile(const dvm_scaled_matmul_desc& d) {
  const int64_t each = dvm_up(d.rows, d.groups), across = dvm_up(d.n, DVM_SCALE_BLOCK) * d.groups;
  if (each <= 12 || (each <= 32 && dvm_up(each, 16) * across <= DVM_SCALED_UNITS)) return 16;
  return dvm_up(each, 64) * across <= DVM_SCALED_UNITS ? 64 : DVM_SCALED_MANY;
}

extern "C" int dvm_encode_routing(const dvm_routing_desc* d, void* code, size_t code_capacity, size_t* code_size) { return encode(d, code, code_capacity, code_size); }
extern "C" int dvm_encode_quantize(const dvm_quantize_desc* d, void* code, size_t code_capacity, size_t* code_size) { return encode(d, code, code_capacity, code_size); }
extern "C" int dvm_encode_scaled_matmul(const dvm_scaled_matmul_desc* d, void* code, size_t code_capacity, size_t* code_size) {
  return encode(d, code, code_capacity, code_size);
}
extern "C" int dvm_encode_combine(const dvm_combine_desc* d, void* code, size_t code_capacity, size_t* code_size) { return encode(d, code, code_capacity, code_size); }

int dvm_verify_experts(const uint32_t* w, size_t n_words) {
  const uint32_t nt = w[DVM_H_COUNTS] & 0xff;
  if (nt > DVM_MAX_TENSORS) return DVM_ERR_BAD_CODE;
  const size_t bytes = n_words >= DVM_HDR_WORDS + 2 * (size_t)nt ? (n_words - DVM_HDR_WORDS - 2 * (size_t)nt) * 4 : 0;
  switch (w[DVM_H_KERNEL_TYPE]) {
    case DVM_KERNEL_ROUTING: return verify<dvm_routing_desc>(w, n_words, bytes);
    case DVM_KERNEL_QUANTIZE: return verify<dvm_quantize_desc>(w, n_words, bytes);
    case DVM_KERNEL_SCALED_MATMUL: return verify<dvm_scaled_matmul_desc>(w, n_words, bytes);
    default: return verify<dvm_combine_desc>(w, n_words, bytes);
  }
}

void dvm_extents_experts(const uint32_t* w, int64_t* b) {
  with_descriptor(w, [&](const auto& d) { extents(d, b); });
}

int dvm_disassemble_experts(const uint32_t* w, char* buf, size_t cap) {
  int n = -1;
  with_descriptor(w, [&](const auto& d) { n = dump(d, buf, cap); });
  return n >= 0 && (size_t)n < cap ? DVM_OK : DVM_ERR_BUFFER_TOO_SMALL;
}

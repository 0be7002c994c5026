// Host half of the serving meta-kernels (paging, rotary, attention): encode, verify, dump, tensor extents.
// Pure CPU: no CUDA call, no allocation.
#include "dvm_serving.h"

#include <math.h>
#include <stdio.h>
#include <string.h>

namespace {

constexpr int64_t kMaxDim = (1ll << 31) - 1;
constexpr int64_t kMaxBytes = 1ll << 46;  // no tensor reaches farther from its pointer

inline int64_t es_of(int dtype) { return dtype == DVM_BF16 ? 2 : 4; }
inline bool dim_ok(int64_t v, int64_t lo = 0, int64_t hi = kMaxDim) { return v >= lo && v <= hi; }
inline bool float_type(int dt) { return dt == DVM_F32 || dt == DVM_BF16; }

// Bytes from the pointer to the end of the last element of a strided tensor with an adjacent last dim; 0 when it is
// empty, -1 when a stride is negative or the tensor reaches too far.
int64_t extent(const int64_t* size, const int64_t* stride, int n, int64_t last, int64_t es) {
  __int128 far = last;
  bool empty = last == 0;
  for (int i = 0; i < n; ++i) {
    if (size[i] == 0) empty = true;
    if (size[i] > 1) {
      if (stride[i] < 0) return -1;
      far += (__int128)(size[i] - 1) * stride[i];
    }
  }
  if (empty) return 0;
  if (far * es > kMaxBytes) return -1;
  return (int64_t)(far * es);
}

// Whether no element of a strided output is addressed twice: dims in the order of their strides, each stride past all
// that the dims before it reach.
bool distinct(const int64_t* size, const int64_t* stride, int n, int64_t last) {
  int order[3] = {0, 1, 2};
  for (int i = 0; i < n; ++i)
    for (int j = i + 1; j < n; ++j)
      if (stride[order[j]] < stride[order[i]]) { int t = order[i]; order[i] = order[j]; order[j] = t; }
  __int128 reach = last;
  for (int i = 0; i < n; ++i) {
    const int k = order[i];
    if (size[k] <= 1) continue;
    if (stride[k] < reach) return false;
    reach += (__int128)(size[k] - 1) * stride[k];
  }
  return true;
}

int check_paging(const dvm_paging_desc& d) {
  if (!dim_ok(d.requests) || !dim_ok(d.max_blocks) || !dim_ok(d.page_size, 1) || !dim_ok(d.rows) || !dim_ok(d.free_pages)) return DVM_ERR_INVALID_ARG;
  if (d.requests > DVM_MAX_REQUESTS) return DVM_ERR_TOO_LARGE;
  return DVM_OK;
}

int check_rotary(const dvm_rotary_desc& d) {
  if (!dim_ok(d.tokens) || !dim_ok(d.q_heads) || !dim_ok(d.kv_heads) || !dim_ok(d.head_dim, 1) || !dim_ok(d.rotary_dim) ||
      !dim_ok(d.angle_rows) || d.rotary_dim > d.head_dim)
    return DVM_ERR_INVALID_ARG;
  if (!float_type(d.dtype) || !float_type(d.out_dtype) || (d.norm && !float_type(d.weight_dtype))) return DVM_ERR_INVALID_ARG;
  if ((d.norm | d.interleaved | d.paged) & ~1) return DVM_ERR_INVALID_ARG;
  if (d.norm && !(d.eps >= 0.f && isfinite(d.eps))) return DVM_ERR_INVALID_ARG;
  if (d.paged && (!dim_ok(d.pages) || !dim_ok(d.page_size, 1) || d.pages * d.page_size > kMaxDim)) return DVM_ERR_INVALID_ARG;
  if (d.head_dim % 8 || d.head_dim > 256 || d.rotary_dim % 8) return DVM_ERR_UNSUPPORTED;
  if (d.q_heads + 2 * d.kv_heads > 65535) return DVM_ERR_TOO_LARGE;
  const int64_t qs[2] = {d.tokens, d.q_heads}, ks[2] = {d.tokens, d.kv_heads}, cs[3] = {d.pages, d.page_size, d.kv_heads};
  const int64_t ei = es_of(d.dtype), eo = es_of(d.out_dtype), D = d.head_dim;
  if (extent(qs, d.q_stride, 2, D, ei) < 0 || extent(ks, d.k_stride, 2, D, ei) < 0 || extent(qs, d.q_out_stride, 2, D, eo) < 0) return DVM_ERR_INVALID_ARG;
  if (!distinct(qs, d.q_out_stride, 2, D)) return DVM_ERR_INVALID_ARG;
  if (d.angle_rows * d.rotary_dim * 4 > kMaxBytes) return DVM_ERR_INVALID_ARG;
  if (d.paged) {
    if (extent(ks, d.v_stride, 2, D, ei) < 0 || extent(cs, d.k_cache_stride, 3, D, eo) < 0 || extent(cs, d.v_cache_stride, 3, D, eo) < 0) return DVM_ERR_INVALID_ARG;
    if (!distinct(cs, d.k_cache_stride, 3, D) || !distinct(cs, d.v_cache_stride, 3, D)) return DVM_ERR_INVALID_ARG;
  } else {
    if (extent(ks, d.k_out_stride, 2, D, eo) < 0 || !distinct(ks, d.k_out_stride, 2, D)) return DVM_ERR_INVALID_ARG;
  }
  return DVM_OK;
}

int check_attention(const dvm_attention_desc& d) {
  if (!dim_ok(d.requests) || !dim_ok(d.rows) || !dim_ok(d.q_heads, 1) || !dim_ok(d.kv_heads, 1) || !dim_ok(d.head_dim, 1) ||
      !dim_ok(d.pages) || !dim_ok(d.page_size, 1) || !dim_ok(d.max_blocks) || !dim_ok(d.window) || !dim_ok(d.sinks) || !dim_ok(d.max_q, 1))
    return DVM_ERR_INVALID_ARG;
  if (!float_type(d.dtype) || !float_type(d.out_dtype)) return DVM_ERR_INVALID_ARG;
  if (!(d.scale > 0.f) || !isfinite(d.scale)) return DVM_ERR_INVALID_ARG;
  if (d.q_heads % d.kv_heads) return DVM_ERR_SHAPE_MISMATCH;
  if (d.requests > DVM_MAX_REQUESTS) return DVM_ERR_TOO_LARGE;
  if (d.head_dim > 256 || (d.page_size & (d.page_size - 1)) || d.page_size < 8 || d.q_heads / d.kv_heads > 128 || d.q_heads > 65535) return DVM_ERR_UNSUPPORTED;
  if (d.max_blocks * d.page_size > kMaxDim || d.pages * d.page_size > kMaxDim) return DVM_ERR_UNSUPPORTED;  // (positions are 32-bit)
  const int64_t qs[2] = {d.rows, d.q_heads}, cs[3] = {d.pages, d.page_size, d.kv_heads}, D = d.head_dim;
  if (extent(qs, d.q_stride, 2, D, es_of(d.dtype)) < 0 || extent(qs, d.out_stride, 2, D, es_of(d.out_dtype)) < 0 ||
      extent(cs, d.k_stride, 3, D, es_of(d.dtype)) < 0 || extent(cs, d.v_stride, 3, D, es_of(d.dtype)) < 0)
    return DVM_ERR_INVALID_ARG;
  if (!distinct(qs, d.out_stride, 2, D)) return DVM_ERR_INVALID_ARG;
  return DVM_OK;
}

template <class D> int emit(const D& d, uint32_t type, int n_in, int n_out, int64_t tiles, void* code, size_t cap, size_t* size) {
  const int nt = n_in + n_out;
  const size_t total = DVM_HDR_WORDS + 2 * (size_t)nt + (sizeof(D) + 3) / 4;
  static_assert((DVM_HDR_WORDS + 2 * 16) * 4 + sizeof(D) + 4 <= DVM_SERVING_CODE_BYTES, "the code buffer size of the header");
  *size = total * 4;
  if (!code || cap < total * 4) return DVM_ERR_BUFFER_TOO_SMALL;
  uint32_t* w = (uint32_t*)code;
  memset(w, 0, total * 4);
  w[DVM_H_MAGIC] = DVM_MAGIC;
  w[DVM_H_KERNEL_TYPE] = type;
  w[DVM_H_N_TILES] = (uint32_t)tiles;
  w[DVM_H_TOTAL_WORDS] = (uint32_t)total;
  w[DVM_H_COUNTS] = (uint32_t)nt | ((uint32_t)n_in << 8) | ((uint32_t)n_out << 24);
  w[DVM_H_PRIMARY] = 0xffffffffu;
  memcpy(w + DVM_HDR_WORDS + 2 * nt, &d, sizeof(D));
  return DVM_OK;
}

// Pieces of work, 0 for an instance that launches nothing.
int64_t tiles_of(const dvm_paging_desc& d) { return 1 + d.rows / 1024; }  // (an empty batch still writes starts, taken and the padding rows)
int64_t tiles_of(const dvm_rotary_desc& d) { return d.q_heads + d.kv_heads ? d.tokens : 0; }
int64_t tiles_of(const dvm_attention_desc& d) { return d.requests ? d.rows : 0; }

template <class D> bool well_formed(const uint32_t* w, size_t n_words, int nt, int n_in, int64_t tiles) {
  return n_words == DVM_HDR_WORDS + 2 * (size_t)nt + (sizeof(D) + 3) / 4 && w[DVM_H_N_TILES] == (uint32_t)tiles && w[DVM_H_CODE_WORDS] == 0 &&
         w[DVM_H_COUNTS] == ((uint32_t)nt | ((uint32_t)n_in << 8) | ((uint32_t)(nt - n_in) << 24));
}

}  // namespace

RotarySlots dvm_rotary_slots(const dvm_rotary_desc& d) {
  RotarySlots s;
  int n = 0;
  s.q = n++;
  s.k = n++;
  s.v = d.paged ? n++ : -1;
  s.wq = d.norm ? n++ : -1;
  s.wk = d.norm ? n++ : -1;
  s.angles = n++;
  s.positions = n++;
  s.slots = d.paged ? n++ : -1;
  s.n_in = n;
  s.q_out = n++;
  s.k_out = n++;
  s.v_out = d.paged ? n++ : -1;
  s.n = n;
  return s;
}

bool dvm_attention_tensor_cores(const dvm_attention_desc& d) {
  if (d.dtype != DVM_BF16 || d.head_dim % 8 || d.head_dim > 128 || d.pages == 0) return false;
  auto ok = [](int64_t size, int64_t stride) { return size <= 1 || (stride > 0 && stride % 8 == 0 && stride < (1ll << 39)); };  // (a tile copy's strides: multiples of 16 bytes below 2^40)
  return ok(d.rows, d.q_stride[0]) && ok(d.q_heads, d.q_stride[1]) && ok(d.pages, d.k_stride[0]) && ok(d.page_size, d.k_stride[1]) &&
         ok(d.kv_heads, d.k_stride[2]) && ok(d.pages, d.v_stride[0]) && ok(d.page_size, d.v_stride[1]) && ok(d.kv_heads, d.v_stride[2]);
}

extern "C" int dvm_encode_paging(const dvm_paging_desc* d, void* code, size_t code_capacity, size_t* code_size) {
  if (!d || !code_size) return DVM_ERR_INVALID_ARG;
  const int st = check_paging(*d);
  return st != DVM_OK ? st : emit(*d, DVM_KERNEL_PAGING, PG_TABLE, PG_N - PG_TABLE, tiles_of(*d), code, code_capacity, code_size);
}

extern "C" int dvm_encode_rotary(const dvm_rotary_desc* d, void* code, size_t code_capacity, size_t* code_size) {
  if (!d || !code_size) return DVM_ERR_INVALID_ARG;
  const int st = check_rotary(*d);
  if (st != DVM_OK) return st;
  const RotarySlots s = dvm_rotary_slots(*d);
  return emit(*d, DVM_KERNEL_ROTARY, s.n_in, s.n - s.n_in, tiles_of(*d), code, code_capacity, code_size);
}

extern "C" int dvm_encode_attention(const dvm_attention_desc* d, void* code, size_t code_capacity, size_t* code_size) {
  if (!d || !code_size) return DVM_ERR_INVALID_ARG;
  const int st = check_attention(*d);
  return st != DVM_OK ? st : emit(*d, DVM_KERNEL_ATTENTION, AT_OUT, AT_N - AT_OUT, tiles_of(*d), code, code_capacity, code_size);
}

int dvm_verify_serving(const uint32_t* w, size_t n_words) {
  const uint32_t counts = w[DVM_H_COUNTS];
  const uint32_t nt = counts & 0xff;
  if (nt > DVM_MAX_TENSORS) return DVM_ERR_BAD_CODE;
  const size_t desc_bytes = n_words >= DVM_HDR_WORDS + 2 * (size_t)nt ? (n_words - DVM_HDR_WORDS - 2 * (size_t)nt) * 4 : 0;
  if (w[DVM_H_KERNEL_TYPE] == DVM_KERNEL_PAGING) {
    dvm_paging_desc d;
    if (desc_bytes < sizeof d) return DVM_ERR_BAD_CODE;
    dvm_serving_desc(w, &d);
    return check_paging(d) == DVM_OK && well_formed<dvm_paging_desc>(w, n_words, PG_N, PG_TABLE, tiles_of(d)) ? DVM_OK : DVM_ERR_BAD_CODE;
  }
  if (w[DVM_H_KERNEL_TYPE] == DVM_KERNEL_ROTARY) {
    dvm_rotary_desc d;
    if (desc_bytes < sizeof d) return DVM_ERR_BAD_CODE;
    dvm_serving_desc(w, &d);
    if (check_rotary(d) != DVM_OK) return DVM_ERR_BAD_CODE;
    const RotarySlots s = dvm_rotary_slots(d);
    return well_formed<dvm_rotary_desc>(w, n_words, s.n, s.n_in, tiles_of(d)) ? DVM_OK : DVM_ERR_BAD_CODE;
  }
  dvm_attention_desc d;
  if (desc_bytes < sizeof d) return DVM_ERR_BAD_CODE;
  dvm_serving_desc(w, &d);
  return check_attention(d) == DVM_OK && well_formed<dvm_attention_desc>(w, n_words, AT_N, AT_OUT, tiles_of(d)) ? DVM_OK : DVM_ERR_BAD_CODE;
}

void dvm_extents_serving(const uint32_t* w, int64_t* b) {
  if (w[DVM_H_KERNEL_TYPE] == DVM_KERNEL_PAGING) {
    dvm_paging_desc d;
    dvm_serving_desc(w, &d);
    b[PG_CACHED] = b[PG_FRESH] = b[PG_LENGTHS] = d.requests * 4;
    b[PG_FREE] = d.free_pages * 4;
    b[PG_TABLE] = d.requests * d.max_blocks * 4;
    b[PG_STARTS] = (d.requests + 1) * 4;
    b[PG_POSITIONS] = b[PG_SLOTS] = d.rows * 4;
    b[PG_TAKEN] = 4;
    return;
  }
  if (w[DVM_H_KERNEL_TYPE] == DVM_KERNEL_ROTARY) {
    dvm_rotary_desc d;
    dvm_serving_desc(w, &d);
    const RotarySlots s = dvm_rotary_slots(d);
    const int64_t qs[2] = {d.tokens, d.q_heads}, ks[2] = {d.tokens, d.kv_heads}, cs[3] = {d.pages, d.page_size, d.kv_heads};
    const int64_t ei = es_of(d.dtype), eo = es_of(d.out_dtype), D = d.head_dim;
    b[s.q] = extent(qs, d.q_stride, 2, D, ei);
    b[s.k] = extent(ks, d.k_stride, 2, D, ei);
    b[s.angles] = d.angle_rows * d.rotary_dim * 4;
    b[s.positions] = d.tokens * 4;
    b[s.q_out] = extent(qs, d.q_out_stride, 2, D, eo);
    if (d.norm) b[s.wq] = b[s.wk] = D * es_of(d.weight_dtype);
    if (d.paged) {
      b[s.v] = extent(ks, d.v_stride, 2, D, ei);
      b[s.slots] = d.tokens * 4;
      b[s.k_out] = extent(cs, d.k_cache_stride, 3, D, eo);
      b[s.v_out] = extent(cs, d.v_cache_stride, 3, D, eo);
    } else {
      b[s.k_out] = extent(ks, d.k_out_stride, 2, D, eo);
    }
    return;
  }
  dvm_attention_desc d;
  dvm_serving_desc(w, &d);
  const int64_t qs[2] = {d.rows, d.q_heads}, cs[3] = {d.pages, d.page_size, d.kv_heads}, ei = es_of(d.dtype), D = d.head_dim;
  b[AT_Q] = extent(qs, d.q_stride, 2, D, ei);
  b[AT_K] = extent(cs, d.k_stride, 3, D, ei);
  b[AT_V] = extent(cs, d.v_stride, 3, D, ei);
  b[AT_TABLE] = d.requests * d.max_blocks * 4;
  b[AT_STARTS] = (d.requests + 1) * 4;
  b[AT_LENGTHS] = d.requests * 4;
  b[AT_OUT] = extent(qs, d.out_stride, 2, D, es_of(d.out_dtype));
  b[AT_WS] = dvm_attention_workspace(d);
}

int dvm_disassemble_serving(const uint32_t* w, char* buf, size_t cap) {
  int n;
  if (w[DVM_H_KERNEL_TYPE] == DVM_KERNEL_PAGING) {
    dvm_paging_desc d;
    dvm_serving_desc(w, &d);
    n = snprintf(buf, cap, "kernel paging  requests %lld  max_blocks %lld  page_size %lld  rows %lld  free_pages %lld\n", (long long)d.requests,
                 (long long)d.max_blocks, (long long)d.page_size, (long long)d.rows, (long long)d.free_pages);
  } else if (w[DVM_H_KERNEL_TYPE] == DVM_KERNEL_ROTARY) {
    dvm_rotary_desc d;
    dvm_serving_desc(w, &d);
    n = snprintf(buf, cap, "kernel rotary  tokens %lld  q_heads %lld  kv_heads %lld  head_dim %lld  rotary_dim %lld%s%s%s  %s -> %s\n", (long long)d.tokens,
                 (long long)d.q_heads, (long long)d.kv_heads, (long long)d.head_dim, (long long)d.rotary_dim, d.norm ? "  norm" : "",
                 d.interleaved ? "  interleaved" : "", d.paged ? "  paged" : "", d.dtype == DVM_BF16 ? "bf16" : "f32", d.out_dtype == DVM_BF16 ? "bf16" : "f32");
  } else {
    dvm_attention_desc d;
    dvm_serving_desc(w, &d);
    n = snprintf(buf, cap, "kernel attention  requests %lld  rows %lld  q_heads %lld  kv_heads %lld  head_dim %lld  pages %lld x %lld  window %lld  sinks %lld  max_q %lld  %s -> %s\n",
                 (long long)d.requests, (long long)d.rows, (long long)d.q_heads, (long long)d.kv_heads, (long long)d.head_dim, (long long)d.pages,
                 (long long)d.page_size, (long long)d.window, (long long)d.sinks, (long long)d.max_q, d.dtype == DVM_BF16 ? "bf16" : "f32",
                 d.out_dtype == DVM_BF16 ? "bf16" : "f32");
  }
  return n >= 0 && (size_t)n < cap ? DVM_OK : DVM_ERR_BUFFER_TOO_SMALL;
}

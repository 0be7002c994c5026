// What the encoders of descriptor codes share (serving operators, operators of a layer of experts): sizes, strides, the code
// itself.
//   [ header : DVM_HDR_WORDS words ][ tensor table : 2 words per tensor slot, unused ][ the descriptor, padded to words ]
#pragma once
#include <stddef.h>
#include <stdint.h>
#include <string.h>

#include "../../include/dvm.h"
#include "dvm_format.h"

constexpr int64_t kMaxDim = (1ll << 31) - 1;
constexpr int64_t kMaxBytes = 1ll << 46;  // no tensor reaches farther from its pointer

inline int64_t es_of(int dtype) { return dtype == DVM_BF16 ? 2 : 4; }
inline bool dim_ok(int64_t v, int64_t lo = 0, int64_t hi = kMaxDim) { return v >= lo && v <= hi; }
inline bool float_type(int dt) { return dt == DVM_F32 || dt == DVM_BF16; }

// Bytes from the pointer to the end of the last element of a strided tensor with an adjacent last dim; 0 when it is
// empty, -1 when a stride is negative or the tensor reaches too far.
inline int64_t extent(const int64_t* size, const int64_t* stride, int n, int64_t last, int64_t es) {
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
inline bool distinct(const int64_t* size, const int64_t* stride, int n, int64_t last) {
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

template <size_t CAPACITY, class D> int dvm_emit_descriptor(const D& d, uint32_t type, int n_in, int n_out, int64_t tiles, void* code, size_t cap, size_t* size) {
  const int nt = n_in + n_out;
  const size_t total = DVM_HDR_WORDS + 2 * (size_t)nt + (sizeof(D) + 3) / 4;
  static_assert((DVM_HDR_WORDS + 2 * 16) * 4 + sizeof(D) + 4 <= CAPACITY, "the code buffer size of the header");
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

template <class D> bool dvm_descriptor_well_formed(const uint32_t* w, size_t n_words, int nt, int n_in, int64_t tiles) {
  return n_words == DVM_HDR_WORDS + 2 * (size_t)nt + (sizeof(D) + 3) / 4 && w[DVM_H_N_TILES] == (uint32_t)tiles && w[DVM_H_CODE_WORDS] == 0 &&
         w[DVM_H_COUNTS] == ((uint32_t)nt | ((uint32_t)n_in << 8) | ((uint32_t)(nt - n_in) << 24));
}

template <class D> inline const D& dvm_descriptor(const uint32_t* w, D* d) {
  memcpy(d, w + DVM_HDR_WORDS + 2 * (w[DVM_H_COUNTS] & 0xff), sizeof(D));
  return *d;
}

// Codes of the serving meta-kernels (private to libdvm): paging, rotary, attention.
//   [ header : DVM_HDR_WORDS words ][ tensor table : 2 words per tensor slot, unused ][ the descriptor, padded to words ]
// The descriptor of dvm_serving.h travels as it was given; dvm_verify checks it the way the encoder did, so a launch
// may rely on every limit below.
#pragma once
#include <cuda_runtime.h>
#include <stddef.h>
#include <stdint.h>

#include "../../include/dvm_serving.h"
#include "dvm_format.h"

enum { DVM_KERNEL_PAGING = 4, DVM_KERNEL_ROTARY = 5, DVM_KERNEL_ATTENTION = 6 };

// tensor slots
enum { PG_CACHED, PG_FRESH, PG_FREE, PG_TABLE, PG_STARTS, PG_LENGTHS, PG_POSITIONS, PG_SLOTS, PG_TAKEN, PG_N };
enum { AT_Q, AT_K, AT_V, AT_TABLE, AT_STARTS, AT_LENGTHS, AT_OUT, AT_WS, AT_N };
struct RotarySlots { int q, k, v, wq, wk, angles, positions, slots, q_out, k_out, v_out, n_in, n; };  // -1: not there
RotarySlots dvm_rotary_slots(const dvm_rotary_desc& d);

inline bool dvm_is_serving(uint32_t kernel_type) { return kernel_type >= DVM_KERNEL_PAGING && kernel_type <= DVM_KERNEL_ATTENTION; }
template <class D> inline const D& dvm_serving_desc(const uint32_t* w, D* d) {
  const uint8_t* src = (const uint8_t*)(w + DVM_HDR_WORDS + 2 * (w[DVM_H_COUNTS] & 0xff));
  for (size_t i = 0; i < sizeof(D); ++i) ((uint8_t*)d)[i] = src[i];
  return *d;
}

int dvm_verify_serving(const uint32_t* w, size_t n_words);
int dvm_disassemble_serving(const uint32_t* w, char* buf, size_t cap);
void dvm_extents_serving(const uint32_t* w, int64_t* bytes_needed);  // (of a verified code)
int dvm_launch_serving(const uint32_t* w, void* const* tensors, int n_tensors, cudaStream_t stream);

// the single-token attention kernel: CTAs that share its work (two per SM of a B200), and the keys of one tile
#define DVM_ATT_UNITS 296
#define DVM_ATT_TOKEN_TILE 64
// whether an attention code's sizes, types and strides suit the tensor-core kernels (the pointers are looked at per launch)
bool dvm_attention_tensor_cores(const dvm_attention_desc& d);
// ... and which one: single tokens with at most 16 query heads per kv head, else prompts
inline bool dvm_attention_single(const dvm_attention_desc& d) { return d.max_q == 1 && d.q_heads / d.kv_heads <= 16; }

// bytes of the workspace of a single-token code: every CTA leaves at most two parts of a head group (its range of tiles may
// start and end inside one), each a row of head_dim sums, a maximum and a sum of weights per query head, and 16 bytes
// that say which
inline int64_t dvm_attention_workspace(const dvm_attention_desc& d) {
  if (!d.requests || !d.rows || !dvm_attention_tensor_cores(d) || !dvm_attention_single(d)) return 0;
  return (int64_t)DVM_ATT_UNITS * (16 + 2 * (d.q_heads / d.kv_heads) * (d.head_dim + 2) * 4);
}

int dvm_launch_paging(const dvm_paging_desc& d, void* const* t, cudaStream_t stream);
int dvm_launch_rotary(const dvm_rotary_desc& d, void* const* t, cudaStream_t stream);
int dvm_launch_attention(const dvm_attention_desc& d, void* const* t, cudaStream_t stream);

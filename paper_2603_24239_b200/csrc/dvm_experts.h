// Codes of the operators of a layer of experts (private to libdvm): routing, quantize, scaled matmul, combine.
// The descriptor of dvm_experts.h travels as it was given (dvm_describe.h); dvm_verify checks it the way the encoder did, so
// a launch may rely on every limit below.
#pragma once
#include <cuda_runtime.h>
#include <stddef.h>
#include <stdint.h>

#include "../../include/dvm_experts.h"
#include "dvm_format.h"

enum { DVM_KERNEL_ROUTING = 7, DVM_KERNEL_QUANTIZE = 8, DVM_KERNEL_SCALED_MATMUL = 9, DVM_KERNEL_COMBINE = 10 };
inline bool dvm_is_experts(uint32_t kernel_type) { return kernel_type >= DVM_KERNEL_ROUTING && kernel_type <= DVM_KERNEL_COMBINE; }

// tensor slots; -1: not there
struct RoutingSlots { int logits, bias, positions, ids, weights, places, starts, ws, n_in, n; };
struct QuantizeSlots { int x, places, codes, scales, n_in, n; };
struct ScaledSlots { int x, xs, w, ws, starts, out, work, n_in, n; };
struct CombineSlots { int y, places, weights, base, out, n_in, n; };
RoutingSlots dvm_slots(const dvm_routing_desc& d);
QuantizeSlots dvm_slots(const dvm_quantize_desc& d);
ScaledSlots dvm_slots(const dvm_scaled_matmul_desc& d);
CombineSlots dvm_slots(const dvm_combine_desc& d);

int dvm_verify_experts(const uint32_t* w, size_t n_words);
int dvm_disassemble_experts(const uint32_t* w, char* buf, size_t cap);
void dvm_extents_experts(const uint32_t* w, int64_t* bytes_needed);  // (of a verified code)
int dvm_launch_experts(const uint32_t* w, void* const* tensors, int n_tensors, cudaStream_t stream);

inline int64_t dvm_up(int64_t a, int64_t b) { return (a + b - 1) / b; }

// Routing: up to DVM_ROUTE_ONE tokens are one launch of a cluster.  More are taken in rounds of DVM_ROUTE_ROUND, a warp to each, by
// chunks of whole rounds; a chunk is one CTA and has at most 15 of these: its counts are bytes.
#define DVM_ROUTE_ONE 128
#define DVM_ROUTE_ROUND 16
#define DVM_ROUTE_CHUNKS 592
inline int64_t dvm_route_rounds(const dvm_routing_desc& d) {  // rounds of one chunk
  if (d.tokens <= DVM_ROUTE_ONE) return 1;
  const int64_t rounds = dvm_up(dvm_up(d.tokens, DVM_ROUTE_ROUND), DVM_ROUTE_CHUNKS);
  return rounds < 15 ? rounds : 15;
}
inline int64_t dvm_route_chunks(const dvm_routing_desc& d) { return d.tokens <= DVM_ROUTE_ONE ? 1 : dvm_up(d.tokens, DVM_ROUTE_ROUND * dvm_route_rounds(d)); }
// bytes of its workspace: tokens of every expert in every chunk, where there are several
inline int64_t dvm_routing_workspace(const dvm_routing_desc& d) {
  const int64_t chunks = dvm_route_chunks(d);
  return chunks > 1 ? chunks * dvm_up(d.experts, 16) * 16 : 0;
}

// Scaled products: CTAs that share the work of the kernel for few rows (one per SM of a B200), and the rows of its tiles.
#define DVM_SCALED_UNITS 148
#define DVM_SCALED_MANY 128   // rows of a tile of the kernel for many (16 or 64 in the one for few)
int dvm_scaled_tile(const dvm_scaled_matmul_desc& d);
inline int64_t dvm_scaled_workspace(const dvm_scaled_matmul_desc& d) {
  const int tile = dvm_scaled_tile(d);
  return d.rows && tile != DVM_SCALED_MANY ? (int64_t)DVM_SCALED_UNITS * (32 + 2 * 128 * tile * 4) : 0;
}

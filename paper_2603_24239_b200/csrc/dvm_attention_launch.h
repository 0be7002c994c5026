// Launch-side declarations of the attention meta-kernel's translation units.
#pragma once
#include <cuda.h>

#include "dvm_attention.cuh"
#include "dvm_launch.h"

// A paged cache [pages, page_size, kv_heads, head_dim] of bf16 as a tensor map (head_dim, token of the page, kv head,
// page) whose box is 64 elements of min(page_size, most) tokens of one head, 128-byte swizzle.  What a box reaches beyond
// the tensor -- elements past head_dim, a page of -1 -- is filled with zeros.
int dvm_cache_map(const dvm_attention_desc& d, const int64_t* stride, const void* ptr, int most, CUtensorMap* map);

// The query rows [rows, q_heads, head_dim] as (head_dim, head of the group, kv head, row), a box of 64 elements of all heads
// of one group and `tokens` rows: row r of the box is token r / group, head r % group.
int dvm_query_map(const dvm_attention_desc& d, const void* ptr, int tokens, CUtensorMap* map);

int dvm_launch_attention_prompt(const dvm_attention_desc& d, const dvm::att::Args& a, int device, cudaStream_t stream);
int dvm_launch_attention_single(const dvm_attention_desc& d, const dvm::att::Args& a, int device, cudaStream_t stream);

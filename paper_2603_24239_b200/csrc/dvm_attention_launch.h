// Launch-side declarations of the attention meta-kernel's translation units.
#pragma once
#include <cuda.h>

#include "dvm_attention.cuh"
#include "dvm_launch.h"

// A paged cache [pages, page_size, kv_heads, head_dim] of bf16 as a tensor map (head_dim, token of the page, kv head,
// page) whose box is 64 elements of min(page_size, most) tokens of one head, 128-byte swizzle.  What a box reaches beyond
// the tensor -- elements past head_dim, a page of -1 -- is filled with zeros.
int dvm_cache_map(const dvm_attention_desc& d, const int64_t* stride, const void* ptr, int most, CUtensorMap* map);

int dvm_launch_attention_single(const dvm_attention_desc& d, const dvm::att::Args& a, cudaStream_t stream);

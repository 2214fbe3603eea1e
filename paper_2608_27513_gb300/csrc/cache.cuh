// cache.cuh -- the 8-bit cache of softmax-attention layers: record geometry and codes.
//
// A pool of pages of 32 tokens; a (page, KV head) is one record: 32 key rows of d codes, 32 value
// rows, then the FP32 scales of the keys and of the values and 8 unused bytes.  A code c stands for
// (c - 128) s.  Of a token's row the 16-byte chunk m lies at chunk m ^ h(t), h a permutation of
// t & 7: eight tokens' chunks m lie in eight different 16-byte columns of a 128-byte line, four of
// them (2c + e, c = 0 .. 3) with two neighbouring chunks too, and a pair of tokens with four chunks:
// the three ways in which warps read rows from shared memory, all without bank conflicts (d >= 128).
#pragma once

#include "damp_common.cuh"
#include "damp_internal.h"

namespace damp {

__host__ __device__ constexpr int cache_swizzle(int t, int d) { return ((t & 7) ^ ((t & 1) << 2)) & (d / 16 - 1); }
__host__ __device__ constexpr int cache_rows_bytes(int d) { return kCachePage * d; }  // keys or values of a record
__host__ __device__ constexpr int cache_record_bytes(int d) { return 2 * cache_rows_bytes(d) + 16; }
// byte of chunk m of token t's row inside the keys or the values
__device__ __forceinline__ int cache_chunk(int t, int m, int d) { return t * d + 16 * (m ^ cache_swizzle(t, d)); }

// tokens that a row's page table holds at most
__device__ __forceinline__ int cache_clamp(int n, int table) { return max(0, min(n, table * kCachePage)); }
// the page of an entry, -1 for a bad one
__device__ __forceinline__ int64_t cache_page(int32_t e, int64_t num_pages) { return e < 0 || e >= num_pages ? -1 : (int64_t)e; }

}  // namespace damp

// The paged 8-bit key-value cache: layout and addressing shared by the append and the
// attention kernels (gfx950).
//
// Keys and values are E4M3 codes.  The 16 tokens of a block share, for one kv head, one exponent
// for their keys and one for their values: value = code 2^(e - 127), e a byte.  A page holds
// `page` tokens (a multiple of 16) of every kv head:
//
//   k_codes  [pages, heads, page, dim]            a token's key in one piece
//   v_codes  [pages, heads, page / 16, dim, 16]   a block's values transposed
//   k_exps, v_exps  [pages, heads, page / 16]
//
// The products with the values contract over tokens, so their matrix-core operand is runs of
// tokens for one dimension: transposed blocks are read as such, 16 bytes a lane.
#pragma once
#include "moe_internal.h"
#include "common.h"

namespace moe {

constexpr int kKvBlock = 16;      // tokens that share an exponent

// Index of (page, head, block) among all blocks of the cache: of its exponents, and, times
// 16 dim, of its codes (keys and values alike).
__device__ __forceinline__ int64_t kv_block(int64_t page, int head, int block, int heads, int blocks_per_page) {
  return (page * heads + head) * blocks_per_page + block;
}

}  // namespace moe

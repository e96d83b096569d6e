// Pages of 4-bit keys and values (gl_cache4): the order of their bytes, and where the tokens of a call lie.  The index
// arithmetic also runs on the host, where it can be tested without a GPU.
//
// Group of 16 tokens of one kv head (17 * D bytes, one bulk copy): codes of K, scales of K, codes of V, scales of V.
// Inside a token's row of codes the order is the one the tensor-core fragments want, so that a thread reads all it
// needs of a token in one access and converts whole 32-bit words:
//   K: word (j, b) = dims 32 b + 8 j .. + 7 of block b, at word j * NB + b           (NB = D / 32 blocks)
//   V: half word (g, b) = dims 32 b + 4 g .. + 3, at half word (g ^ s) * NB + b, s = 4 for tokens with bit 1 set
// (the exclusive or spreads the four tokens that a warp reads together over all banks).
#pragma once
#include <cuda_runtime.h>

#include <cstdint>

#include "gl_launch.cuh"

namespace {

using gl::FastDiv;

constexpr int kGroup = 16;   // tokens per group

__host__ __device__ constexpr int group_bytes(int d) { return 17 * d; }
__host__ __device__ constexpr int k_scales_at(int d) { return 8 * d; }
__host__ __device__ constexpr int v_codes_at(int d) { return 8 * d + d / 2; }
__host__ __device__ constexpr int v_scales_at(int d) { return 16 * d + d / 2; }

struct CacheView {
  uint8_t* data;
  const int32_t* table;
  const int32_t* lengths;
  int64_t pages;
  int64_t head_stride, page_stride;   // bytes
  int kv_heads, page_tokens, batch, width;
  int capacity;                       // tokens a sequence can have: width * page_tokens
  FastDiv div_page;
};

__host__ __device__ __forceinline__ int clamped_length(const CacheView& c, int b) { return min(max(c.lengths[b], 0), c.capacity); }

struct TokensParams {
  CacheView c;
  int T, D;
  int64_t pitch;         // elements between tokens of the dense side
  uint32_t items;        // batch * T * kv_heads * (D / 8)
  FastDiv div_row, div_heads, div_T;
};

struct TokenAt {
  int w;                 // which eight dims
  int tok;               // place in its group
  int64_t dense;         // element of the dense side
  uint8_t* group;        // null: not in the cache
};

// The place of an item.  Threads past the last one (they still take part in the shuffles) have none, and read neither the
// lengths nor the table.
__host__ __device__ __forceinline__ TokenAt token_at(const TokensParams& p, uint32_t item) {
  TokenAt t = {0, 0, 0, nullptr};
  if (item >= p.items) return t;
  uint32_t row, w, token, h, b, i;
  p.div_row.divmod(item, row, w);
  p.div_heads.divmod(row, token, h);
  p.div_T.divmod(token, b, i);
  t.w = static_cast<int>(w);
  t.dense = static_cast<int64_t>(token) * p.pitch + static_cast<int64_t>(h) * p.D + w * 8u;
  const int pos = clamped_length(p.c, static_cast<int>(b)) - p.T + static_cast<int>(i);
  if (pos >= 0) {
    uint32_t slot, in_page;
    p.c.div_page.divmod(static_cast<uint32_t>(pos), slot, in_page);
    const int page = p.c.table[static_cast<int64_t>(b) * p.c.width + slot];
    t.tok = static_cast<int>(in_page % kGroup);
    if (page >= 0 && page < p.c.pages)
      t.group = p.c.data + page * p.c.page_stride + h * p.c.head_stride + static_cast<int64_t>(in_page / kGroup) * group_bytes(p.D);
  }
  return t;
}

// The thread of dims 32 b + 8 j .. + 7 stores, of V, the four bytes that hold dims 4 g .. + 3, g = 2 j + (b & 1), of the blocks
// b & ~1 and b | 1: offset in the token's row of codes.
__host__ __device__ __forceinline__ int v_offset(int NB, int b, int j, int tok) {
  return (((2 * j + (b & 1)) ^ ((tok & 2) ? 4 : 0)) * NB + (b & ~1)) * 2;
}

}  // namespace

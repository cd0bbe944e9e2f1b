// The paged 8-bit cache (include/taskpress.h): block layout and the arguments of its kernels.
//
// As in the 4-bit cache, codes sit where v_mfma_f32_16x16x32_f16 takes its A operand, here a byte a code: lane l of a
// product holds 8 bytes, and the 8 bytes of two products that follow each other are adjacent, so that a load takes 16
// bytes a lane and 1 KB a wave in a row.
//  - keys: rows of the operand are tokens, its k index channels: tile u of 16 tokens, product s of 32 channels; lane l
//    takes token 16 u + l % 16, channels 32 s + 8 (l / 16) + 0..7.
//  - values: rows are channels, k is tokens: tile j of 16 channels; lane l takes channel 16 j + l % 16, tokens
//    4 (l / 16) + 0..3 of both halves of the block, the tokens whose weights the lane holds after the key products.
#pragma once

#include "cache_block.h"

namespace tp {

template <int D>
struct Cache8Block {
  static constexpr int kKeys = 0;               // [2 tiles][D / 64][64 lanes][2 products][8]
  static constexpr int kValues = 32 * D;        // [D / 32][64 lanes][2 tiles][8]
  static constexpr int kValueScales = 64 * D;   // fp32 [32]
  static constexpr int kKeyScale = 64 * D + 128;
  static constexpr int kBytes = 64 * D + 144;
};

__host__ __device__ inline int64_t cache8_block_bytes(int d) { return 64 * d + 144; }

// The 8 bytes of the channels 8 piece .. 8 piece + 7 of a token's key.
template <int D>
__device__ inline int key8_place(int token, int piece) {
  return (token >> 4) * 16 * D + (piece >> 3) * 1024 + ((piece & 3) * 16 + (token & 15)) * 16 + ((piece >> 2) & 1) * 8;
}
// The byte of a token's value in channel x, from the values' start.
__device__ inline int value8_place(int token, int x) {
  return (x >> 5) * 1024 + (((token >> 2) & 3) * 16 + (x & 15)) * 16 + ((x >> 4) & 1) * 8 + (token >> 4) * 4 + (token & 3);
}

// Block j of a sequence for one (layer, head) in its page, or nullptr where that is no page.
template <int D>
__device__ inline uint8_t* cache8_block(const CacheArgs& c, int layer, int head, int32_t page, int j) {
  if (page < 0 || page >= c.num_pages) return nullptr;
  const int64_t at = (((int64_t)layer * c.num_pages + page) * c.Hkv + head) << c.page_shift;
  return c.pages + (at + (j & ((1 << c.page_shift) - 1))) * Cache8Block<D>::kBytes;
}

struct Cache8WriteArgs : CacheWriteArgs {
  int32_t fp8;      // e4m3 codes (else integers, a byte c + 128)
  int32_t nibbles;  // the loaded codes are two to a byte
};
hipError_t launch_cache8_append(Cache8WriteArgs& a, int head_dim, hipStream_t stream);
hipError_t launch_cache8_load(Cache8WriteArgs& a, int head_dim, hipStream_t stream);
hipError_t launch_cache8_read(CacheReadArgs& a, bool fp8, int head_dim, hipStream_t stream);

CachePlan cache8_plan(int32_t L, int32_t Hq, int32_t Hkv, int32_t head_dim, int32_t batch, int32_t max_new,
                      int32_t max_len);
hipError_t launch_cache8_attention(const CacheAttnArgs& a, bool fp8, int head_dim, hipStream_t stream);

}  // namespace tp

// The paged 4-bit cache (include/taskpress.h): block layout, page lookup, and the arguments of its
// kernels.
//
// A block holds 32 tokens of one (layer, KV head), contiguous: key codes, value codes, key scales,
// value scales.  Codes sit where v_mfma_f32_16x16x32_f16 takes its A operand, so that the attention
// loads 16 bytes a lane and needs no shuffle and no LDS:
//  - keys: rows of the operand are tokens, its k index channels.  Lane l takes token l % 16 and, in
//    product s, channels 32 s + 8 (l / 16) + 0..7: the words of product 0, 1, .. are adjacent, and a
//    product covers one scale group.
//  - values: rows are channels, k is tokens.  Lane l takes channel 16 j + l % 16 and tokens 4 (l / 16) +
//    0..3 of both halves of the block, the same tokens whose weights the lane holds after the key
//    products (their D layout: row 4 (l / 16) + r of the tile, column l % 16).
// A word's nibbles i and i + 4 are elements 2 i and 2 i + 1, so (word >> 4 i) & 0x000F000F is a pair in
// the 16-bit halves of a register.
#pragma once

#include <hip/hip_runtime.h>
#include <stdint.h>

#include "tp_internal.h"

namespace tp {

constexpr int kCacheBlock = 32;  // tokens

template <int D>
struct CacheBlock {
  static constexpr int kKeys = 0;                 // [32][D / 8] words
  static constexpr int kValues = 16 * D;          // [D / 64][64 lanes][4] words
  static constexpr int kKeyScales = 32 * D;       // bf16 [32][D / 32]
  static constexpr int kValueScales = 34 * D;     // fp32 [32]
  static constexpr int kBytes = 34 * D + 128;
};

__host__ __device__ inline int64_t cache_block_bytes(int d) { return 34 * d + 128; }

struct CacheArgs {
  uint8_t* pages;
  const int32_t* table;  // [batch][max_pages]
  const int32_t* lens;   // [batch]
  int64_t num_pages;
  int32_t max_pages, batch;
  int32_t page_shift;    // log2 of the blocks of a page
  int32_t max_len;       // longest sequence that counts: max_pages * page_tokens, or the caller's bound
  int32_t L, Hkv;
};

// Division of 0 <= n < 2^31 by a d >= 1 that the host knows: a multiply and a shift (T. Granlund and P. Montgomery,
// "Division by Invariant Integers using Multiplication", 1994), where the compiler's takes 20 instructions and
// leaves a uniform quotient in vector registers.
struct Divisor {
  uint32_t d, m, l;
  __host__ static Divisor of(int64_t d) {
    Divisor r = {(uint32_t)d, 0, 0};
    while (((int64_t)1 << r.l) < d) ++r.l;
    r.m = (uint32_t)((((uint64_t)1 << 32) * (((uint64_t)1 << r.l) - (uint64_t)d)) / (uint64_t)d + 1);
    return r;
  }
  __device__ int div(int n) const { return (int)((__umulhi((uint32_t)n, m) + (uint32_t)n) >> l); }
  __device__ int mod(int n, int quotient) const { return n - quotient * (int)d; }
};

// New tokens of sequence b: its rows of the step's tensors and its tokens of the cache.
struct StepArgs {
  const int32_t* offsets;  // [batch + 1] or nullptr
  int32_t total, max_new;
};
struct StepSeq {
  int32_t row, count, len;  // first row, new tokens, tokens held (0 where the length does not count)
};
// An element that the whole wave reads and no kernel running beside this one writes: a scalar load.
__device__ inline int32_t scalar_load(const int32_t* p) {
  return *(const __attribute__((address_space(4))) int32_t*)(uintptr_t)p;
}
// Whether a sequence's range of rows counts.
__device__ inline bool step_range(const StepArgs& s, int32_t lo, int32_t hi) {
  return lo >= 0 && hi > lo && hi <= s.total && hi - lo <= s.max_new;
}
__device__ inline StepSeq step_sequence(const CacheArgs& c, const StepArgs& s, int b) {
  StepSeq q;
  q.row = b;
  q.count = 1;
  if (s.offsets != nullptr) {
    const int32_t lo = scalar_load(s.offsets + b), hi = scalar_load(s.offsets + b + 1);
    const bool good = step_range(s, lo, hi);
    q.row = good ? lo : 0;
    q.count = good ? hi - lo : 0;
  }
  const int32_t len = scalar_load(c.lens + b);
  q.len = len < 0 || len > c.max_len ? 0 : len;
  return q;
}

// Block j of sequence b for one (layer, head), or nullptr where the sequence has no such page.
// j < max_pages << page_shift.
template <int D>
__device__ inline uint8_t* cache_block(const CacheArgs& c, int layer, int head, int b, int j) {
  const int32_t page = c.table[(int64_t)b * c.max_pages + (j >> c.page_shift)];
  if (page < 0 || page >= c.num_pages) return nullptr;
  const int64_t at = (((int64_t)layer * c.num_pages + page) * c.Hkv + head) << c.page_shift;
  return c.pages + (at + (j & ((1 << c.page_shift) - 1))) * CacheBlock<D>::kBytes;
}

// Strides in elements (bf16).
struct RowsArgs {
  uint16_t* data;
  int64_t layer, token, head;
};

struct CacheWriteArgs {
  CacheArgs c;
  StepArgs s;
  RowsArgs k, v, q, q_out;
  const int32_t* positions;  // [total]
  const float* cos_sin;      // [num_positions][rotary_dim] or nullptr: no rotation
  int64_t num_positions;
  int32_t rotary_dim, pairs;
  int32_t Hq;
  int32_t blocks;            // blocks that a sequence's new tokens may lie in
  Divisor heads, by_Hkv, by_blocks, by_total;  // set by the launch
  // tp_cache_load: sequence b's tokens are rows [kept_off[b], kept_off[b + 1]) of contiguous head-major tensors
  const uint8_t* v_q;        // [L][Hkv][K_tot][D / 2]
  const float* v_scales;     // [L][Hkv][K_tot]
  int64_t kept_off[TP_MAX_BATCH + 1];
};
hipError_t launch_cache_append(CacheWriteArgs& a, int head_dim, hipStream_t stream);
hipError_t launch_cache_load(CacheWriteArgs& a, int head_dim, hipStream_t stream);

struct CacheReadArgs {
  CacheArgs c;
  uint16_t* k;  // bf16 [L][Hkv][N_tot][D]
  uint16_t* v;
  int32_t blocks;
  Divisor heads, by_Hkv;  // set by the launch
  int64_t off[TP_MAX_BATCH + 1];
  int64_t first[TP_MAX_BATCH];
};
hipError_t launch_cache_read(CacheReadArgs& a, int head_dim, hipStream_t stream);

// The attention's plan: `tiles` tiles of 16 query rows a workgroup (rows of a KV head: new token, then query head of
// its group), `row_groups` of them for max_new tokens; context in `chunks` chunks of `chunk` tokens (a multiple of
// 128), whose partial results are merged when there are several.
struct CachePlan {
  int32_t tiles, row_groups, chunk, chunks;
  int32_t waves; // of a workgroup
  int32_t once;  // whether the loads leave the caches alone: the cache is read once a call, and no call finds it there
  size_t stat_off, o_off, total;  // workspace: (max, sum) float2 and output fp32 [D] of each row and chunk
};
CachePlan cache_plan(int32_t L, int32_t Hq, int32_t Hkv, int32_t head_dim, int32_t batch, int32_t max_new,
                     int32_t max_len);

struct CacheAttnArgs {
  CacheArgs c;
  StepArgs s;
  RowsArgs q, o;
  float* lse;       // [L][Hq][total] or nullptr
  float2* stat;
  float* part;
  int32_t Hq;
  Divisor R;        // query heads of a KV head
  Divisor heads, by_Hkv, by_groups, by_chunk;  // L * Hkv, Hkv, row_groups, chunk
  float scale_log2; // softmax_scale * log2(e)
  int32_t tiles, row_groups, chunk, chunks, waves, once;
};
hipError_t launch_cache_attention(const CacheAttnArgs& a, int head_dim, hipStream_t stream);

}  // namespace tp

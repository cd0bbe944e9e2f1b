// Attention over the paged 4-bit cache (tp_cache_attention): the newest tokens of each sequence, from one
// (decoding) to a prompt's chunk, against all its tokens.
//
// A workgroup takes 16 to 64 query rows of one (sequence, KV head) (rows: new token, then query head of the
// group) and one chunk of the context; its four or eight waves take every fourth or eighth block, with the
// softmax's running reference and sum in one pass, and join at the end through LDS.  Where a call has several
// chunks, their (maximum, sum, output) go to the workspace and k_cache_merge joins them.
//
// Products on v_mfma_f32_16x16x32_f16, both with the cache as the A operand, so that a lane's column is one
// query row from the scores to the output and the weights never leave their registers:
//   scores  S^T = K Q^T: codes times their group's scale, exact in fp16, one chain of products through the groups;
//   output  O^T += V^T P^T, with the values' scales multiplied into the weights P.
// Codes become fp16 operands by bit operations on pairs: 0x6400 | u is 1024 + u for a 4-bit number u = c + 8, and
// one packed fp16 operation more gives c exactly (a published way: Y. J. Kim et al., "Who Says Elephants Can't Run:
// Bringing Large Scale MoE Models into Cloud Scale Production", 2022; here with an offset of 8).  fp16 holds
// queries exactly once a row is brought near 2^14 by a power of two (a bf16 number has 8 significant bits, fp16 11;
// what lies 2^28 below the row's largest channel is off by 2^-39 of that one), and keeps the weights' rounding,
// 2^-11, below the output's (with bf16 operands the output's error was 1.4 times that of its own rounding).
//
// Measured at d = 128: one row tile is bound by HBM (64 sequences of 6K to 32K tokens, 64 query heads: 1.16 GB in
// 223 us, 5.2 TB/s; two of 262144 and 131073: 440 MB in 77 us), four by the vector ALU (chunks of 1024 and 300
// tokens against 17333 and 4096, 32 query heads: 302 GFLOP in 325 us).  Of 272 vector instructions a block with
// one tile, 446 with four, 176 turn codes into operands.
//
// The running reference m of a row bounds the weights that are rounded, p * scale of the value, not p alone:
// p = exp2(x - m) and the sum of the p's are fp32, in which the reference may be anywhere.
#include <algorithm>

#include "cache_join.h"

namespace tp {
namespace {

// Key scales as fp16 numbers: a power of two for all of them sets the largest of a block to exponent field 24 (2^9),
// and is kept while a block's scales lie in the fields 1 to 27: a code times a scale stays below 2^16 and is exact, 3 by
// 8 bits in fp16's 11.  Where no power holds all of a block's scales (more than 2^23 between them), its scores are
// formed in parts; the check for that costs a block no instruction more than the check of the largest alone.
constexpr int kScaleSet = 24, kScaleLeast = 1 << 7, kScaleHigh = 28 << 7;

__device__ inline u16x2 pair(uint32_t w) { return __builtin_bit_cast(u16x2, w); }
__device__ inline u16x2 max_pair(u16x2 a, u16x2 b) { return __builtin_elementwise_max(a, b); }
__device__ inline u16x2 min_pair(u16x2 a, u16x2 b) { return __builtin_elementwise_min(a, b); }

// Eight codes as fp16 numbers c.  magic: 0x64006400 in a vector register (with both constants scalar, the
// and and the or cannot be one instruction).
__device__ inline Frag codes(uint32_t w, uint32_t magic) {
  Frag f;
  const f16x2 low = {(_Float16)-1032.0f, (_Float16)-1032.0f}, high = {(_Float16)-72.0f, (_Float16)-72.0f};
  const f16x2 sixteenth = {(_Float16)0.0625f, (_Float16)0.0625f};
#pragma unroll
  for (int i = 0; i < 4; i += 2) {
    const uint32_t x = w >> (4 * i);
    const f16x2 a = __builtin_bit_cast(f16x2, (x & 0x000F000Fu) | magic) + low;  // 1024 + u
    const f16x2 b = __builtin_elementwise_fma(__builtin_bit_cast(f16x2, (x & 0x00F000F0u) | magic), sixteenth,
                                              high);  // 1024 + 16 u
    f.w[i] = __builtin_bit_cast(uint32_t, a);
    f.w[i + 1] = __builtin_bit_cast(uint32_t, b);
  }
  return f;
}

// NR tiles of 16 rows, W waves.  ONCE: the cache is read once and is not found in a cache by the next call (loads leave it out).
template <int D, int NR, int W, bool ONCE>
__global__ __launch_bounds__(64 * W, (NR == 1 ? 4 : NR == 2 ? 3 : 2) + (D == 64)) void k_cache_attention(CacheAttnArgs a) {
  using B = CacheBlock<D>;
  constexpr int KS = D / 32;  // products of a score: channels in steps of 32
  constexpr int ND = D / 16;  // output tiles: channels in steps of 16
  constexpr int kStride = D + 4;
  constexpr int kPolicy = ONCE ? 2 : 0;  // nontemporal
  __shared__ float lds_o[W][16][kStride];
  __shared__ float2 lds_stat[W][16 * NR];

  const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane((int)threadIdx.x >> 6);
  const int g = lane >> 4, n = lane & 15;
  const int rest = a.heads.div((int)blockIdx.x), lh = a.heads.mod((int)blockIdx.x, rest);
  const int layer = a.by_Hkv.div(lh), head = a.by_Hkv.mod(lh, layer);
  const int chunk = a.by_groups.div(rest), group = a.by_groups.mod(rest, chunk);
  const int b = blockIdx.y;
  // 64 of the chunk's pages from page0 on, one a lane
  int page0 = (chunk * a.chunk / kCacheBlock) >> a.c.page_shift;
  const int32_t* row_pages = a.c.table + (int64_t)b * a.c.max_pages;
  const auto load_pages = [&] {
    const uint32_t at = (uint32_t)(page0 + lane);
    return (int)at < a.c.max_pages ? *(const int32_t*)((const char*)row_pages + 4 * at) : -1;
  };
  int pages = load_pages();
  const StepSeq q = step_sequence(a.c, a.s, b);
  const RowGroup rg = row_group(a, q, group, 16 * NR);
  if (rg.row0 >= rg.rows || (chunk > 0 && chunk * a.chunk >= rg.keys)) return;
  if (pages >= a.c.num_pages) pages = -1;

  // Queries as the products' B operand: in registers, or, for several tiles, in LDS, one copy for the waves, which
  // leaves registers for three (two tiles) or two (four) waves a SIMD.
  constexpr bool kShared = NR > 1;
  __shared__ u32x4 lds_q[kShared ? NR * KS * 64 : 1];
  Frag qf[kShared ? 1 : NR][KS];
  __shared__ int lds_shift[kShared ? 16 * NR : 1];  // the powers of two that the rows were multiplied by
  int shift = 0;                                    // (one tile: the lane's row's)
  // softmax_scale * log2(e), less that power and the key scales'
  __shared__ float lds_scale[kShared ? W : 1][16 * NR];
  float scale = 0.0f;
#pragma unroll
  for (int r = 0; r < NR; ++r) {
    if (kShared && r != wave) continue;  // a wave prepares one tile
    const int row = rg.row0 + r * 16 + n;
    const int t = a.R.div(row);
    const bool in = row < rg.rows;
    const uint16_t* p = a.q.data + layer * a.q.layer + (q.row + t) * a.q.token + (head * (int)a.R.d + a.R.mod(row, t)) * a.q.head;
    uint4 x[KS];
    uint32_t top = 0;  // the row's largest magnitude, as bf16 bits
#pragma unroll
    for (int s = 0; s < KS; ++s) {
      x[s] = in ? *(const uint4*)(p + s * 32 + g * 8) : make_uint4(0, 0, 0, 0);
      const uint32_t w[4] = {x[s].x, x[s].y, x[s].z, x[s].w};
#pragma unroll
      for (int i = 0; i < 4; ++i) top = max(top, max(w[i] & 0x7FFFu, (w[i] >> 16) & 0x7FFFu));
    }
    top = row_max(top);
    const int e = 15 - __builtin_amdgcn_frexp_expf(__uint_as_float(top << 16));  // the largest comes to [2^14, 2^15)
    shift = e;
    if (kShared && g == 0) lds_shift[r * 16 + n] = e;
#pragma unroll
    for (int s = 0; s < KS; ++s) {
      const uint32_t w[4] = {x[s].x, x[s].y, x[s].z, x[s].w};
      Frag f;
#pragma unroll
      for (int i = 0; i < 4; ++i)
        f.w[i] = pack_h(__builtin_amdgcn_ldexpf(__uint_as_float(w[i] << 16), e),
                        __builtin_amdgcn_ldexpf(__uint_as_float(w[i] & 0xFFFF0000u), e));
      if (!kShared)
        qf[kShared ? 0 : r][s] = f;
      else
        lds_q[(r * KS + s) * 64 + lane] = (u32x4){f.w[0], f.w[1], f.w[2], f.w[3]};
    }
  }
  if (kShared) __syncthreads();
  const auto set_scales = [&](int power) {
#pragma unroll
    for (int r = 0; r < NR; ++r) {
      // above 0 and finite, so that an unseen token's -infinity and a score of 0 stay that
      const float x = __builtin_amdgcn_fmed3f(
          __builtin_amdgcn_ldexpf(a.scale_log2, power - (kShared ? lds_shift[r * 16 + n] : shift)), 0x1p-149f, -kNoMax);
      if (kShared)
        lds_scale[wave][r * 16 + n] = x;
      else
        scale = x;
    }
  };
  set_scales(-112);
  const auto query = [&](int r, int s) {
    if (!kShared) return qf[kShared ? 0 : r][s];
    Frag f;
    const u32x4 x = lds_q[(r * KS + s) * 64 + lane];
    f.w[0] = x.x;
    f.w[1] = x.y;
    f.w[2] = x.z;
    f.w[3] = x.w;
    return f;
  };

  uint32_t magic = 0x64006400u;
  asm("" : "+v"(magic));

  f32x4 acc[NR][ND];
  float m[NR], l[NR];
#pragma unroll
  for (int r = 0; r < NR; ++r) {
    m[r] = -kFar;
    l[r] = 0.0f;
#pragma unroll
    for (int x = 0; x < ND; ++x) acc[r][x] = (f32x4){0, 0, 0, 0};
  }

  const int key0 = chunk * a.chunk, key1 = min(rg.keys, key0 + a.chunk);
  const int j0 = key0 / kCacheBlock + wave, j1 = (key1 + kCacheBlock - 1) / kCacheBlock;  // every W-th block
  const int all_seen = rg.before + a.R.div(rg.row0) + 1;  // keys before this one are seen by every row of the group

  // Block j's part of the lane, in registers: keys' words and scales, values' words and scales.
  u32x4 kw[2], vw[ND / 4], vs[2];
  u32x2 ks[2];
  const auto page_of = [&](int j) { return __builtin_amdgcn_readlane(pages, (j >> a.c.page_shift) - page0); };
  const auto block_at = [&](int j) {
    const int page = max(page_of(j), 0);  // a missing page: any
    const int64_t at = (((int64_t)layer * a.c.num_pages + page) * a.c.Hkv + head) << a.c.page_shift;
    uint8_t* blk = a.c.pages + (at + (j & ((1 << a.c.page_shift) - 1))) * B::kBytes;
    return __builtin_amdgcn_make_buffer_rsrc(blk, 0, B::kBytes, 0x00020000);
  };
  // the lane's places in a block
  const int at_key = n * (D / 2) + g * KS * 4, at_key_scale = n * KS * 2;
  const int at_value = lane * 16, at_value_scale = g * 16;
  const auto load_keys = [&](__amdgpu_buffer_rsrc_t blk) {
#pragma unroll
    for (int u = 0; u < 2; ++u) {
      if (KS == 4) {
        kw[u] = __builtin_amdgcn_raw_buffer_load_b128(blk, at_key, B::kKeys + u * 8 * D, kPolicy);
        ks[u] = __builtin_amdgcn_raw_buffer_load_b64(blk, at_key_scale, B::kKeyScales + u * D, kPolicy);
      } else {
        const u32x2 w = __builtin_amdgcn_raw_buffer_load_b64(blk, at_key, B::kKeys + u * 8 * D, kPolicy);
        kw[u] = (u32x4){w.x, w.y, 0, 0};
        ks[u] = (u32x2){__builtin_amdgcn_raw_buffer_load_b32(blk, at_key_scale, B::kKeyScales + u * D, kPolicy), 0};
      }
    }
  };
  const auto load_values = [&](__amdgpu_buffer_rsrc_t blk) {
#pragma unroll
    for (int x = 0; x < ND / 4; ++x) vw[x] = __builtin_amdgcn_raw_buffer_load_b128(blk, at_value, B::kValues + x * 1024, kPolicy);
#pragma unroll
    for (int u = 0; u < 2; ++u) vs[u] = __builtin_amdgcn_raw_buffer_load_b128(blk, at_value_scale, B::kValueScales + u * 64, kPolicy);
  };
  if (j0 < j1) {
    const auto blk = block_at(j0);
    load_keys(blk);
    load_values(blk);
  }
  // the group's tiles: a decoding sequence beside a prompt's chunk has one, whose weights alone are formed
  const int tiles = (rg.rows - rg.row0 + 15) / 16;
  int bias = 0;  // bf16 bits taken off a key scale: it becomes an fp16 number times 2^(bias / 128 - 112)
  // A key scale's bits, opaque, so that nothing formed from it is kept in registers over the loop.
  const auto scale_of = [&](int u, int s) {
    uint32_t w = ks[u][s >> 1];
    asm volatile("" : "+v"(w));
    return (int)((s & 1) ? w >> 16 : w & 0xFFFFu);
  };
  // A block with key scales out of the power's range: another power, if it is the largest or one that is not 0.  Returns
  // whether that does not hold all of them; if it does, the zeros, also out of range, become what the power takes for 0.
  const auto fit_scales = [&] {
    u16x2 top = {0, 0};
#pragma unroll
    for (int u = 0; u < 2; ++u)
#pragma unroll
      for (int i = 0; i < KS / 2; ++i) top = max_pair(top, pair(ks[u][i]));
    const int most = max((int)top.x, (int)top.y);
    const auto small = [&] {
      if (bias == 0) return false;
      u16x2 least = {0xFFFF, 0xFFFF};  // less 1: a 0 is the largest
#pragma unroll
      for (int u = 0; u < 2; ++u)
#pragma unroll
        for (int i = 0; i < KS / 2; ++i) least = min_pair(least, pair(ks[u][i]) - (u16x2){1, 1});
      return __builtin_amdgcn_ballot_w64(min((int)least.x, (int)least.y) < bias + kScaleLeast - 1) != 0;
    };
    const bool large = __builtin_amdgcn_ballot_w64(most - bias >= kScaleHigh) != 0;
    bool split = false;
    if (large || small()) {
      bias = __builtin_amdgcn_readfirstlane(max((int)(wave_max((uint32_t)most) >> 7) - kScaleSet, 0) << 7);
      set_scales((bias >> 7) - 112);
      split = small();
    }
    if (!split) {
      const u16x2 zero = {(unsigned short)bias, (unsigned short)bias};
#pragma unroll
      for (int u = 0; u < 2; ++u)
#pragma unroll
        for (int i = 0; i < KS / 2; ++i) ks[u][i] = __builtin_bit_cast(uint32_t, max_pair(pair(ks[u][i]), zero));
    }
    return split;
  };
  // The scores of a block whose key scales no power holds: those that one does at a time, from the largest down, and the
  // products summed in fp32 at the scores' power.
  const auto apart = [&](f32x4 (&xs)[2][NR]) {
#pragma unroll
    for (int u = 0; u < 2; ++u)
#pragma unroll
      for (int r = 0; r < NR; ++r) xs[u][r] = (f32x4){0, 0, 0, 0};
    int below = 0x8000;  // above the bits of the scales that are left
    while (true) {
      int left = 0;
#pragma unroll
      for (int u = 0; u < 2; ++u)
#pragma unroll
        for (int s = 0; s < KS; ++s) {
          const int v = scale_of(u, s);
          left = max(left, v < below ? v : 0);
        }
      left = __builtin_amdgcn_readfirstlane((int)wave_max((uint32_t)left));
      if (left == 0) break;
      const int power = max((left >> 7) - kScaleSet, 0);
      const int from = power == 0 ? 0 : (power << 7) + kScaleLeast;
      const float weight = __builtin_amdgcn_ldexpf(1.0f, power - (bias >> 7));
#pragma unroll
      for (int u = 0; u < 2; ++u) {
#pragma unroll
        for (int r = 0; r < NR; ++r) {
          f32x4 x = {0, 0, 0, 0};
#pragma unroll
          for (int s = 0; s < KS; ++s) {
            const int v = scale_of(u, s);
            const uint16_t bits = v < below && v >= from ? (uint16_t)((v - (power << 7)) << 3) : 0;
            const _Float16 one = __builtin_bit_cast(_Float16, bits);
            uint32_t w = kw[u][s];
            asm volatile("" : "+v"(w));
            Frag k = codes(w, magic);
#pragma unroll
            for (int i = 0; i < 4; ++i)
              k.w[i] = __builtin_bit_cast(uint32_t, __builtin_bit_cast(f16x2, k.w[i]) * (f16x2){one, one});
            x = mfma(k, query(r, s), x);
          }
          xs[u][r] += x * weight;
        }
      }
      below = from;
    }
  };
  for (int j = j0; j < j1; j += W) {
    const bool missing = page_of(j) < 0;
    const bool masked = missing || (j + 1) * kCacheBlock > all_seen;
    if (masked) {  // scales of slots that no row sees may be anything, of those that one does not see must be finite
      const uint32_t held = bias == 0 ? 0 : (uint32_t)(bias + (kScaleSet << 7)) * 0x10001u;  // in the power's range
#pragma unroll
      for (int u = 0; u < 2; ++u) {
        if (missing || j * kCacheBlock + u * 16 + n >= rg.keys) ks[u] = (u32x2){held, held};
#pragma unroll
        for (int i = 0; i < 4; ++i)
          vs[u][i] = __float_as_uint(__builtin_amdgcn_fmed3f(__uint_as_float(vs[u][i]), 0.0f, -kNoMax));
      }
    }
    // Key scales to fp16: bf16 bits, with the exponent brought into range and the mantissa moved by 3 bits.  One
    // comparison finds the scales on both sides of the range: those below wrap to large numbers.
    const auto in_range = [&](u16x2 (&t)[2][KS / 2]) {
      const u16x2 off = {(unsigned short)(bias + kScaleLeast), (unsigned short)(bias + kScaleLeast)};
      u16x2 top = {0, 0};
#pragma unroll
      for (int u = 0; u < 2; ++u)
#pragma unroll
        for (int i = 0; i < KS / 2; ++i) {
          t[u][i] = pair(ks[u][i]) - off;
          top = u == 0 && i == 0 ? t[u][i] : max_pair(top, t[u][i]);
        }
      return __builtin_amdgcn_ballot_w64(max((int)top.x, (int)top.y) >= kScaleHigh - kScaleLeast) == 0;
    };
    u16x2 scales[2][KS / 2];
    bool split = false;
    if (!__builtin_expect(in_range(scales), true)) {
      split = fit_scales();
      in_range(scales);
    }
    f32x4 xs[2][NR];
    if (__builtin_expect(split, false)) {
      apart(xs);
    } else {
      const u16x2 eight = {8, 8}, least = {8 * kScaleLeast, 8 * kScaleLeast};
#pragma unroll
      for (int u = 0; u < 2; ++u) {
        f16x2 sc[KS / 2];
#pragma unroll
        for (int i = 0; i < KS / 2; ++i) sc[i] = __builtin_bit_cast(f16x2, scales[u][i] * eight + least);
#pragma unroll
        for (int r = 0; r < NR; ++r) xs[u][r] = (f32x4){0, 0, 0, 0};
#pragma unroll
        for (int s = 0; s < KS; ++s) {
          const _Float16 one = sc[s >> 1][s & 1];
          Frag k = codes(kw[u][s], magic);
#pragma unroll
          for (int i = 0; i < 4; ++i)
            k.w[i] = __builtin_bit_cast(uint32_t, __builtin_bit_cast(f16x2, k.w[i]) * (f16x2){one, one});
#pragma unroll
          for (int r = 0; r < NR; ++r) xs[u][r] = mfma(k, query(r, s), xs[u][r]);
        }
      }
    }
    // (after the last block, that block once more: no branch, so the registers stay in place)
    const int jn = j + W < j1 ? j + W : j;
    if ((jn >> a.c.page_shift) - page0 >= 64) {
      page0 = jn >> a.c.page_shift;
      pages = load_pages();
      if (pages >= a.c.num_pages) pages = -1;
    }
    const auto next = block_at(jn);
    __builtin_amdgcn_sched_barrier(0);
    load_keys(next);

    Frag pf[NR] = {};
#pragma unroll
    for (int r = 0; r < NR; ++r) {
      if (r > 0 && r >= tiles) break;
      float w[8], p[8], sum, top;
      const float factor = kShared ? lds_scale[wave][r * 16 + n] : scale;
#pragma unroll
      for (int i = 0; i < 8; ++i) w[i] = __uint_as_float(vs[i >> 2][i & 3]);
      if (masked) {
        const int row = rg.row0 + r * 16 + n;
        const int seen = missing || row >= rg.rows ? 0 : rg.before + a.R.div(row) + 1;
#pragma unroll
        for (int i = 0; i < 8; ++i)
          if (j * kCacheBlock + (i >> 2) * 16 + g * 4 + (i & 3) >= seen) xs[i >> 2][r][i & 3] = -INFINITY;
      }
      const auto weigh = [&] {
#pragma unroll
        for (int i = 0; i < 8; ++i) {
          p[i] = __builtin_amdgcn_exp2f(fmaf(xs[i >> 2][r][i & 3], factor, -m[r]));
          sum = i == 0 ? p[i] : sum + p[i];
          p[i] *= w[i];
          top = i == 0 ? p[i] : fmaxf(top, p[i]);
        }
      };
      weigh();
      if (__builtin_amdgcn_ballot_w64(fmaxf(top, sum * kLeastScale) > kLimit) != 0) {
        float next = kNoMax;
#pragma unroll
        for (int i = 0; i < 8; ++i) {
          next = fmaxf(next, fmaf(xs[i >> 2][r][i & 3], factor, __builtin_amdgcn_logf(fmaxf(w[i], kLeastScale)) - kSet));
        }
        next = fmaxf(row_max(next), m[r]);
        const float f = __builtin_amdgcn_exp2f(m[r] - next);
        m[r] = next;
        l[r] *= f;
#pragma unroll
        for (int i = 0; i < ND; ++i) acc[r][i] *= f;
        weigh();
      }
      l[r] += sum;
#pragma unroll
      for (int i = 0; i < 4; ++i) pf[r].w[i] = pack_h(p[2 * i], p[2 * i + 1]);
    }
#pragma unroll
    for (int x = 0; x < ND; ++x) {
      const Frag v = codes(vw[x >> 2][x & 3], magic);
#pragma unroll
      for (int r = 0; r < NR; ++r) acc[r][x] = mfma(v, pf[r], acc[r][x]);
    }
    __builtin_amdgcn_sched_barrier(0);
    load_values(next);
  }

  // join the waves
#pragma unroll
  for (int r = 0; r < NR; ++r) {
    l[r] = row_sum(l[r]);
    if (g == 0) lds_stat[wave][r * 16 + n] = make_float2(m[r], l[r]);
  }
  __syncthreads();
#pragma unroll
  for (int r = 0; r < NR; ++r) {
    if (r > 0 && r >= tiles) break;
    float top = kNoMax;
#pragma unroll
    for (int w = 0; w < W; ++w) top = fmaxf(top, lds_stat[w][r * 16 + n].x);
    const float f = __builtin_amdgcn_exp2f(m[r] - top);
    if (r > 0) __syncthreads();
#pragma unroll
    for (int x = 0; x < ND; ++x) {
      const f32x4 o = acc[r][x] * f;
      *(f32x4*)&lds_o[wave][n][x * 16 + g * 4] = o;
    }
    __syncthreads();
    // a row's channels by 4 W threads
    constexpr int CH = D / (4 * W);
    const int row16 = threadIdx.x / (4 * W), c0 = (threadIdx.x % (4 * W)) * CH;
    const int row = rg.row0 + r * 16 + row16;
    if (row < rg.rows) {
      float2 st = make_float2(kNoMax, 0.0f);
#pragma unroll
      for (int w = 0; w < W; ++w) st.x = fmaxf(st.x, lds_stat[w][r * 16 + row16].x);
#pragma unroll
      for (int w = 0; w < W; ++w) {
        const float2 s = lds_stat[w][r * 16 + row16];
        st.y += s.y * __builtin_amdgcn_exp2f(s.x - st.x);
      }
      float o[CH];
#pragma unroll
      for (int i = 0; i < CH; ++i) {
        o[i] = 0.0f;
#pragma unroll
        for (int w = 0; w < W; ++w) o[i] += lds_o[w][row16][c0 + i];
      }
      const int t = a.R.div(row), hq = head * (int)a.R.d + a.R.mod(row, t);
      const int64_t token = q.row + t;
      if (rg.keys <= a.chunk) {  // the only chunk
        store_output<CH>(a, layer, token, hq, c0, o, st);
      } else {
        const int64_t at = partial_row(a, chunk, b, lh, row);
        if (c0 == 0) a.stat[at] = st;
#pragma unroll
        for (int i = 0; i < CH; ++i) a.part[at * D + c0 + i] = o[i];
      }
    }
  }
}

}  // namespace

constexpr int64_t kWhole = 4096, kCus = 256;
constexpr int64_t kStreamed = 256 << 20;  // bytes of a cache that the chip's caches do not hold

// Chunks: merging costs a launch (4 us) and, for each row and chunk, 4 d + 8 bytes written and read.
//  - Rows of one or two tiles (decoding, drafts): chunks of 4096 tokens where the (sequence, head) pairs occupy
//    every CU (32 sequences of 8 heads and 2049 to 2548 tokens: 27.2 us whole, 29.9 in chunks of 640); fewer pairs
//    get about 1024 workgroups, in chunks of 512 at least (one sequence of 13215, 8 heads: 11.1 us at 512, 13.5
//    at 1024, 25.9 at 4096; two of 262144 and 131073: 78.0 us at 4096, 92.1 at 1024, 94.1 at 8192), unless
//    what the idle CUs would take, n (1 - pairs / CUs), is less than the split costs: about 960 tokens of a CU with
//    one tile, 640 with two (8 heads; split and whole: one sequence of 520 tokens 8.5 and 7.3 us, of 1024 9.0 and
//    9.2; 8 of 800 9.4 and 8.6, of 1400 10.0 and 11.0; 17 of 2048 15.9 and 14.6, of 4096 22.8 and 23.4; 25 of 2600
//    21.9 and 17.6, and with lengths down to a tenth of that 18.8 and 17.3; two tiles: 8 of 1024 12.8 and 14.2, 20
//    of 1024 18.2 and 15.1).
//    Whole sequences of at most two workgroups a CU take eight waves (those 32 sequences: 26.2 us with four, 23.4
//    with eight, the append before it 5.8 of them; 64 of their lengths: 35.0 and 36.3; 64 of 6K to 32K tokens in
//    chunks: 235 and 249).
//  - Four tiles (prompts): the least cost of the busiest CU, in blocks of the cache: those of its workgroups (0.3 us
//    each; with one workgroup a CU half as much again), and, where there are chunks, 16 a workgroup for its partial
//    rows and 6 for the merge.  Measured with 32 query, 8 KV heads: 256 new tokens against 4096 in 4 chunks 36 us, in
//    2 40, in 8 50; 512 against 1024 whole 22, in 2 29; 1024 against 4096 whole 83, in 2 100; 64 against 1024 in 2 18,
//    whole 21.
// All of this at d = 128.  At d = 64 a block takes two thirds of the time, and the same choices are the better ones (17
// sequences of 2048 11.5 us whole, 13.0 split; 25 of 2600 13.7 and 17.2; those 32 with four waves 16.5, with eight 13.7;
// 20 of 1024 with two tiles 12.1 whole, 14.2 split; 256 new against 4096 in 4 27.2, in 2 31.0, in 8 34.8; 64 against 1024
// in 2 14.2, whole 16.6) but near a border (one sequence of 1024 9.1 split, 7.8 whole; 8 of 1400 9.4 and 8.9).
//
// max_len and max_new stand for every sequence, and a call pays for what they allow beyond what its sequences hold: those 32
// sequences, alone, take 19 us with a bound of 2548 or 4096, 32 with 8192 (chunks: four waves and a merge; streamed), 55
// with 32768, 64 with 131072 (workgroups that end at once).  Decoding sequences beside a prompt's chunk take the chunk's
// row groups and are not split: 15 of 8192 beside 1024 new tokens against 4096 199 us, apart 46 and 84; 63 of them 538,
// apart 149 and 84 (bound 32768).
CachePlan cache_plan(int32_t L, int32_t Hq, int32_t Hkv, int32_t head_dim, int32_t batch, int32_t max_new,
                     int32_t max_len) {
  constexpr int64_t kUnit = 128;  // tokens: a block for each of four waves
  constexpr int64_t kLeast = 512, kWorkgroups = 1024;
  constexpr int64_t kMost = 8;    // workgroups a CU
  CachePlan p;
  const int64_t rows = (int64_t)(Hq / Hkv) * max_new;
  p.tiles = rows <= 16 ? 1 : rows <= 32 ? 2 : 4;
  p.row_groups = (int32_t)((rows + 16 * p.tiles - 1) / (16 * p.tiles));
  const int64_t heads = (int64_t)L * Hkv * batch, units = heads * p.row_groups;
  const int64_t n = max_len, finest = (n + kLeast - 1) / kLeast, whole = (n + kWhole - 1) / kWhole;
  int64_t chunks;
  if (p.tiles == 4) {
    int64_t least = 0;
    chunks = 0;
    for (int64_t w = 0; w <= kMost; ++w) {  // whole, and the most chunks of w workgroups a CU
      const int64_t c = w == 0 ? 1 : std::min(finest, w * kCus / units);
      if (c <= chunks) continue;
      const int64_t each = (units * c + kCus - 1) / kCus, blocks = each * ((n + c * kCacheBlock - 1) / (c * kCacheBlock));
      const int64_t cost = (each == 1 ? blocks * 3 / 2 : blocks) + (c == 1 ? 0 : 6 + 16 * each);
      if (chunks != 0 && cost >= least) continue;
      chunks = c;
      least = cost;
    }
  } else {
    const bool few_idle = n * (kCus - units) <= (p.tiles == 1 ? 960 : 640) * kCus;
    chunks = few_idle ? whole : std::max(whole, std::min(finest, (kWorkgroups + units - 1) / units));
  }
  p.chunk = (int32_t)(((n + chunks - 1) / chunks + kUnit - 1) / kUnit * kUnit);
  p.chunks = (int32_t)((n + p.chunk - 1) / p.chunk);
  // Partial rows, heads * rows * chunks.  One or two tiles: rows <= 32 and chunks <= max(whole, kWorkgroups / heads + 1), so
  // at most 32 (kWorkgroups + heads * whole).  Four: heads * rows <= 64 units and, where there are chunks, chunks <=
  // kMost * kCus / units.  Both bounds in one, which grows with every argument, so a buffer for the longest call serves
  // the others.
  static_assert(32 * kWorkgroups <= 64 * kMost * kCus);
  const int64_t partials = finest == 1 ? 0 : std::min(heads * rows * finest, 64 * kMost * kCus + 32 * heads * whole);
  p.waves = p.tiles == 1 && p.chunks == 1 && units <= 2 * kCus ? 8 : 4;
  p.once = p.row_groups == 1 &&
           (double)heads * max_len * (double)(cache_block_bytes(head_dim) / kCacheBlock) > (double)kStreamed;
  p.stat_off = 0;
  p.o_off = ((size_t)partials * sizeof(float2) + 255) / 256 * 256;
  p.total = p.o_off + (size_t)partials * head_dim * sizeof(float);
  return p;
}

namespace {

template <int D, int NR, int W>
void launch_part(const CacheAttnArgs& a, dim3 grid, hipStream_t stream) {
  // (eight waves: at most 2 kCus whole sequences, which at d = 64 are never that many bytes)
  constexpr bool kMayStream = W == 4 || 2 * kCus * kWhole * (CacheBlock<D>::kBytes / kCacheBlock) > kStreamed;
  if (kMayStream && a.once)
    hipLaunchKernelGGL((k_cache_attention<D, NR, W, kMayStream>), grid, dim3(64 * W), 0, stream, a);
  else
    hipLaunchKernelGGL((k_cache_attention<D, NR, W, false>), grid, dim3(64 * W), 0, stream, a);
}

template <int D>
hipError_t launch_attention(const CacheAttnArgs& a, hipStream_t stream) {
  const unsigned heads = (unsigned)(a.c.L * a.c.Hkv), batch = (unsigned)a.c.batch;
  const dim3 grid(heads * a.row_groups * a.chunks, batch);
  if (a.tiles == 1 && a.waves == 8) launch_part<D, 1, 8>(a, grid, stream);
  else if (a.tiles == 1) launch_part<D, 1, 4>(a, grid, stream);
  else if (a.tiles == 2) launch_part<D, 2, 4>(a, grid, stream);
  else launch_part<D, 4, 4>(a, grid, stream);
  const hipError_t e = hipGetLastError();
  if (e != hipSuccess || a.chunks == 1) return e;
  const unsigned rows = heads * a.row_groups * a.tiles * 16;  // 16 a tile
  if (a.chunks >= 8)
    hipLaunchKernelGGL((k_cache_merge<D, 4>), dim3(rows, batch), dim3(kMergeThreads), 0, stream, a);
  else
    hipLaunchKernelGGL((k_cache_merge<D, 1>), dim3(rows / 4, batch), dim3(kMergeThreads), 0, stream, a);
  return hipGetLastError();
}

}  // namespace

hipError_t launch_cache_attention(const CacheAttnArgs& a, int head_dim, hipStream_t stream) {
  return head_dim == 128 ? launch_attention<128>(a, stream) : launch_attention<64>(a, stream);
}

}  // namespace tp

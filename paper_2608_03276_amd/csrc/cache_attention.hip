// Attention over the paged 4-bit cache (tp_cache_attention): the newest tokens of each sequence, from one
// (decoding) to a prompt's chunk, against all its tokens.
//
// A workgroup takes 16 to 64 query rows of one (sequence, KV head) (rows: new token, then query head of the
// group) and one chunk of the context; its four waves take a quarter of the chunk's blocks each, with the
// softmax's running maximum and sum in one pass, and join at the end through LDS.  Where a call has several
// chunks, their (maximum, sum, output) go to the workspace and k_cache_merge joins them.
//
// Products on v_mfma_f32_16x16x32_f16, both with the cache as the A operand, so that a lane's column is one
// query row from the scores to the output and the weights never leave their registers:
//   scores  S^T = K Q^T: one product per group of 32 channels; its result times the group's scale is summed
//           in fp32;
//   output  O^T += V^T P^T, with the values' scales multiplied into the weights P.
// Codes become fp16 operands by bit operations on pairs: 0x6400 | u is 1024 + u for a 4-bit number u = c + 8,
// and one packed fp16 operation more gives c exactly.  fp16 holds queries exactly once a row is brought near
// 2^14 by a power of two (a bf16 number has 8 significant bits, fp16 11; what lies 2^28 below the row's largest
// channel is off by 2^-39 of that one), and keeps the weights' rounding, 2^-11, below the output's (with bf16
// operands the output's error was 1.4 times that of its own rounding).
//
// The running reference m of a row bounds the weights that are rounded, p * scale of the value, not p alone:
// p = exp2(x - m) and the sum of the p's are fp32, in which the reference may be anywhere.
#include <algorithm>

#include "cache_block.h"

namespace tp {
namespace {

typedef __bf16 bf16x2 __attribute__((ext_vector_type(2)));
typedef _Float16 f16x8 __attribute__((ext_vector_type(8)));
typedef _Float16 f16x2 __attribute__((ext_vector_type(2)));
typedef unsigned short u16x2 __attribute__((ext_vector_type(2)));
typedef uint32_t u32x2 __attribute__((ext_vector_type(2)));
typedef uint32_t u32x4 __attribute__((ext_vector_type(4)));
typedef float f32x4 __attribute__((ext_vector_type(4)));

constexpr int kAttnThreads = 256;
constexpr int kAttnWaves = kAttnThreads / 64;
constexpr float kNoMax = -3.402823466e38f;  // (maximum, sum) of nothing is (kNoMax, 0): joining it changes nothing
constexpr float kLn2 = 0.6931471805599453f;
// A row's reference is set so that its largest weight is 2^kSet, and raised when one exceeds 2^kLimit (fp16
// ends below 2^16): most blocks skip the rescaling and the reduction across lanes, and weights down to
// 2^-22 of the largest are normal fp16 numbers.
constexpr float kSet = 8.0f, kLimit = 16384.0f;
// Scales below 2^-60 count as that in the reference, and sums of p above 2^74 raise it too, so that tokens
// with tiny or zero values cannot overflow the sum.
constexpr float kLeastScale = 0x1p-60f;

// Key scales as fp16 numbers: the largest of a block is set to exponent field 24 (2^9), and the setting is kept
// while the largest of a block has field 14 to 27 (a code times a scale stays below 2^16).
constexpr int kScaleSet = 24, kScaleLow = 14 << 7, kScaleHigh = 28 << 7;

union Frag {
  uint32_t w[4];
  f16x8 h;
};

__device__ inline f32x4 mfma(const Frag& a, const Frag& b, const f32x4& c) {
  return __builtin_amdgcn_mfma_f32_16x16x32_f16(a.h, b.h, c, 0, 0, 0);
}
__device__ inline uint32_t pack_h(float lo, float hi) {
  const f16x2 two = {(_Float16)lo, (_Float16)hi};
  return __builtin_bit_cast(uint32_t, two);
}

__device__ inline u16x2 pair(uint32_t w) { return __builtin_bit_cast(u16x2, w); }
__device__ inline u16x2 max_pair(u16x2 a, u16x2 b) { return __builtin_elementwise_max(a, b); }

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

// The keys that a group of query rows sees, and the chunks they take.
struct RowGroup {
  int row0, rows;      // the group's first row, and the sequence's rows
  int before;          // tokens before the step's (negative: the sequence holds fewer than the step)
  int keys;            // keys of the group's last row: chunk c has some where c * chunk < keys
};
__device__ inline RowGroup row_group(const CacheAttnArgs& a, const StepSeq& q, int group, int width) {
  RowGroup r;
  r.row0 = group * width;
  r.rows = q.count * (int)a.R.d;
  r.before = q.len - q.count;
  r.keys = __builtin_amdgcn_readfirstlane(max(0, r.before + a.R.div(max(min(r.rows, r.row0 + width) - 1, 0)) + 1));
  return r;
}

template <int D, int NR>
__global__ __launch_bounds__(kAttnThreads, NR == 1 ? 4 : NR == 2 ? 2 : 1) void k_cache_attention(CacheAttnArgs a) {
  using B = CacheBlock<D>;
  constexpr int KS = D / 32;  // products of a score: channels in steps of 32
  constexpr int ND = D / 16;  // output tiles: channels in steps of 16
  constexpr int kStride = D + 4;
  __shared__ float lds_o[kAttnWaves][16][kStride];
  __shared__ float2 lds_stat[kAttnWaves][16 * NR];

  const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane((int)threadIdx.x >> 6);
  const int g = lane >> 4, n = lane & 15;
  const int rest = a.heads.div((int)blockIdx.x), lh = a.heads.mod((int)blockIdx.x, rest);
  const int layer = a.by_Hkv.div(lh), head = a.by_Hkv.mod(lh, layer);
  const int chunk = a.by_groups.div(rest), group = a.by_groups.mod(rest, chunk);
  const int b = blockIdx.y;
  // the chunk's pages, one a lane (a chunk has at most 64)
  const int page0 = (chunk * a.chunk / kCacheBlock) >> a.c.page_shift;
  int pages = page0 + lane < a.c.max_pages ? a.c.table[(int64_t)b * a.c.max_pages + page0 + lane] : -1;
  const StepSeq q = step_sequence(a.c, a.s, b);
  const RowGroup rg = row_group(a, q, group, 16 * NR);
  if (rg.row0 >= rg.rows || (chunk > 0 && chunk * a.chunk >= rg.keys)) return;
  if (pages >= a.c.num_pages) pages = -1;

  Frag qf[NR][KS];
  int shift[NR];    // the power of two that the row was multiplied by
  float scale[NR];  // softmax_scale * log2(e), less that power and the key scales'
  int seen[NR];     // keys of the lane's row
#pragma unroll
  for (int r = 0; r < NR; ++r) {
    const int row = rg.row0 + r * 16 + n;
    const int t = a.R.div(row);
    const bool in = row < rg.rows;
    seen[r] = in ? rg.before + t + 1 : 0;
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
    top = max(top, (uint32_t)__shfl_xor((int)top, 16));
    top = max(top, (uint32_t)__shfl_xor((int)top, 32));
    const int e = 15 - __builtin_amdgcn_frexp_expf(__uint_as_float(top << 16));  // the largest comes to [2^14, 2^15)
    shift[r] = e;
    scale[r] = __builtin_amdgcn_ldexpf(a.scale_log2, -112 - e);
#pragma unroll
    for (int s = 0; s < KS; ++s) {
      const uint32_t w[4] = {x[s].x, x[s].y, x[s].z, x[s].w};
#pragma unroll
      for (int i = 0; i < 4; ++i)
        qf[r][s].w[i] = pack_h(__builtin_amdgcn_ldexpf(__uint_as_float(w[i] << 16), e),
                               __builtin_amdgcn_ldexpf(__uint_as_float(w[i] & 0xFFFF0000u), e));
    }
  }

  uint32_t magic = 0x64006400u;
  asm("" : "+v"(magic));

  f32x4 acc[NR][ND];
  float m[NR], l[NR];
#pragma unroll
  for (int r = 0; r < NR; ++r) {
    m[r] = kNoMax;
    l[r] = 0.0f;
#pragma unroll
    for (int x = 0; x < ND; ++x) acc[r][x] = (f32x4){0, 0, 0, 0};
  }

  const int key0 = chunk * a.chunk, key1 = min(rg.keys, key0 + a.chunk);
  const int j0 = key0 / kCacheBlock + wave, j1 = (key1 + kCacheBlock - 1) / kCacheBlock;  // every fourth block
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
        kw[u] = __builtin_amdgcn_raw_buffer_load_b128(blk, at_key, B::kKeys + u * 8 * D, 0);
        ks[u] = __builtin_amdgcn_raw_buffer_load_b64(blk, at_key_scale, B::kKeyScales + u * D, 0);
      } else {
        const u32x2 w = __builtin_amdgcn_raw_buffer_load_b64(blk, at_key, B::kKeys + u * 8 * D, 0);
        kw[u] = (u32x4){w.x, w.y, 0, 0};
        ks[u] = (u32x2){__builtin_amdgcn_raw_buffer_load_b32(blk, at_key_scale, B::kKeyScales + u * D, 0), 0};
      }
    }
  };
  const auto load_values = [&](__amdgpu_buffer_rsrc_t blk) {
#pragma unroll
    for (int x = 0; x < ND / 4; ++x) vw[x] = __builtin_amdgcn_raw_buffer_load_b128(blk, at_value, B::kValues + x * 1024, 0);
#pragma unroll
    for (int u = 0; u < 2; ++u) vs[u] = __builtin_amdgcn_raw_buffer_load_b128(blk, at_value_scale, B::kValueScales + u * 64, 0);
  };
  if (j0 < j1) {
    const auto blk = block_at(j0);
    load_keys(blk);
    load_values(blk);
  }
  int bias = 0;  // bf16 bits taken off a key scale: it becomes an fp16 number times 2^(bias / 128 - 112)
  for (int j = j0; j < j1; j += kAttnWaves) {
    const bool missing = page_of(j) < 0;
    const bool masked = missing || (j + 1) * kCacheBlock > all_seen;
    if (masked) {  // scales of slots that no row sees may be anything
#pragma unroll
      for (int u = 0; u < 2; ++u)
        if (missing || j * kCacheBlock + u * 16 + n >= rg.keys) ks[u] = (u32x2){0, 0};
    }
    // Key scales to fp16: bf16 bits, with the exponent brought into range and the mantissa moved by 3 bits.
    const u16x2 top2 = max_pair(max_pair(pair(ks[0].x), pair(ks[1].x)), max_pair(pair(ks[0].y), pair(ks[1].y)));
    const int most = max((int)top2.x, (int)top2.y);
    if (__builtin_amdgcn_ballot_w64(most - bias >= kScaleHigh) != 0 ||
        (bias > 0 && __builtin_amdgcn_ballot_w64(most - bias >= kScaleLow) == 0)) {
      int all = most;
#pragma unroll
      for (int i = 1; i < 64; i *= 2) all = max(all, __shfl_xor(all, i));
      bias = __builtin_amdgcn_readfirstlane(max((all >> 7) - kScaleSet, 0) << 7);
#pragma unroll
      for (int r = 0; r < NR; ++r) scale[r] = __builtin_amdgcn_ldexpf(a.scale_log2, (bias >> 7) - 112 - shift[r]);
    }
    const u16x2 off = {(unsigned short)bias, (unsigned short)bias};
    f32x4 xs[2][NR];
#pragma unroll
    for (int u = 0; u < 2; ++u) {
      f16x2 sc[KS / 2];
#pragma unroll
      for (int i = 0; i < KS / 2; ++i)
        sc[i] = __builtin_bit_cast(f16x2, __builtin_elementwise_sub_sat(pair(ks[u][i]), off) << 3);
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
        for (int r = 0; r < NR; ++r) xs[u][r] = mfma(k, qf[r][s], xs[u][r]);
      }
    }
    // (after the last block, that block once more: no branch, so the registers stay in place)
    const auto next = block_at(j + kAttnWaves < j1 ? j + kAttnWaves : j);
    __builtin_amdgcn_sched_barrier(0);
    load_keys(next);

    Frag pf[NR];
#pragma unroll
    for (int r = 0; r < NR; ++r) {
      float x[8], w[8];
#pragma unroll
      for (int i = 0; i < 8; ++i) {
        x[i] = xs[i >> 2][r][i & 3] * scale[r];
        w[i] = __uint_as_float(vs[i >> 2][i & 3]);
      }
      if (masked) {
#pragma unroll
        for (int i = 0; i < 8; ++i) {
          const bool out = missing || j * kCacheBlock + (i >> 2) * 16 + g * 4 + (i & 3) >= seen[r];
          x[i] = out ? -INFINITY : x[i];
          w[i] = out ? 0.0f : w[i];
        }
      }
      float p[8], sum, top;
      const auto weigh = [&] {
        sum = top = 0.0f;
#pragma unroll
        for (int i = 0; i < 8; ++i) {
          p[i] = __builtin_amdgcn_exp2f(x[i] - m[r]);
          sum += p[i];
          p[i] *= w[i];
          top = fmaxf(top, p[i]);
        }
      };
      weigh();
      if (__builtin_amdgcn_ballot_w64(fmaxf(top, sum * kLeastScale) > kLimit) != 0) {
        float next = kNoMax;
#pragma unroll
        for (int i = 0; i < 8; ++i)  // (of an unseen slot: -infinity)
          next = fmaxf(next, x[i] + __builtin_amdgcn_logf(fmaxf(w[i], kLeastScale)) - kSet);
        next = fmaxf(next, __shfl_xor(next, 16));
        next = fmaxf(next, __shfl_xor(next, 32));
        next = fmaxf(next, m[r]);
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

  // join the four waves
#pragma unroll
  for (int r = 0; r < NR; ++r) {
    l[r] += __shfl_xor(l[r], 16);
    l[r] += __shfl_xor(l[r], 32);
    if (g == 0) lds_stat[wave][r * 16 + n] = make_float2(m[r], l[r]);
  }
  __syncthreads();
#pragma unroll
  for (int r = 0; r < NR; ++r) {
    float top = kNoMax;
#pragma unroll
    for (int w = 0; w < kAttnWaves; ++w) top = fmaxf(top, lds_stat[w][r * 16 + n].x);
    const float f = __builtin_amdgcn_exp2f(m[r] - top);
    if (r > 0) __syncthreads();
#pragma unroll
    for (int x = 0; x < ND; ++x) {
      const f32x4 o = acc[r][x] * f;
      *(f32x4*)&lds_o[wave][n][x * 16 + g * 4] = o;
    }
    __syncthreads();
    // a row's channels by 16 threads
    const int row16 = threadIdx.x >> 4, c0 = (threadIdx.x & 15) * (D / 16);
    const int row = rg.row0 + r * 16 + row16;
    if (row < rg.rows) {
      float2 st = make_float2(kNoMax, 0.0f);
#pragma unroll
      for (int w = 0; w < kAttnWaves; ++w) st.x = fmaxf(st.x, lds_stat[w][r * 16 + row16].x);
#pragma unroll
      for (int w = 0; w < kAttnWaves; ++w) {
        const float2 s = lds_stat[w][r * 16 + row16];
        st.y += s.y * __builtin_amdgcn_exp2f(s.x - st.x);
      }
      float o[D / 16];
#pragma unroll
      for (int i = 0; i < D / 16; ++i) {
        o[i] = 0.0f;
#pragma unroll
        for (int w = 0; w < kAttnWaves; ++w) o[i] += lds_o[w][row16][c0 + i];
      }
      const int t = a.R.div(row), hq = head * (int)a.R.d + a.R.mod(row, t);
      const int64_t token = q.row + t;
      if (rg.keys <= a.chunk) {  // the only chunk
        const float inv = st.y > 0.0f ? 1.0f / st.y : 0.0f;
        uint16_t* to = a.o.data + layer * a.o.layer + token * a.o.token + hq * a.o.head + c0;
#pragma unroll
        for (int i = 0; i < D / 16; i += 2) {
          const bf16x2 two = {(__bf16)(o[i] * inv), (__bf16)(o[i + 1] * inv)};
          *(bf16x2*)(to + i) = two;
        }
        if (a.lse != nullptr && (threadIdx.x & 15) == 0)
          a.lse[((int64_t)layer * a.Hq + hq) * a.s.total + token] =
              st.y > 0.0f ? (st.x + __builtin_amdgcn_logf(st.y)) * kLn2 : -INFINITY;
      } else {
        const int64_t rows = (int64_t)a.c.L * a.s.total * a.Hq;
        const int64_t at = chunk * rows + (layer * (int64_t)a.s.total + token) * a.Hq + hq;
        if ((threadIdx.x & 15) == 0) a.stat[at] = st;
#pragma unroll
        for (int i = 0; i < D / 16; i += 4) *(f32x4*)(a.part + at * D + c0 + i) = (f32x4){o[i], o[i + 1], o[i + 2], o[i + 3]};
      }
    }
  }
}

// Joins the chunks of a row: one wave each.
template <int D>
__global__ __launch_bounds__(kAttnThreads) void k_cache_merge(CacheAttnArgs a) {
  constexpr int CH = D / 64;  // channels of a lane
  const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
  const int width = 16 * a.tiles;
  const int rest = a.heads.div((int)blockIdx.x), lh = a.heads.mod((int)blockIdx.x, rest);
  const int layer = a.by_Hkv.div(lh), head = a.by_Hkv.mod(lh, layer);
  const int b = blockIdx.y;
  const StepSeq q = step_sequence(a.c, a.s, b);
  const int row = rest * kAttnWaves + wave;
  const RowGroup rg = row_group(a, q, row / width, width);
  if (row >= rg.rows || rg.keys <= a.chunk) return;
  const int active = a.by_chunk.div(rg.keys + a.chunk - 1);
  const int t = a.R.div(row), hq = head * (int)a.R.d + a.R.mod(row, t);
  const int64_t token = q.row + t;
  const int64_t rows = (int64_t)a.c.L * a.s.total * a.Hq;
  const int64_t at = (layer * (int64_t)a.s.total + token) * a.Hq + hq;
  float top = kNoMax;
  for (int c = lane; c < active; c += 64) top = fmaxf(top, a.stat[c * rows + at].x);
#pragma unroll
  for (int s = 1; s < 64; s *= 2) top = fmaxf(top, __shfl_xor(top, s));
  float sum = 0.0f, o[CH] = {};
#pragma unroll 4
  for (int c = 0; c < active; ++c) {
    const float2 st = a.stat[c * rows + at];
    const float f = __builtin_amdgcn_exp2f(st.x - top);
    sum += st.y * f;
    const float* p = a.part + (c * rows + at) * D + lane * CH;
#pragma unroll
    for (int i = 0; i < CH; ++i) o[i] = fmaf(p[i], f, o[i]);
  }
  const float inv = sum > 0.0f ? 1.0f / sum : 0.0f;
  uint16_t* to = a.o.data + layer * a.o.layer + token * a.o.token + hq * a.o.head + lane * CH;
#pragma unroll
  for (int i = 0; i < CH; ++i) to[i] = __builtin_bit_cast(uint16_t, (__bf16)(o[i] * inv));
  if (a.lse != nullptr && lane == 0)
    a.lse[((int64_t)layer * a.Hq + hq) * a.s.total + token] =
        sum > 0.0f ? (top + __builtin_amdgcn_logf(sum)) * kLn2 : -INFINITY;
}

}  // namespace

CachePlan cache_plan(int32_t L, int32_t Hq, int32_t Hkv, int32_t head_dim, int32_t page_tokens, int32_t batch,
                     int32_t total, int32_t max_new, int32_t max_len) {
  constexpr int64_t kUnit = 32 * kAttnWaves;  // tokens: a block for each wave
  constexpr int64_t kWorkgroups = 1024;       // four for every CU
  const int64_t kMost = std::min(64 * page_tokens, 8192);  // tokens: a chunk's pages fit a wave's lanes
  CachePlan p;
  const int64_t rows = (int64_t)(Hq / Hkv) * max_new;
  p.tiles = rows <= 16 ? 1 : rows <= 32 ? 2 : 4;
  p.row_groups = (int32_t)((rows + 16 * p.tiles - 1) / (16 * p.tiles));
  const int64_t units = (int64_t)L * Hkv * batch * p.row_groups;
  const int64_t all_rows = (int64_t)L * Hq * total;
  // The workspace holds a partial result of every row for each chunk of the longest allowed length, or as
  // many as the chunks of kWorkgroups workgroups of 64 rows give: a bound that grows with every argument.
  // The chunks stay within it.
  const int64_t least = (max_len + kMost - 1) / kMost;
  const int64_t finest = (max_len + kUnit - 1) / kUnit;
  int64_t partials = std::max(all_rows * least, std::min(all_rows * finest, all_rows + 64 * kWorkgroups));
  int64_t chunks = std::max(least, std::min(finest, (kWorkgroups + units - 1) / units));
  chunks = std::max<int64_t>(least, std::min(chunks, partials / all_rows));
  p.chunk = (int32_t)(((max_len + chunks - 1) / chunks + kUnit - 1) / kUnit * kUnit);
  p.chunks = (int32_t)((max_len + p.chunk - 1) / p.chunk);
  if (finest == 1) partials = 0;  // one chunk whatever the plan
  p.stat_off = 0;
  p.o_off = ((size_t)partials * sizeof(float2) + 255) / 256 * 256;
  p.total = p.o_off + (size_t)partials * head_dim * sizeof(float);
  return p;
}

hipError_t launch_cache_attention(const CacheAttnArgs& a, int head_dim, hipStream_t stream) {
  const int heads = a.c.L * a.c.Hkv;
  const dim3 grid((unsigned)(heads * a.row_groups * a.chunks), (unsigned)a.c.batch);
#define TP_CACHE_ATTENTION(D_, NR_) \
  hipLaunchKernelGGL((k_cache_attention<D_, NR_>), grid, dim3(kAttnThreads), 0, stream, a)
  if (head_dim == 128) {
    if (a.tiles == 1) TP_CACHE_ATTENTION(128, 1);
    else if (a.tiles == 2) TP_CACHE_ATTENTION(128, 2);
    else TP_CACHE_ATTENTION(128, 4);
  } else {
    if (a.tiles == 1) TP_CACHE_ATTENTION(64, 1);
    else if (a.tiles == 2) TP_CACHE_ATTENTION(64, 2);
    else TP_CACHE_ATTENTION(64, 4);
  }
#undef TP_CACHE_ATTENTION
  hipError_t e = hipGetLastError();
  if (e != hipSuccess || a.chunks == 1) return e;
  const dim3 merge((unsigned)(heads * a.row_groups * a.tiles * 16 / kAttnWaves), (unsigned)a.c.batch);
  if (head_dim == 128)
    hipLaunchKernelGGL(k_cache_merge<128>, merge, dim3(kAttnThreads), 0, stream, a);
  else
    hipLaunchKernelGGL(k_cache_merge<64>, merge, dim3(kAttnThreads), 0, stream, a);
  return hipGetLastError();
}

}  // namespace tp

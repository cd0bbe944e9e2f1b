// Rows into and out of the paged 8-bit cache: tp_cache8_append, tp_cache8_load, tp_cache8_read.
//
// One workgroup handles one block (32 tokens of one head): d/8 lanes hold a row, 16 bytes each.  The block's keys
// share a scale, so a workgroup finds the largest magnitude of its new keys before it forms a code; where that is
// beyond the scale that the block has, the scale is raised by the least power of two that holds it and the codes of
// the earlier tokens are rounded again.  (A power of two: the error of an integer code is then at most the sum
// 1/2 (1 + 1/2 + 1/4 + ...) of a step however often the scale rises, and an e4m3 code keeps its significant bits.)
// A row's 8 codes are 8 bytes of the block's keys and single bytes of its values.  They go out by way of LDS, 16 bytes a
// lane, where the whole block is written (the keys written from registers: loads 464 us, so 453), and by themselves where
// it is not: nothing else is read or written of it.
//
// Measured at d = 128, 8 KV heads.  HBM bounds long calls: an append of 8191 and 5003 tokens with 64 query heads rotated moves
// 514 MB in 110 us, 4.7 TB/s; a load of 13107 tokens of 32 layers 2.17 GB in 429 to 453, 4.9; reading them back 2.59 GB in 500,
// 5.2 (a plain large copy 5.3 to 5.5, one with nontemporal loads and stores 6.2).
// Short ones take their launch and dependent loads (offsets, lengths, page, block's scale): 4.4 to 5.5 us.
#include "cache8_block.h"
#include "cache_rotate.h"
#include "quant_row.h"

namespace tp {
namespace {

constexpr int kRowsThreads = 256;
// An append of one token a sequence at d = 128 has a pass of 512 threads a block and rotates a token's queries in one or two:
// the chain of loads bounds it (64 sequences, 32 heads: 10.8 us, 256 threads 11.2; 64 heads 12.2, 13.6).  With more tokens 256
// threads take two passes, whose loads are in flight together (4 tokens a sequence: 15.3 -> 13.9 us).
constexpr int kOneThreads = 512;
// From this many query heads on (three passes of 256 threads and more) a token's query rows are loaded four passes ahead at
// d = 128: 13194 tokens of 64 heads in pairs 148 -> 132 us, in halves 158 -> 154; with 16 heads 81 -> 89 and 88 -> 98 (the
// registers leave fewer blocks in flight); at d = 64, 64 heads 88 -> 98.  Few tokens lose by it (two each of 64 sequences, 64
// heads: 15.2 -> 16.7), which the rule does not look at.
constexpr int kManyHeads = 33;

// In LDS: the 256 bytes of 16 tokens' keys that lanes of the same channels hold, so that channels begin in different banks.
constexpr int kKeyGroup = 256 + 16;

// Scales between which the corrected quotient below has normal numbers throughout.
constexpr float kLeastDivisor = 0x1p-70f, kMostDivisor = 0x1p100f;

// Low bytes of eight words.
__device__ inline uint2 low_bytes(const uint32_t (&c)[8]) {
  const uint32_t a = __builtin_amdgcn_perm(c[1], c[0], 0x0c0c0400u), b = __builtin_amdgcn_perm(c[3], c[2], 0x0c0c0400u);
  const uint32_t d = __builtin_amdgcn_perm(c[5], c[4], 0x0c0c0400u), e = __builtin_amdgcn_perm(c[7], c[6], 0x0c0c0400u);
  return make_uint2(__builtin_amdgcn_perm(b, a, 0x05040100u), __builtin_amdgcn_perm(e, d, 0x05040100u));
}

// The bytes of 8 bf16 values in the scale g (0 where g is): the code of the fp32 quotient, which a product with the
// reciprocal and one correction give (quant_row.h) where g is ordinary, and a division elsewhere.  Quotients are at
// most the format's largest code and an ulp.
template <bool FP8>
__device__ inline uint2 codes8(const uint4& x, float g) {
  const uint32_t w[4] = {x.x, x.y, x.z, x.w};
  const bool plain = g >= kLeastDivisor && g <= kMostDivisor;
  uint2 out;
  if (__builtin_amdgcn_ballot_w64(!plain) == 0) {
    const float y = 1.0f / g;
    if (FP8) return codes_fast_e4m3(w, g, y);
    uint32_t code[8];
    codes_fast<kQByte>(w, g, y, code);
    out = low_bytes(code);
  } else {
    uint32_t code[8];
    codes_divided(w, g, QuantFmt{!FP8, false, FP8 ? 448.0f : 127.0f}, code);
    out = low_bytes(code);
  }
  if (!FP8) out = make_uint2(out.x ^ 0x80808080u, out.y ^ 0x80808080u);
  return out;
}

// Four bytes of codes, in a scale 2^n times theirs.
template <bool FP8>
__device__ inline uint32_t coarser(uint32_t w, int n) {
  if (FP8) {
    float f[4] = {__builtin_amdgcn_cvt_f32_fp8((int)w, 0), __builtin_amdgcn_cvt_f32_fp8((int)w, 1),
                  __builtin_amdgcn_cvt_f32_fp8((int)w, 2), __builtin_amdgcn_cvt_f32_fp8((int)w, 3)};
#pragma unroll
    for (int i = 0; i < 4; ++i) f[i] = __builtin_amdgcn_ldexpf(f[i], -n);
    const int lo = __builtin_amdgcn_cvt_pk_fp8_f32(f[0], f[1], 0, false);
    return (uint32_t)__builtin_amdgcn_cvt_pk_fp8_f32(f[2], f[3], lo, true);
  }
  uint32_t out = 0;
#pragma unroll
  for (int i = 0; i < 4; ++i) {
    const int c = (int)((w >> (8 * i)) & 0xFFu) - 128;
    out |= ((uint32_t)(int)__builtin_rintf(__builtin_amdgcn_ldexpf((float)c, -n)) + 128u) << (8 * i);
  }
  return out;
}

// Eight codes of at most 4 bits, element 2 i in the low nibble of byte i (two's complement), as bytes c + 128.
__device__ inline uint2 widened(uint32_t w) {
  const uint32_t lo = w & 0x0F0F0F0Fu, hi = (w >> 4) & 0x0F0F0F0Fu;
  const uint32_t a = __builtin_amdgcn_perm(hi, lo, 0x05010400u), b = __builtin_amdgcn_perm(hi, lo, 0x07030602u);
  return make_uint2((a ^ 0x08080808u) + 0x78787878u, (b ^ 0x08080808u) + 0x78787878u);
}

// One token's query rows, kAhead passes of loads in flight.  The loads come first, then what decides whether they count.
template <int D, int T, int kAhead>
__device__ inline void rotate_query_rows(const CacheWriteArgs& a, int unit) {
  constexpr int LPT = D / 8, kHeads = T / LPT;
  const int layer = a.by_total.div(unit), row = a.by_total.mod(unit, layer);
  const int piece = threadIdx.x % LPT;
  const bool turn = rotates(a, piece);
  const int other = turn && !a.pairs ? partner(a, piece) : piece;
  const uint16_t* from = a.q.data + layer * a.q.layer + row * a.q.token;
  uint16_t* to = a.q_out.data + layer * a.q_out.layer + row * a.q_out.token;
  uint4 x[kAhead], y[kAhead];
  const auto load = [&](int h0) {
#pragma unroll
    for (int i = 0; i < kAhead; ++i) {
      const int h = h0 + i * kHeads + (int)threadIdx.x / LPT;
      x[i] = y[i] = make_uint4(0, 0, 0, 0);
      if (h >= a.Hq) continue;
      x[i] = *((const uint4*)(from + h * a.q.head) + piece);
      if (!a.pairs) y[i] = *((const uint4*)(from + h * a.q.head) + other);
    }
  };
  load(0);
  const int64_t pos = scalar_load(a.positions + row);
  if (pos < 0 || pos >= a.num_positions) return;
  Angles g = {};
  if (turn) g = load_angles(a, a.cos_sin + pos * a.rotary_dim, piece);
  if (a.s.offsets == nullptr ? row >= a.c.batch : !in_a_sequence(a.s, a.c.batch, row)) return;
  for (int h0 = 0;;) {
#pragma unroll
    for (int i = 0; i < kAhead; ++i) {
      const int h = h0 + i * kHeads + (int)threadIdx.x / LPT;
      if (h >= a.Hq) break;
      if (turn) x[i] = rotated(a.pairs, x[i], y[i], g);
      // (a row's lanes are of one wave and load before they store, so q_out may be q)
      *((uint4*)(to + h * a.q_out.head) + piece) = x[i];
    }
    h0 += kAhead * kHeads;
    if (h0 >= a.Hq) break;
    load(h0);
  }
}

template <int D, bool FP8, bool LOAD, int T, int AHEAD>
__global__ __launch_bounds__(T) void k_cache8_write(Cache8WriteArgs a, int kv_units) {
  using B = Cache8Block<D>;
  constexpr int LPT = D / 8;                         // lanes of a row
  constexpr int kPasses = kCacheBlock * LPT / T;
  constexpr int kStride = D + 8;                     // bytes of a row of value codes in LDS
  __shared__ alignas(16) uint8_t codes[kCacheBlock * kStride];
  __shared__ alignas(16) uint8_t keys[D / 8 * kKeyGroup];
  __shared__ uint32_t tops[T / 64];
  if (!LOAD && (int)blockIdx.x >= kv_units) {
    rotate_query_rows<D, T, AHEAD>(a, (int)blockIdx.x - kv_units);
    return;
  }
  const int rest = a.heads.div((int)blockIdx.x), lh = a.heads.mod((int)blockIdx.x, rest);
  const int layer = a.by_Hkv.div(lh), head = a.by_Hkv.mod(lh, layer);
  int b, j, len;
  int64_t row0;  // the source row of the sequence's token 0 (may be before the source's start)
  int start;     // the first token written
  if (LOAD) {
    b = blockIdx.y;
    j = rest;
    row0 = a.kept_off[b];
    start = 0;
    len = (int)(a.kept_off[b + 1] - row0);
  } else {
    b = a.by_blocks.div(rest);
    const StepSeq q = step_sequence(a.c, a.s, b);
    len = q.count == 0 ? 0 : q.len;
    row0 = (int64_t)q.row - (q.len - q.count);
    start = max(q.len - q.count, 0);
    j = (start >> 5) + a.by_blocks.mod(rest, b);
  }
  if (j * kCacheBlock >= len) return;
  const int32_t page = scalar_load(a.c.table + (int64_t)b * a.c.max_pages + (j >> a.c.page_shift));
  const bool turned = !LOAD && a.cos_sin != nullptr;
  const int piece = threadIdx.x % LPT;
  const bool turn = turned && rotates(a, piece);
  const int other = turn && !a.pairs ? partner(a, piece) : piece;

  // the lane's pieces of its rows
  uint4 kx[kPasses], ky[kPasses], vx[kPasses];
  uint2 vc[kPasses];
  float gamma[kPasses];
  int64_t pos[kPasses];
#pragma unroll
  for (int p = 0; p < kPasses; ++p) {
    const int token = j * kCacheBlock + p * (T / LPT) + (int)threadIdx.x / LPT;
    const int64_t row = row0 + token;
    kx[p] = ky[p] = vx[p] = make_uint4(0, 0, 0, 0);
    vc[p] = make_uint2(0, 0);
    gamma[p] = 0.0f;
    pos[p] = 0;
    if (token < start || token >= len) continue;
    const uint16_t* k = a.k.data + layer * a.k.layer + row * a.k.token + head * a.k.head;
    if (turned) pos[p] = a.positions[row];
    kx[p] = *((const uint4*)k + piece);
    if (turned) ky[p] = *((const uint4*)k + other);
    if (LOAD) {
      const int64_t at = (int64_t)lh * a.kept_off[a.c.batch] + row;
      if (!FP8 && a.nibbles) {
        vc[p] = widened(*((const uint32_t*)(a.v_q + at * (D / 2)) + piece));
      } else {
        vc[p] = *((const uint2*)(a.v_q + at * D) + piece);
        if (!FP8) vc[p] = make_uint2(vc[p].x ^ 0x80808080u, vc[p].y ^ 0x80808080u);
      }
      gamma[p] = a.v_scales[at];
    } else {
      vx[p] = *((const uint4*)(a.v.data + layer * a.v.layer + row * a.v.token + head * a.v.head) + piece);
    }
  }
  // the tokens that are written, the same in every wave
  uint32_t mask;
  {
    const int t = j * kCacheBlock + (int)(threadIdx.x & 63);
    bool in = (threadIdx.x & 63) < kCacheBlock && t >= start && t < len;
    if (turned && in) {
      const int64_t at = a.positions[row0 + t];
      in = at >= 0 && at < a.num_positions;
    }
    mask = (uint32_t)__builtin_amdgcn_ballot_w64(in);
  }
  if (mask == 0) return;
  uint8_t* blk = cache8_block<D>(a.c, layer, head, page, j);
  if (blk == nullptr) return;

  // Tokens of the block before the step's: their scale, and their codes in case it rises.
  const int before = LOAD ? 0 : max(start - j * kCacheBlock, 0);
  uint4* const old_at = (uint4*)(blk + B::kKeys) + threadIdx.x;
  const int old_token = (int)threadIdx.x / D * 16 + ((int)threadIdx.x & 15);  // (D vectors of 16 bytes a tile)
  const bool old_mine = threadIdx.x < 2 * D && old_token < before;
  float held = 0.0f;
  uint4 old = make_uint4(0, 0, 0, 0);
  if (before > 0) {
    held = *(const float*)(blk + B::kKeyScale);
    if (old_mine) old = *old_at;
  }

  uint32_t top = 0;
#pragma unroll
  for (int p = 0; p < kPasses; ++p) {
    const int slot = p * (T / LPT) + (int)threadIdx.x / LPT;
    const bool w = (mask >> slot) & 1u;
    if (__builtin_amdgcn_ballot_w64(w) == 0) continue;
    if (turned) {
      Angles g = {};
      if (turn && w) g = load_angles(a, a.cos_sin + pos[p] * a.rotary_dim, piece);
      const uint4 r = rotated(a.pairs, kx[p], ky[p], g);
      if (turn && w) kx[p] = r;
    }
    const uint32_t words[4] = {kx[p].x, kx[p].y, kx[p].z, kx[p].w};
    const uint32_t mine = row_absmax_bits<LPT>(words);
    if (w) top = max(top, mine);
  }
  // the largest of the wave's rows (every lane of a row has its row's)
  if (LPT == 8) top = max(top, (uint32_t)__builtin_amdgcn_update_dpp(0, (int)top, 0x140, 0xF, 0xF, false));
  top = max(top, (uint32_t)__shfl_xor((int)top, 16));
  top = max(top, (uint32_t)__shfl_xor((int)top, 32));
  if ((threadIdx.x & 63) == 0) tops[threadIdx.x / 64] = top;
  __syncthreads();
#pragma unroll
  for (int i = 0; i < T / 64; ++i) top = max(top, tops[i]);

  // the block's scale (one of 0, below it, infinite or NaN is none)
  const float want = __uint_as_float(top << 16) / (FP8 ? 448.0f : 127.0f);
  int up = 0;
  float scale = want;
  if (held > 0.0f && held < INFINITY) {
    if (want > held)
      up = __builtin_amdgcn_frexp_expf(want) - __builtin_amdgcn_frexp_expf(held) +
           (__builtin_amdgcn_frexp_mantf(want) > __builtin_amdgcn_frexp_mantf(held) ? 1 : 0);
    scale = __builtin_amdgcn_ldexpf(held, up);
    if (up > 0 && old_mine)
      *old_at = make_uint4(coarser<FP8>(old.x, up), coarser<FP8>(old.y, up), coarser<FP8>(old.z, up),
                           coarser<FP8>(old.w, up));
  }
  if (threadIdx.x == 0) *(float*)(blk + B::kKeyScale) = scale;

  const bool whole = mask == 0xFFFFFFFFu;
#pragma unroll
  for (int p = 0; p < kPasses; ++p) {
    const int slot = p * (T / LPT) + (int)threadIdx.x / LPT;
    const bool w = (mask >> slot) & 1u;
    if (__builtin_amdgcn_ballot_w64(w) == 0) continue;  // a wave without a token has nothing to quantise
    const uint2 kc = codes8<FP8>(kx[p], scale);
    if (!LOAD) {
      const uint32_t words[4] = {vx[p].x, vx[p].y, vx[p].z, vx[p].w};
      gamma[p] = __uint_as_float(row_absmax_bits<LPT>(words) << 16) / (FP8 ? 448.0f : 127.0f);
      vc[p] = codes8<FP8>(vx[p], w ? gamma[p] : 1.0f);  // (lanes without a token do not decide the wave's way)
    }
    if (!w) continue;
    const int at = key8_place<D>(slot, piece);
    if (whole)
      *(uint2*)(keys + (at >> 8) * kKeyGroup + (at & 255)) = kc;
    else
      *(uint2*)(blk + B::kKeys + at) = kc;
    if (piece == 0) *((float*)(blk + B::kValueScales) + slot) = gamma[p];
    if (whole) {
      *(uint2*)(codes + slot * kStride + piece * 8) = vc[p];
    } else {
#pragma unroll
      for (int i = 0; i < 8; ++i)
        blk[B::kValues + value8_place(slot, piece * 8 + i)] = (uint8_t)((i < 4 ? vc[p].x : vc[p].y) >> (8 * (i & 3)));
    }
  }
  if (!whole) return;
  __syncthreads();
  for (int i = threadIdx.x; i < 2 * D; i += T) {  // 16 bytes: two tiles' channels of the lane, of eight tokens each
    const int g = (i >> 4) & 3, x = (i >> 6) * 32 + (i & 15);
    uint32_t out[4] = {0, 0, 0, 0};
#pragma unroll
    for (int e = 0; e < 16; ++e) {
      const int token = ((e >> 2) & 1) * 16 + 4 * g + (e & 3);
      out[e >> 2] |= (uint32_t)codes[token * kStride + x + (e >> 3) * 16] << (8 * (e & 3));
    }
    *((uint4*)(blk + B::kValues) + i) = make_uint4(out[0], out[1], out[2], out[3]);
    *((uint4*)(blk + B::kKeys) + i) = *(const uint4*)(keys + (i >> 4) * kKeyGroup + (i & 15) * 16);
  }
}

// The numbers that four bytes of codes stand for.
template <bool FP8>
__device__ inline void numbers(uint32_t w, float* f) {
  if (FP8) {
    f[0] = __builtin_amdgcn_cvt_f32_fp8((int)w, 0);
    f[1] = __builtin_amdgcn_cvt_f32_fp8((int)w, 1);
    f[2] = __builtin_amdgcn_cvt_f32_fp8((int)w, 2);
    f[3] = __builtin_amdgcn_cvt_f32_fp8((int)w, 3);
  } else {
#pragma unroll
    for (int i = 0; i < 4; ++i) f[i] = (float)((w >> (8 * i)) & 0xFFu) - 128.0f;
  }
}

// Eight channels as c * scale in fp32, rounded to bf16.
__device__ inline uint4 held_row(const float (&c)[8], float scale) {
  return make_uint4(pack_bf16(c[0] * scale, c[1] * scale), pack_bf16(c[2] * scale, c[3] * scale),
                    pack_bf16(c[4] * scale, c[5] * scale), pack_bf16(c[6] * scale, c[7] * scale));
}

template <int D, bool FP8>
__global__ __launch_bounds__(kRowsThreads) void k_cache8_read(CacheReadArgs a) {
  using B = Cache8Block<D>;
  constexpr int LPT = D / 8, kPasses = kCacheBlock * LPT / kRowsThreads;
  constexpr int kStride = 1024 + 16;  // of 32 channels, so that their rows begin in different banks
  __shared__ alignas(16) uint8_t values[D / 32 * kStride];
  const int rest = a.heads.div((int)blockIdx.x), lh = a.heads.mod((int)blockIdx.x, rest), b = blockIdx.y;
  const int layer = a.by_Hkv.div(lh), head = a.by_Hkv.mod(lh, layer);
  const int64_t first = a.first[b], n = a.off[b + 1] - a.off[b];
  const int64_t j = (first >> 5) + rest;
  if (j * kCacheBlock >= first + n) return;
  const int32_t raw = scalar_load(a.c.lens + b);
  const int32_t len = raw < 0 || raw > a.c.max_len ? 0 : raw;
  const uint8_t* blk = nullptr;
  if (j * kCacheBlock < len)
    blk = cache8_block<D>(a.c, layer, head, scalar_load(a.c.table + (int64_t)b * a.c.max_pages + (j >> a.c.page_shift)),
                          (int)j);
  const int piece = threadIdx.x % LPT;
  uint2 kc[kPasses];
  float vs[kPasses], ks = 0.0f;
  if (blk != nullptr) {
    if (threadIdx.x < 2 * D)
      *(uint4*)(values + (threadIdx.x >> 6) * kStride + (threadIdx.x & 63) * 16) =
          *((const uint4*)(blk + B::kValues) + threadIdx.x);
    ks = *(const float*)(blk + B::kKeyScale);
#pragma unroll
    for (int p = 0; p < kPasses; ++p) {
      const int slot = p * (kRowsThreads / LPT) + (int)threadIdx.x / LPT;
      kc[p] = *(const uint2*)(blk + B::kKeys + key8_place<D>(slot, piece));
      vs[p] = *((const float*)(blk + B::kValueScales) + slot);
    }
  }
  __syncthreads();
#pragma unroll
  for (int p = 0; p < kPasses; ++p) {
    const int slot = p * (kRowsThreads / LPT) + (int)threadIdx.x / LPT;
    const int64_t t = j * kCacheBlock + slot;
    if (t < first || t >= first + n) continue;
    uint4 k = make_uint4(0, 0, 0, 0), v = k;
    if (blk != nullptr && t < len) {
      float c[8];
      numbers<FP8>(kc[p].x, c);
      numbers<FP8>(kc[p].y, c + 4);
      k = held_row(c, ks);
      uint32_t w[2] = {0, 0};
#pragma unroll
      for (int i = 0; i < 8; ++i) {
        const int at = value8_place(slot, piece * 8 + i);
        w[i >> 2] |= (uint32_t)values[(at >> 10) * kStride + (at & 1023)] << (8 * (i & 3));
      }
      numbers<FP8>(w[0], c);
      numbers<FP8>(w[1], c + 4);
      v = held_row(c, vs[p]);
    }
    const int64_t to = (int64_t)lh * a.off[a.c.batch] + a.off[b] + (t - first);
    *((uint4*)(a.k + to * D) + piece) = k;
    *((uint4*)(a.v + to * D) + piece) = v;
  }
}

// Divisors of the workgroups' numbers.
template <typename Args>
void set_heads(Args& a) {
  a.heads = Divisor::of((int64_t)a.c.L * a.c.Hkv);
  a.by_Hkv = Divisor::of(a.c.Hkv);
}

template <int D, bool LOAD, int T, int AHEAD>
void launch_write(const Cache8WriteArgs& a, dim3 grid, int units, hipStream_t stream) {
  if (a.fp8)
    hipLaunchKernelGGL((k_cache8_write<D, true, LOAD, T, AHEAD>), grid, dim3(T), 0, stream, a, units);
  else
    hipLaunchKernelGGL((k_cache8_write<D, false, LOAD, T, AHEAD>), grid, dim3(T), 0, stream, a, units);
}

}  // namespace

hipError_t launch_cache8_append(Cache8WriteArgs& a, int head_dim, hipStream_t stream) {
  const int units = a.c.L * a.c.Hkv * a.blocks * a.c.batch;
  set_heads(a);
  a.by_blocks = Divisor::of(a.blocks);
  a.by_total = Divisor::of(a.s.total);
  const dim3 grid((unsigned)units + (a.q.data != nullptr ? (unsigned)(a.c.L * a.s.total) : 0u));
  if (head_dim == 64) launch_write<64, false, kRowsThreads, 1>(a, grid, units, stream);
  else if (a.s.max_new == 1) launch_write<128, false, kOneThreads, 1>(a, grid, units, stream);
  else if (a.Hq >= kManyHeads) launch_write<128, false, kRowsThreads, 4>(a, grid, units, stream);
  else launch_write<128, false, kRowsThreads, 1>(a, grid, units, stream);
  return hipGetLastError();
}

hipError_t launch_cache8_load(Cache8WriteArgs& a, int head_dim, hipStream_t stream) {
  const int units = a.c.L * a.c.Hkv * a.blocks;
  const dim3 grid((unsigned)units, (unsigned)a.c.batch);
  set_heads(a);
  if (head_dim == 128) launch_write<128, true, kRowsThreads, 1>(a, grid, units, stream);
  else launch_write<64, true, kRowsThreads, 1>(a, grid, units, stream);
  return hipGetLastError();
}

hipError_t launch_cache8_read(CacheReadArgs& a, bool fp8, int head_dim, hipStream_t stream) {
  const dim3 grid((unsigned)(a.c.L * a.c.Hkv * a.blocks), (unsigned)a.c.batch);
  set_heads(a);
  if (head_dim == 128 && fp8) hipLaunchKernelGGL((k_cache8_read<128, true>), grid, dim3(kRowsThreads), 0, stream, a);
  else if (head_dim == 128) hipLaunchKernelGGL((k_cache8_read<128, false>), grid, dim3(kRowsThreads), 0, stream, a);
  else if (fp8) hipLaunchKernelGGL((k_cache8_read<64, true>), grid, dim3(kRowsThreads), 0, stream, a);
  else hipLaunchKernelGGL((k_cache8_read<64, false>), grid, dim3(kRowsThreads), 0, stream, a);
  return hipGetLastError();
}

}  // namespace tp

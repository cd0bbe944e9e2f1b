// Rows into and out of the paged 4-bit cache: tp_cache_append, tp_cache_load, tp_cache_read.
//
// One workgroup handles one block (32 tokens of one head): d/8 lanes hold a row, 16 bytes each.  The
// value codes of a block are transposed, since a word holds one channel of eight tokens: eight words of
// eight channels become eight words of eight tokens in registers (32 operations), and go out by way of LDS, 16
// bytes a lane.  A block of which only some tokens are written is read before and merged.  A block belongs to
// one workgroup of the launch, so nothing races.  Everything that a workgroup loads hangs on the sequence's
// offsets and length alone, but for the angles (on the positions) and the old values (on the page).
//
// Bound by HBM (d = 128): 13107 kept tokens of 32 layers and 8 heads into pages in 300 us (464 bytes a token and head,
// 5.2 TB/s) and back in 428 (652 bytes, 5.1 TB/s, four fifths of it writes); 12290 new tokens of 64 query and 8 KV
// heads in 105 us (4.5 TB/s).  A decoding step's append is latency: 64 sequences in 5.9 us.
#include "cache_block.h"
#include "quant_row.h"

namespace tp {
namespace {

constexpr int kRowsThreads = 256;
// Threads of a step's append, and where it is of more than one block a sequence: with one token the time is the chain
// of loads and the instructions fetched, so a block is one pass of 512 threads at d = 128 (64 sequences: 6.6 us; 256
// threads in two passes 7.2); long steps want loads in flight (12290 tokens of 64 heads: 222 us; 110).
constexpr int kFewThreads = 512, kFewTokens = 32;
constexpr float kMaxBf16 = 3.3895313892515355e38f;

// The nibble of element e (0..7) of a word.
__host__ __device__ constexpr int nibble_of(int e) { return (e >> 1) + 4 * (e & 1); }

__device__ inline float bf16_lo(uint32_t w) { return __uint_as_float(w << 16); }
__device__ inline float bf16_hi(uint32_t w) { return __uint_as_float(w & 0xFFFF0000u); }

__device__ inline uint32_t pack_bf16(float lo, float hi) {
  typedef __bf16 bf16x2 __attribute__((ext_vector_type(2)));
  const bf16x2 v = {(__bf16)lo, (__bf16)hi};
  return __builtin_bit_cast(uint32_t, v);
}

// Angles of 8 channels (of 4 pairs): cosines, and sines with the sign of the partner's term.
struct Angles {
  float c[8], s[8];
};

// The lane's part of a rotation: no angles where the piece is not rotated.
__device__ inline bool rotates(const CacheWriteArgs& a, int piece) { return piece * 8 < a.rotary_dim; }
// The piece whose channels are the partners' (half-split pairs).
__device__ inline int partner(const CacheWriteArgs& a, int piece) {
  const int half = a.rotary_dim / 16;
  return piece < half ? piece + half : piece - half;
}
__device__ inline Angles load_angles(const CacheWriteArgs& a, const float* cs, int piece) {
  const int half = a.rotary_dim / 2;
  Angles g;
  if (a.pairs) {
    const float4 c = *(const float4*)(cs + piece * 4), s = *(const float4*)(cs + half + piece * 4);
    const float cc[4] = {c.x, c.y, c.z, c.w}, ss[4] = {s.x, s.y, s.z, s.w};
#pragma unroll
    for (int i = 0; i < 8; ++i) {
      g.c[i] = cc[i / 2];
      g.s[i] = (i & 1) ? ss[i / 2] : -ss[i / 2];
    }
  } else {
    const bool first = piece * 8 < half;
    const int at = first ? piece * 8 : piece * 8 - half;
    const float4 c0 = *(const float4*)(cs + at), c1 = *(const float4*)(cs + at + 4);
    const float4 s0 = *(const float4*)(cs + half + at), s1 = *(const float4*)(cs + half + at + 4);
    const float cc[8] = {c0.x, c0.y, c0.z, c0.w, c1.x, c1.y, c1.z, c1.w};
    const float ss[8] = {s0.x, s0.y, s0.z, s0.w, s1.x, s1.y, s1.z, s1.w};
#pragma unroll
    for (int i = 0; i < 8; ++i) {
      g.c[i] = cc[i];
      g.s[i] = first ? -ss[i] : ss[i];
    }
  }
  return g;
}

// x c + y s in 64 bits (a product of a bf16 and an fp32 number is exact there), as the nearest fp32 number, for
// rounding to bf16; within its range, so that no rotation of finite rows gives an infinity.
__device__ inline float rotated64(float x, float y, float c, float s) {
  const double r = (double)x * (double)c + (double)y * (double)s;
  float f = (float)__builtin_fmax(__builtin_fmin(r, (double)kMaxBf16), -(double)kMaxBf16);
  asm("" : "+v"(f));  // (two roundings, not one to bf16: the compiler may not join them)
  return f;
}

// Eight channels x, rotated with their partners' y (for pairs of neighbours, y = x).  The fp32 result r is off by
// at most 2^-24 (|x c| + 2 |y s|), r - delta and r + delta by 2^-24 (|x c| + |y s|) more; delta is 3.1 * 2^-24
// (|x c| + |y s|), and 2^-147 for subnormal numbers.  Where r - delta and r + delta round to the same bf16 number, so do the
// exact value and the fp32 number next to it.  A wave with a
// channel where they do not (1 in 10, of 512 channels each) forms its channels in 64 bits, at six times the
// instructions.
__device__ inline uint4 rotated(bool pairs, const uint4& x4, const uint4& y4, const Angles& g) {
  const uint32_t xw[4] = {x4.x, x4.y, x4.z, x4.w}, yw[4] = {y4.x, y4.y, y4.z, y4.w};
  float x[8], y[8];
  uint32_t out[4], unsure = 0;
#pragma unroll
  for (int i = 0; i < 4; ++i) {
    x[2 * i] = bf16_lo(xw[i]);
    x[2 * i + 1] = bf16_hi(xw[i]);
    y[2 * i] = pairs ? x[2 * i + 1] : bf16_lo(yw[i]);
    y[2 * i + 1] = pairs ? x[2 * i] : bf16_hi(yw[i]);
  }
#pragma unroll
  for (int i = 0; i < 4; ++i) {
    float lo[2], hi[2];
#pragma unroll
    for (int e = 0; e < 2; ++e) {
      const int k = 2 * i + e;
      const float p = y[k] * g.s[k], r = fmaf(x[k], g.c[k], p);
      const float sum = fmaf(fabsf(x[k]), fabsf(g.c[k]), fabsf(p));
      const float delta = fmaf(sum, 0x1.9p-23f, fminf(sum, 0x1p-147f));  // (0 of zeros)
      lo[e] = r - delta;
      hi[e] = r + delta;
    }
    out[i] = pack_bf16(lo[0], lo[1]);
    unsure |= out[i] ^ pack_bf16(hi[0], hi[1]);
  }
  // (an infinity or NaN of the bounds shows as a magnitude from 0x7F80 on)
#pragma unroll
  for (int i = 0; i < 4; ++i) unsure |= (out[i] & 0x7F80u) == 0x7F80u || (out[i] & 0x7F800000u) == 0x7F800000u;
  if (__builtin_amdgcn_ballot_w64(unsure != 0) != 0) {
#pragma unroll
    for (int i = 0; i < 4; ++i)
      out[i] = pack_bf16(rotated64(x[2 * i], y[2 * i], g.c[2 * i], g.s[2 * i]),
                         rotated64(x[2 * i + 1], y[2 * i + 1], g.c[2 * i + 1], g.s[2 * i + 1]));
  }
  return make_uint4(out[0], out[1], out[2], out[3]);
}

// Codes (one word) and scale (bf16 bits) of 8 channels of a key; the 4 lanes of a quad hold a scale
// group and call together.  The quotient v / g of bf16 numbers lies 2^-9 or more from a half unless it
// is one (2 v - c g, c odd, is a multiple of the smaller of their units in the last place), so a product
// with the reciprocal, off by at most 2^-20, rounds right once it is put on the grid of 2^-11, where
// every half lies: the first addition does that, the second rounds to an integer, whose low bits are
// the code.
__device__ inline uint32_t key_codes(const uint4& x, uint32_t& scale_bits) {
  typedef unsigned short u16x2 __attribute__((ext_vector_type(2)));
  const uint32_t w[4] = {x.x, x.y, x.z, x.w};
  u16x2 m2 = {0, 0};
#pragma unroll
  for (int i = 0; i < 4; ++i) m2 = __builtin_elementwise_max(m2, __builtin_bit_cast(u16x2, w[i] & 0x7FFF7FFFu));
  uint32_t mx = max((uint32_t)m2.x, (uint32_t)m2.y);
  // quad_perm [1,0,3,2] and [2,3,0,1]
  mx = max(mx, (uint32_t)__builtin_amdgcn_update_dpp(0, (int)mx, 0xB1, 0xF, 0xF, false));
  mx = max(mx, (uint32_t)__builtin_amdgcn_update_dpp(0, (int)mx, 0x4E, 0xF, 0xF, false));
  scale_bits = pack_bf16(__uint_as_float(mx << 16) / 7.0f, 0.0f);
  const float g = __uint_as_float(scale_bits << 16);
  uint32_t word = 0;
  if (__builtin_amdgcn_ballot_w64(g != 0.0f && (g < 0x1p-100f || g > 0x1p100f)) == 0) {
    const float y = g == 0.0f ? 0.0f : 1.0f / g;
#pragma unroll
    for (int i = 0; i < 8; ++i) {
      const float v = (i & 1) ? bf16_hi(w[i >> 1]) : bf16_lo(w[i >> 1]);
      // 1.5 * 2^12, then up to 1.5 * 2^23 + 8
      const uint32_t c = __float_as_uint((v * y + 6144.0f) + (12582912.0f - 6144.0f + 8.0f));
      word |= (c & 0xFu) << (4 * nibble_of(i));
    }
  } else if (g == 0.0f) {
    word = 0x88888888u;
  } else {
    // both brought near 1 by a power of two (exact), so that no reciprocal overflows; a subnormal scale may be
    // rounded down so far that codes have to be clamped
    const int e = -__builtin_amdgcn_frexp_expf(g);
    const float y = 1.0f / __builtin_amdgcn_ldexpf(g, e);
#pragma unroll
    for (int i = 0; i < 8; ++i) {
      const float v = (i & 1) ? bf16_hi(w[i >> 1]) : bf16_lo(w[i >> 1]);
      const float t = (__builtin_amdgcn_ldexpf(v, e) * y + 6144.0f) - 6144.0f;
      const int c = (int)__builtin_amdgcn_fmed3f(__builtin_rintf(t), -7.0f, 7.0f);
      word |= (uint32_t)(c + 8) << (4 * nibble_of(i));
    }
  }
  return word;
}

// Codes (one word, element i in nibble i, two's complement) and scale of 8 channels of a value, as
// quant_piece's for rows outside its common path: no tables to build for a few tokens.
template <int LPT>
__device__ inline uint32_t value_codes(const uint4& x, float& gamma) {
  const uint32_t w[4] = {x.x, x.y, x.z, x.w};
  const QuantFmt f{true, true, 7.0f};
  const uint32_t mx = row_absmax_bits<LPT>(w);
  const int ef = (int)(mx >> 7);
  gamma = __uint_as_float(mx << 16) / 7.0f;
  uint32_t code[8], word = 0;
  if (__builtin_amdgcn_ballot_w64(ef <= 27) != 0 && ef <= 27) {
    codes_divided(w, gamma, f, code);
  } else {
    const float sc = __builtin_amdgcn_ldexpf(1.0f, 127 - ef);
    const float gs = gamma * sc;
    codes_scaled(w, sc, gs, 1.0f / gs, f, code);
  }
#pragma unroll
  for (int i = 0; i < 8; ++i) word |= (code[i] & 0xFu) << (4 * i);
  return word;
}

// Words of 8 tokens' channels (element t of the tokens in nibble nibble_of(t)) from 8 tokens' words of 8
// channels (channel i in nibble i): an 8 x 8 transpose of nibbles, halves, then bytes, then nibbles.
__device__ inline void transpose(const uint32_t (&in)[8], uint32_t (&out)[8]) {
  uint32_t a[8], b[8];
#pragma unroll
  for (int t = 0; t < 8; ++t) a[nibble_of(t)] = in[t];  // row n becomes nibble n
#pragma unroll
  for (int n = 0; n < 4; ++n) {
    b[n] = __builtin_amdgcn_perm(a[n + 4], a[n], 0x05040100u);
    b[n + 4] = __builtin_amdgcn_perm(a[n + 4], a[n], 0x07060302u);
  }
#pragma unroll
  for (int n = 0; n < 8; n += 4)
#pragma unroll
    for (int k = 0; k < 2; ++k) {
      a[n + k] = __builtin_amdgcn_perm(b[n + k + 2], b[n + k], 0x06020400u);
      a[n + k + 2] = __builtin_amdgcn_perm(b[n + k + 2], b[n + k], 0x07030501u);
    }
#pragma unroll
  for (int n = 0; n < 8; n += 2) {
    out[n] = (a[n] & 0x0F0F0F0Fu) | ((a[n + 1] & 0x0F0F0F0Fu) << 4);
    out[n + 1] = ((a[n] >> 4) & 0x0F0F0F0Fu) | (a[n + 1] & 0xF0F0F0F0u);
  }
}

// Whether some sequence's range holds the row; the wave calls together and looks at 64 entries at a time.  In
// nondecreasing offsets the last entry up to the row starts the only range that can hold it; where that one does
// not (a row behind the last sequence, or offsets that fall), all ranges are looked at.
__device__ inline bool in_a_sequence(const StepArgs& s, int batch, int32_t row) {
  const int lane = threadIdx.x & 63;
  const auto holds = [&](int b) {
    const int32_t lo = s.offsets[b], hi = s.offsets[b + 1];
    return step_range(s, lo, hi) && row >= lo && row < hi;
  };
  int base = 0, n = batch + 1;
  while (n > 1) {
    const int step = (n + 63) / 64;
    const bool below = lane * step < n && s.offsets[base + lane * step] <= row;
    const int found = max(__builtin_popcountll(__builtin_amdgcn_ballot_w64(below)), 1);
    base += (found - 1) * step;
    n = min(step, n - (found - 1) * step);
  }
  if (base < batch && holds(base)) return true;
  for (int b = 0; b < batch; b += 64)
    if (__builtin_amdgcn_ballot_w64(b + lane < batch && holds(b + lane)) != 0) return true;
  return false;
}

// One token's query rows.  The loads come first, then what decides whether they count.
template <int D, int T>
__device__ inline void rotate_queries(const CacheWriteArgs& a, int unit) {
  constexpr int LPT = D / 8, kHeads = T / LPT;
  const int layer = a.by_total.div(unit), row = a.by_total.mod(unit, layer);
  const int piece = threadIdx.x % LPT;
  const bool turn = rotates(a, piece);
  const int other = turn && !a.pairs ? partner(a, piece) : piece;
  const uint16_t* from = a.q.data + layer * a.q.layer + row * a.q.token;
  uint16_t* to = a.q_out.data + layer * a.q_out.layer + row * a.q_out.token;
  int h = (int)threadIdx.x / LPT;
  uint4 x = make_uint4(0, 0, 0, 0), y = x;
  if (h < a.Hq) {
    x = *((const uint4*)(from + h * a.q.head) + piece);
    y = *((const uint4*)(from + h * a.q.head) + other);
  }
  const int64_t pos = scalar_load(a.positions + row);
  if (pos < 0 || pos >= a.num_positions) return;
  Angles g = {};
  if (turn) g = load_angles(a, a.cos_sin + pos * a.rotary_dim, piece);
  if (a.s.offsets == nullptr ? row >= a.c.batch : !in_a_sequence(a.s, a.c.batch, row)) return;
  while (h < a.Hq) {
    if (turn) x = rotated(a.pairs, x, y, g);
    // (a row's lanes are of one wave and load before they store, so q_out may be q)
    *((uint4*)(to + h * a.q_out.head) + piece) = x;
    h += kHeads;
    if (h >= a.Hq) break;
    x = *((const uint4*)(from + h * a.q.head) + piece);
    y = *((const uint4*)(from + h * a.q.head) + other);
  }
}

template <int D, bool LOAD, int T>
__global__ __launch_bounds__(T) void k_cache_write(CacheWriteArgs a, int kv_units) {
  using B = CacheBlock<D>;
  constexpr int LPT = D / 8;                         // lanes of a row
  constexpr int kPasses = kCacheBlock * LPT / T;
  __shared__ uint32_t codes[kCacheBlock][LPT + 1];   // value codes, element i in nibble i
  __shared__ uint4 words[D];                         // the block's value words
  if (!LOAD && (int)blockIdx.x >= kv_units) {
    rotate_queries<D, T>(a, (int)blockIdx.x - kv_units);
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
  uint32_t vc[kPasses];
  float gamma[kPasses];
  int64_t pos[kPasses];
#pragma unroll
  for (int p = 0; p < kPasses; ++p) {
    const int token = j * kCacheBlock + p * (T / LPT) + (int)threadIdx.x / LPT;
    const int64_t row = row0 + token;
    kx[p] = ky[p] = vx[p] = make_uint4(0, 0, 0, 0);
    vc[p] = 0;
    gamma[p] = 0.0f;
    pos[p] = 0;
    if (token < start || token >= len) continue;
    const uint16_t* k = a.k.data + layer * a.k.layer + row * a.k.token + head * a.k.head;
    if (turned) pos[p] = a.positions[row];
    kx[p] = *((const uint4*)k + piece);
    if (turned) ky[p] = *((const uint4*)k + other);
    if (LOAD) {
      const int64_t at = (int64_t)lh * a.kept_off[a.c.batch] + row;
      vc[p] = *((const uint32_t*)(a.v_q + at * (D / 2)) + piece);
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
  if (page < 0 || page >= a.c.num_pages || mask == 0) return;
  uint8_t* blk = a.c.pages + ((((((int64_t)layer * a.c.num_pages + page) * a.c.Hkv + head) << a.c.page_shift) +
                               (j & ((1 << a.c.page_shift) - 1))) * B::kBytes);
  uint4* out = (uint4*)(blk + B::kValues) + threadIdx.x;
  uint4 old = make_uint4(0, 0, 0, 0);
  if (mask != 0xFFFFFFFFu && threadIdx.x < D) old = *out;
#pragma unroll
  for (int p = 0; p < kPasses; ++p) {
    const int slot = p * (T / LPT) + (int)threadIdx.x / LPT;
    const bool w = (mask >> slot) & 1u;
    if (__builtin_amdgcn_ballot_w64(w) == 0) continue;  // a wave without a token has nothing to quantise
    if (turned) {
      Angles g = {};
      if (turn && w) g = load_angles(a, a.cos_sin + pos[p] * a.rotary_dim, piece);
      const uint4 r = rotated(a.pairs, kx[p], ky[p], g);
      if (turn && w) kx[p] = r;
    }
    uint32_t scale;
    const uint32_t word = key_codes(kx[p], scale);  // every lane takes part
    if (!LOAD) vc[p] = value_codes<LPT>(vx[p], gamma[p]);
    codes[slot][piece] = vc[p];
    if (w) {
      *((uint32_t*)(blk + B::kKeys) + slot * LPT + (piece & 3) * (D / 32) + (piece >> 2)) = word;
      if ((piece & 3) == 0) *((uint16_t*)(blk + B::kKeyScales) + slot * (D / 32) + (piece >> 2)) = (uint16_t)scale;
      if (piece == 0) *((float*)(blk + B::kValueScales) + slot) = gamma[p];
    }
  }
  __syncthreads();
  if (threadIdx.x < 4 * LPT) {  // the tokens of a group g, eight channels
    const int g = threadIdx.x / LPT, c8 = threadIdx.x % LPT;
    uint32_t in[8], tr[8];
#pragma unroll
    for (int e = 0; e < 8; ++e) in[e] = codes[(e >> 2) * 16 + 4 * g + (e & 3)][c8];
    transpose(in, tr);
#pragma unroll
    for (int i = 0; i < 8; ++i)  // two's complement to c + 8: the sign bits flipped
      ((uint32_t*)words)[(c8 >> 3) * 256 + (16 * g + (c8 & 1) * 8 + i) * 4 + ((c8 >> 1) & 3)] = tr[i] ^ 0x88888888u;
  }
  __syncthreads();
  if (threadIdx.x < D) {
    const int g = (threadIdx.x & 63) >> 4;
    uint32_t set = 0;  // the nibbles of the tokens that are written
#pragma unroll
    for (int e = 0; e < 8; ++e)
      if ((mask >> ((e >> 2) * 16 + 4 * g + (e & 3))) & 1u) set |= 0xFu << (4 * nibble_of(e));
    if (set == 0) return;
    uint4 x = words[threadIdx.x];
    x.x = (old.x & ~set) | (x.x & set);
    x.y = (old.y & ~set) | (x.y & set);
    x.z = (old.z & ~set) | (x.z & set);
    x.w = (old.w & ~set) | (x.w & set);
    *out = x;
  }
}

// Eight channels as c * scale in fp32, rounded to bf16.
__device__ inline uint4 held_row(const float (&c)[8], float scale) {
  return make_uint4(pack_bf16(c[0] * scale, c[1] * scale), pack_bf16(c[2] * scale, c[3] * scale),
                    pack_bf16(c[4] * scale, c[5] * scale), pack_bf16(c[6] * scale, c[7] * scale));
}

// 16 bytes that pass once: ONCE leaves them out of the caches.
typedef uint32_t u32x4 __attribute__((ext_vector_type(4)));
template <bool ONCE>
__device__ inline uint4 load16(const uint4* p) {
  if (!ONCE) return *p;
  const u32x4 x = __builtin_nontemporal_load((const u32x4*)p);
  return make_uint4(x.x, x.y, x.z, x.w);
}
template <bool ONCE>
__device__ inline void store16(uint4* p, const uint4& x) {
  if (ONCE)
    __builtin_nontemporal_store((u32x4){x.x, x.y, x.z, x.w}, (u32x4*)p);
  else
    *p = x;
}

// ONCE: the rows are more than the chip's caches hold, so no later kernel finds them there (8 layers and heads, 29755
// tokens: 254 us, 240 with it).
template <int D, bool ONCE>
__global__ __launch_bounds__(kRowsThreads) void k_cache_read(CacheReadArgs a) {
  using B = CacheBlock<D>;
  constexpr int LPT = D / 8, kPasses = kCacheBlock * LPT / kRowsThreads;
  __shared__ uint4 words[D];
  const int rest = a.heads.div((int)blockIdx.x), lh = a.heads.mod((int)blockIdx.x, rest), b = blockIdx.y;
  const int layer = a.by_Hkv.div(lh), head = a.by_Hkv.mod(lh, layer);
  const int64_t first = a.first[b], n = a.off[b + 1] - a.off[b];
  const int64_t j = (first >> 5) + rest;
  if (j * kCacheBlock >= first + n) return;
  const int32_t raw = scalar_load(a.c.lens + b);
  const int32_t len = raw < 0 || raw > a.c.max_len ? 0 : raw;
  const uint8_t* blk = j * kCacheBlock < len ? cache_block<D>(a.c, layer, head, b, (int)j) : nullptr;
  const int piece = threadIdx.x % LPT;
  uint32_t kw[kPasses], ks[kPasses];
  float vs[kPasses];
  if (blk != nullptr) {
    if (threadIdx.x < D) words[threadIdx.x] = load16<ONCE>((const uint4*)(blk + B::kValues) + threadIdx.x);
#pragma unroll
    for (int p = 0; p < kPasses; ++p) {
      const int slot = p * (kRowsThreads / LPT) + (int)threadIdx.x / LPT;
      kw[p] = *((const uint32_t*)(blk + B::kKeys) + slot * LPT + (piece & 3) * (D / 32) + (piece >> 2));
      ks[p] = *((const uint16_t*)(blk + B::kKeyScales) + slot * (D / 32) + (piece >> 2));
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
#pragma unroll
      for (int e = 0; e < 8; ++e) c[e] = (float)((int)((kw[p] >> (4 * nibble_of(e))) & 0xFu) - 8);
      k = held_row(c, __uint_as_float(ks[p] << 16));
      const int g = (slot >> 2) & 3, shift = 4 * nibble_of((slot >> 4) * 4 + (slot & 3));
#pragma unroll
      for (int i = 0; i < 8; ++i) {
        const int x = piece * 8 + i;
        const uint32_t vw = ((const uint32_t*)words)[(x >> 6) * 256 + (g * 16 + (x & 15)) * 4 + ((x >> 4) & 3)];
        c[i] = (float)((int)((vw >> shift) & 0xFu) - 8);
      }
      v = held_row(c, vs[p]);
    }
    const int64_t to = (int64_t)lh * a.off[a.c.batch] + a.off[b] + (t - first);
    store16<ONCE>((uint4*)(a.k + to * D) + piece, k);
    store16<ONCE>((uint4*)(a.v + to * D) + piece, v);
  }
}

// Divisors of the workgroups' numbers.
template <typename Args>
void set_heads(Args& a) {
  a.heads = Divisor::of((int64_t)a.c.L * a.c.Hkv);
  a.by_Hkv = Divisor::of(a.c.Hkv);
}

}  // namespace

hipError_t launch_cache_append(CacheWriteArgs& a, int head_dim, hipStream_t stream) {
  const int units = a.c.L * a.c.Hkv * a.blocks * a.c.batch;
  set_heads(a);
  a.by_blocks = Divisor::of(a.blocks);
  a.by_total = Divisor::of(a.s.total);
  const dim3 grid((unsigned)units + (a.q.data != nullptr ? (unsigned)(a.c.L * a.s.total) : 0u));
  if (head_dim == 128 && a.s.max_new <= kFewTokens)
    hipLaunchKernelGGL((k_cache_write<128, false, kFewThreads>), grid, dim3(kFewThreads), 0, stream, a, units);
  else if (head_dim == 128)
    hipLaunchKernelGGL((k_cache_write<128, false, kRowsThreads>), grid, dim3(kRowsThreads), 0, stream, a, units);
  else
    hipLaunchKernelGGL((k_cache_write<64, false, kRowsThreads>), grid, dim3(kRowsThreads), 0, stream, a, units);
  return hipGetLastError();
}

hipError_t launch_cache_load(CacheWriteArgs& a, int head_dim, hipStream_t stream) {
  const int units = a.c.L * a.c.Hkv * a.blocks;
  const dim3 grid((unsigned)units, (unsigned)a.c.batch);
  set_heads(a);
  if (head_dim == 128)
    hipLaunchKernelGGL((k_cache_write<128, true, kRowsThreads>), grid, dim3(kRowsThreads), 0, stream, a, units);
  else
    hipLaunchKernelGGL((k_cache_write<64, true, kRowsThreads>), grid, dim3(kRowsThreads), 0, stream, a, units);
  return hipGetLastError();
}

hipError_t launch_cache_read(CacheReadArgs& a, int head_dim, hipStream_t stream) {
  const dim3 grid((unsigned)(a.c.L * a.c.Hkv * a.blocks), (unsigned)a.c.batch);
  set_heads(a);
  const bool once = (double)a.c.L * a.c.Hkv * (double)a.off[a.c.batch] * head_dim * 4.0 > (double)(256 << 20);
  if (head_dim == 128 && once)
    hipLaunchKernelGGL((k_cache_read<128, true>), grid, dim3(kRowsThreads), 0, stream, a);
  else if (head_dim == 128)
    hipLaunchKernelGGL((k_cache_read<128, false>), grid, dim3(kRowsThreads), 0, stream, a);
  else if (once)
    hipLaunchKernelGGL((k_cache_read<64, true>), grid, dim3(kRowsThreads), 0, stream, a);
  else
    hipLaunchKernelGGL((k_cache_read<64, false>), grid, dim3(kRowsThreads), 0, stream, a);
  return hipGetLastError();
}

}  // namespace tp

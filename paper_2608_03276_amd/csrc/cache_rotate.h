// Rotation of key and query rows by their positions, shared by the kernels that append to a paged cache (4-bit and
// 8-bit): d/8 lanes hold a row, 16 bytes each.
#pragma once

#include "cache_block.h"

namespace tp {
namespace {

constexpr float kMaxBf16 = 3.3895313892515355e38f;

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

}  // namespace
}  // namespace tp

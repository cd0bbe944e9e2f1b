// What the attentions over the paged caches (4-bit and 8-bit) share: operand fragments, the softmax's running
// reference, reductions over a row's lanes, the rows of a workgroup, the output, and the kernel that joins chunks.
#pragma once

#include "cache_block.h"

namespace tp {
namespace {

typedef _Float16 f16x8 __attribute__((ext_vector_type(8)));
typedef _Float16 f16x2 __attribute__((ext_vector_type(2)));
typedef unsigned short u16x2 __attribute__((ext_vector_type(2)));
typedef uint32_t u32x2 __attribute__((ext_vector_type(2)));
typedef uint32_t u32x4 __attribute__((ext_vector_type(4)));
typedef float f32x4 __attribute__((ext_vector_type(4)));

constexpr int kMergeThreads = 256;
constexpr float kNoMax = -3.402823466e38f;  // (maximum, sum) of nothing is (kNoMax, 0): joining it changes nothing
constexpr float kLn2 = 0.6931471805599453f;
// A row's reference is set so that its largest weight is 2^kSet, and raised when one exceeds 2^kLimit (fp16
// ends below 2^16): most blocks skip the rescaling and the reduction across lanes, and weights down to
// 2^-22 of the largest are normal fp16 numbers.
constexpr float kSet = 8.0f, kLimit = 16384.0f;
// A reference is one fp32 number, so the exponent x - m is off by half its unit: 4 at 2^26, between kSet and kLimit.
// Scores beyond that (where one rounding of a score changes a weight by 2^4) count as infinities: a reference starts at
// -2^26, which leaves keys below that no weight, and one above 2^26 makes the row NaN.
constexpr float kFar = 0x1p26f;
// Scales below 2^-60 count as that in the reference, and sums of p above 2^74 raise it too, so that tokens
// with tiny or zero values cannot overflow the sum.
constexpr float kLeastScale = 0x1p-60f;

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

// Reductions over the four lanes of a row (lane, lane ^ 16, ^ 32, ^ 48) and over the wave, without LDS: a swap of
// a register with itself leaves the two sides of an exchange in its two results.
__device__ inline u32x2 swap16(uint32_t x) { return __builtin_bit_cast(u32x2, __builtin_amdgcn_permlane16_swap(x, x, false, false)); }
__device__ inline u32x2 swap32(uint32_t x) { return __builtin_bit_cast(u32x2, __builtin_amdgcn_permlane32_swap(x, x, false, false)); }
__device__ inline float row_max(float x) {
  u32x2 s = swap16(__float_as_uint(x));
  x = fmaxf(__uint_as_float(s.x), __uint_as_float(s.y));
  s = swap32(__float_as_uint(x));
  return fmaxf(__uint_as_float(s.x), __uint_as_float(s.y));
}
__device__ inline float row_sum(float x) {
  u32x2 s = swap16(__float_as_uint(x));
  x = __uint_as_float(s.x) + __uint_as_float(s.y);
  s = swap32(__float_as_uint(x));
  return __uint_as_float(s.x) + __uint_as_float(s.y);
}
__device__ inline uint32_t row_max(uint32_t x) {
  u32x2 s = swap16(x);
  s = swap32(max(s.x, s.y));
  return max(s.x, s.y);
}
__device__ inline uint32_t wave_max(uint32_t x) {
  // quad_perm [1,0,3,2], [2,3,0,1], row_half_mirror, row_mirror
  x = max(x, (uint32_t)__builtin_amdgcn_update_dpp(0, (int)x, 0xB1, 0xF, 0xF, false));
  x = max(x, (uint32_t)__builtin_amdgcn_update_dpp(0, (int)x, 0x4E, 0xF, 0xF, false));
  x = max(x, (uint32_t)__builtin_amdgcn_update_dpp(0, (int)x, 0x141, 0xF, 0xF, false));
  x = max(x, (uint32_t)__builtin_amdgcn_update_dpp(0, (int)x, 0x140, 0xF, 0xF, false));
  return row_max(x);
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

// Place of a row's partial result: [chunks][batch][L * Hkv][R * max_new].
__device__ inline int64_t partial_row(const CacheAttnArgs& a, int chunk, int b, int lh, int row) {
  return (((int64_t)chunk * a.c.batch + b) * (int)a.heads.d + lh) * ((int64_t)a.R.d * a.s.max_new) + row;
}

// CH channels of a row from c0: the sum of weighted values over the sum of weights (st.y), and the log-sum-exp.  The sum
// is 0 where no key was seen; a row with a score of +infinity (its reference is beyond kFar) or NaN is NaN throughout.
template <int CH>
__device__ inline void store_output(const CacheAttnArgs& a, int layer, int64_t token, int hq, int c0, const float (&o)[CH],
                                    const float2& st) {
  const float sum = st.x > kFar ? NAN : st.y, inv = sum == 0.0f ? 0.0f : 1.0f / sum;
  uint16_t* to = a.o.data + layer * a.o.layer + token * a.o.token + hq * a.o.head + c0;
  typedef __bf16 bf16s __attribute__((ext_vector_type(CH)));
  bf16s v;
#pragma unroll
  for (int i = 0; i < CH; ++i) v[i] = (__bf16)(o[i] * inv);
  *(bf16s*)to = v;
  if (a.lse != nullptr && c0 == 0)
    a.lse[((int64_t)layer * a.Hq + hq) * a.s.total + token] =
        sum == 0.0f ? -INFINITY : (st.x + __builtin_amdgcn_logf(sum)) * kLn2;
}

// Joins the chunks of a row: by WPR waves, whose groups of D / 4 lanes take every kGroups-th chunk, four channels a
// lane, each with a reference of its own.
template <int D, int WPR>
__global__ __launch_bounds__(kMergeThreads) void k_cache_merge(CacheAttnArgs a) {
  constexpr int kLanes = D / 4;
  constexpr int kGroups = WPR * 64 / kLanes;
  constexpr int kRows = kMergeThreads / 64 / WPR;
  __shared__ f32x4 lds_o[kRows][kGroups][kLanes];
  __shared__ float2 lds_stat[kRows][kGroups];
  const int width = 16 * a.tiles;
  const int rest = a.heads.div((int)blockIdx.x), lh = a.heads.mod((int)blockIdx.x, rest);
  const int layer = a.by_Hkv.div(lh), head = a.by_Hkv.mod(lh, layer);
  const int b = blockIdx.y;
  const int mine = threadIdx.x / (WPR * 64);                      // row of the workgroup
  const int part = threadIdx.x % (WPR * 64) / kLanes, lane = threadIdx.x % kLanes;
  const StepSeq q = step_sequence(a.c, a.s, b);
  const int row = rest * kRows + mine;
  const RowGroup rg = row_group(a, q, row / width, width);
  const bool in = row < rg.rows && rg.keys > a.chunk;
  const int t = a.R.div(row), hq = head * (int)a.R.d + a.R.mod(row, t);
  const int64_t token = q.row + t;
  const int64_t at = partial_row(a, 0, b, lh, row), rows = partial_row(a, 1, 0, 0, 0);
  float2 st = make_float2(kNoMax, 0.0f);
  f32x4 o = {0, 0, 0, 0};
  if (in) {
    const int active = a.by_chunk.div(rg.keys + a.chunk - 1);
#pragma unroll 4
    for (int c = part; c < active; c += kGroups) {
      const float2 s = a.stat[c * rows + at];
      const f32x4 p = *(const f32x4*)(a.part + (c * rows + at) * D + lane * 4);
      const float top = fmaxf(st.x, s.x);
      const float f = __builtin_amdgcn_exp2f(st.x - top), fs = __builtin_amdgcn_exp2f(s.x - top);
      st = make_float2(top, st.y * f + s.y * fs);
      o = o * f + p * fs;
    }
    lds_o[mine][part][lane] = o;
    if (lane == 0) lds_stat[mine][part] = st;
  }
  __syncthreads();
  if (!in || part != 0) return;
  float top = kNoMax;
#pragma unroll
  for (int i = 0; i < kGroups; ++i) top = fmaxf(top, lds_stat[mine][i].x);
  st = make_float2(top, 0.0f);
  o = (f32x4){0, 0, 0, 0};
#pragma unroll
  for (int i = 0; i < kGroups; ++i) {
    const float2 s = lds_stat[mine][i];
    const float f = __builtin_amdgcn_exp2f(s.x - top);
    st.y += s.y * f;
    o += lds_o[mine][i][lane] * f;
  }
  const float x[4] = {o.x, o.y, o.z, o.w};
  store_output<4>(a, layer, token, hq, lane * 4, x, st);
}

}  // namespace
}  // namespace tp

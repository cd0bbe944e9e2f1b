// Rows into and out of the paged 4-bit cache: tp_cache_append, tp_cache_load, tp_cache_read.
//
// One workgroup handles one block (32 tokens of one head): d/8 lanes hold a row, 16 bytes each.  The
// value codes of a block are transposed in LDS, since a word holds one channel of eight tokens; words
// of which only some tokens are written are read, merged and written back.  A block belongs to one
// workgroup of the launch, so nothing races.
#include "cache_block.h"
#include "quant_row.h"

namespace tp {
namespace {

constexpr int kRowsThreads = 256;
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

// f, the fp32 number next to a value that differs from it by `rest` (its sign is all that counts), as an fp32
// number that rounds to the bf16 number the value itself rounds to: f may lie halfway between two only by its own
// rounding.
__device__ inline float for_bf16(float f, float rest) {
  const uint32_t b = __float_as_uint(f);
  if ((b & 0xFFFFu) != 0x8000u || rest == 0.0f) return f;
  return __uint_as_float((rest > 0.0f) == ((int32_t)b >= 0) ? b + 1 : b - 1);
}

// For rounding to bf16 once; within its range, so that no rotation of finite rows gives an infinity.
__device__ inline float rounded(double r) {
  r = __builtin_fmax(__builtin_fmin(r, (double)kMaxBf16), -(double)kMaxBf16);
  const float f = (float)r;
  const double rest = r - (double)f;
  return for_bf16(f, rest > 0.0 ? 1.0f : rest < 0.0 ? -1.0f : 0.0f);
}

// Piece `piece` (8 channels) of a row, rotated by the angles of the row cs of the table.  In 64 bits
// (a product of a bf16 and an fp32 number is exact there): the codes behind it are those of the exact
// rotation, and the kernels are bound by memory all the same.
__device__ inline uint4 rotated_piece(const CacheWriteArgs& a, const uint16_t* row, int piece, const float* cs) {
  const uint4 x = *((const uint4*)row + piece);
  if (piece * 8 >= a.rotary_dim) return x;
  const int half = a.rotary_dim / 2;
  const uint32_t xw[4] = {x.x, x.y, x.z, x.w};
  uint32_t out[4];
  if (a.pairs) {
    const float4 c = *(const float4*)(cs + piece * 4), s = *(const float4*)(cs + half + piece * 4);
    const float cc[4] = {c.x, c.y, c.z, c.w}, ss[4] = {s.x, s.y, s.z, s.w};
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      const double p = bf16_lo(xw[i]), q = bf16_hi(xw[i]), ci = cc[i], si = ss[i];
      out[i] = pack_bf16(rounded(p * ci - q * si), rounded(q * ci + p * si));
    }
  } else {
    const bool first = piece * 8 < half;
    const int at = first ? piece * 8 : piece * 8 - half;
    const uint4 y = *((const uint4*)row + (first ? piece + half / 8 : piece - half / 8));
    const uint32_t yw[4] = {y.x, y.y, y.z, y.w};
    const float4 c0 = *(const float4*)(cs + at), c1 = *(const float4*)(cs + at + 4);
    const float4 s0 = *(const float4*)(cs + half + at), s1 = *(const float4*)(cs + half + at + 4);
    const float cc[8] = {c0.x, c0.y, c0.z, c0.w, c1.x, c1.y, c1.z, c1.w};
    const float ss[8] = {s0.x, s0.y, s0.z, s0.w, s1.x, s1.y, s1.z, s1.w};
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      const double p0 = bf16_lo(xw[i]), p1 = bf16_hi(xw[i]), q0 = bf16_lo(yw[i]), q1 = bf16_hi(yw[i]);
      const double g0 = first ? -(double)ss[2 * i] : (double)ss[2 * i];
      const double g1 = first ? -(double)ss[2 * i + 1] : (double)ss[2 * i + 1];
      out[i] = pack_bf16(rounded(p0 * (double)cc[2 * i] + q0 * g0), rounded(p1 * (double)cc[2 * i + 1] + q1 * g1));
    }
  }
  return make_uint4(out[0], out[1], out[2], out[3]);
}

// Codes (one word) and scale (bf16 bits) of 8 channels of a key; the 4 lanes of a quad hold a scale
// group and call together.  The quotient v / g of bf16 numbers lies 2^-9 or more from a half unless it
// is one (2 v - c g, c odd, is a multiple of the smaller of their units in the last place), so a product
// with the reciprocal, off by at most 2^-20, rounds right once it is put on the grid of 2^-11, where
// every half lies.
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
  if (g == 0.0f) return 0x88888888u;
  // both brought near 1 by a power of two (exact), so that no reciprocal overflows
  const int e = -__builtin_amdgcn_frexp_expf(g);
  const float y = 1.0f / __builtin_amdgcn_ldexpf(g, e);
  uint32_t word = 0;
#pragma unroll
  for (int i = 0; i < 8; ++i) {
    const float v = (i & 1) ? bf16_hi(w[i >> 1]) : bf16_lo(w[i >> 1]);
    const float t = (__builtin_amdgcn_ldexpf(v, e) * y + 6144.0f) - 6144.0f;  // the grid of 2^-11: 1.5 * 2^12
    const int c = (int)__builtin_amdgcn_fmed3f(__builtin_rintf(t), -7.0f, 7.0f);
    word |= (uint32_t)(c + 8) << (4 * nibble_of(i));
  }
  return word;
}

// Largest b with offsets[b] <= row, over batch + 1 nondecreasing entries; -1 if there is none.  The wave
// looks at 64 entries at a time.  (Of other offsets, some b in the same range.)
__device__ inline int sequence_of(const int32_t* offsets, int batch, int32_t row) {
  const int lane = threadIdx.x & 63;
  int base = 0, n = batch + 1;
  for (;;) {
    const int step = (n + 63) / 64;
    const bool below = lane * step < n && offsets[base + lane * step] <= row;
    const int found = __builtin_popcountll(__builtin_amdgcn_ballot_w64(below));
    if (found == 0) return -1;
    base += (found - 1) * step;
    n = min(step, n - (found - 1) * step);
    if (n <= 1) return base;
  }
}

// One token's query rows.
template <int D>
__device__ inline void rotate_queries(const CacheWriteArgs& a, int unit) {
  constexpr int LPT = D / 8;
  const int layer = unit / a.s.total, row = unit % a.s.total;
  const int b = a.s.offsets == nullptr ? row : sequence_of(a.s.offsets, a.c.batch, row);
  if (b < 0 || b >= a.c.batch) return;
  const StepSeq q = step_sequence(a.c, a.s, b);
  if (row < q.row || row - q.row >= q.count) return;
  const int64_t pos = a.positions[row];
  if (pos < 0 || pos >= a.num_positions) return;
  const float* cs = a.cos_sin + pos * a.rotary_dim;
  const int piece = threadIdx.x % LPT;
  for (int h = threadIdx.x / LPT; h < a.Hq; h += kRowsThreads / LPT) {
    const uint16_t* from = a.q.data + layer * a.q.layer + row * a.q.token + h * a.q.head;
    const uint4 x = rotated_piece(a, from, piece, cs);
    *((uint4*)(a.q_out.data + layer * a.q_out.layer + row * a.q_out.token + h * a.q_out.head) + piece) = x;
  }
}

template <int D, bool LOAD>
__global__ __launch_bounds__(kRowsThreads) void k_cache_write(CacheWriteArgs a, int kv_units) {
  using B = CacheBlock<D>;
  constexpr int LPT = D / 8;                         // lanes of a row
  constexpr int kPasses = kCacheBlock * LPT / kRowsThreads;
  __shared__ QuantTables tab;
  __shared__ uint32_t codes[kCacheBlock][LPT + 1];   // value codes, element i in nibble i
  __shared__ uint32_t written;                       // the block's tokens that are written
  if (!LOAD && (int)blockIdx.x >= kv_units) {
    rotate_queries<D>(a, (int)blockIdx.x - kv_units);
    return;
  }
  const int heads = a.c.L * a.c.Hkv;
  const int lh = (int)blockIdx.x % heads, rest = (int)blockIdx.x / heads;
  const int layer = lh / a.c.Hkv, head = lh % a.c.Hkv;
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
    b = rest / a.blocks;
    const StepSeq q = step_sequence(a.c, a.s, b);
    len = q.count == 0 ? 0 : q.len;
    row0 = (int64_t)q.row - (q.len - q.count);
    start = max(q.len - q.count, 0);
    j = (start >> 5) + rest % a.blocks;
  }
  if (j * kCacheBlock >= len) return;
  uint8_t* blk = cache_block<D>(a.c, layer, head, b, j);
  if (blk == nullptr) return;
  if (!LOAD) build_tables(tab, 7.0f, a.ro.off);
  if (threadIdx.x < 64) {
    const int t = j * kCacheBlock + (int)threadIdx.x;
    bool w = threadIdx.x < kCacheBlock && t >= start && t < len;
    if (!LOAD && w && a.cos_sin != nullptr) {
      const int64_t pos = a.positions[row0 + t];
      w = pos >= 0 && pos < a.num_positions;
    }
    const uint32_t m = (uint32_t)__builtin_amdgcn_ballot_w64(w);
    if (threadIdx.x == 0) written = m;
  }
  __syncthreads();
  const uint32_t mask = written;
  const int piece = threadIdx.x % LPT;
#pragma unroll
  for (int p = 0; p < kPasses; ++p) {
    const int slot = (int)threadIdx.x / LPT + p * (kRowsThreads / LPT);
    const bool w = (mask >> slot) & 1u;
    const int64_t row = row0 + j * kCacheBlock + slot;
    uint4 kx = make_uint4(0, 0, 0, 0);
    if (w) {
      const uint16_t* k = a.k.data + layer * a.k.layer + row * a.k.token + head * a.k.head;
      if (!LOAD && a.cos_sin != nullptr)
        kx = rotated_piece(a, k, piece, a.cos_sin + (int64_t)a.positions[row] * a.rotary_dim);
      else
        kx = *((const uint4*)k + piece);
    }
    uint32_t scale;
    const uint32_t word = key_codes(kx, scale);  // every lane takes part
    if (w) {
      *((uint32_t*)(blk + B::kKeys) + slot * LPT + (piece & 3) * (D / 32) + (piece >> 2)) = word;
      if ((piece & 3) == 0) *((uint16_t*)(blk + B::kKeyScales) + slot * (D / 32) + (piece >> 2)) = (uint16_t)scale;
    }
    if (LOAD) {
      const int64_t at = (int64_t)lh * a.kept_off[a.c.batch] + row;
      if (w) {
        codes[slot][piece] = *((const uint32_t*)(a.v_q + at * (D / 2)) + piece);
        if (piece == 0) *((float*)(blk + B::kValueScales) + slot) = a.v_scales[at];
      }
    } else {
      const uint4 vx = w ? *((const uint4*)(a.v.data + layer * a.v.layer + row * a.v.token + head * a.v.head) + piece)
                         : make_uint4(0, 0, 0, 0);
      const QuantFmt f{true, true, 7.0f};
      uint2 c;
      const float gamma = quant_piece<LPT, kQNibble>(vx, tab, f, c);
      codes[slot][piece] = c.x;
      if (w && piece == 0) *((float*)(blk + B::kValueScales) + slot) = gamma;
    }
  }
  __syncthreads();
  // the value words: channel x of eight tokens
  for (int i = threadIdx.x; i < 4 * D; i += kRowsThreads) {
    const int lane = (i & 255) >> 2, g = lane >> 4;
    const int x = (i >> 8) * 64 + (i & 3) * 16 + (lane & 15);
    uint32_t set = 0, word = 0;
#pragma unroll
    for (int e = 0; e < 8; ++e) {
      const int slot = (e >> 2) * 16 + 4 * g + (e & 3);
      if ((mask >> slot) & 1u) {
        set |= 0xFu << (4 * nibble_of(e));
        // two's complement to c + 8: the sign bit flipped
        word |= (((codes[slot][x >> 3] >> (4 * (x & 7))) ^ 8u) & 0xFu) << (4 * nibble_of(e));
      }
    }
    uint32_t* to = (uint32_t*)(blk + B::kValues) + i;
    if (set == 0) continue;
    *to = set == 0xFFFFFFFFu ? word : ((*to & ~set) | word);
  }
}

// Eight channels as c * scale, rounded to bf16 once (a product's error in fp32 is exact by one fma).
__device__ inline uint4 held_row(const float (&c)[8], float scale) {
  float x[8];
#pragma unroll
  for (int i = 0; i < 8; ++i) {
    x[i] = c[i] * scale;
    x[i] = for_bf16(x[i], fmaf(c[i], scale, -x[i]));
  }
  return make_uint4(pack_bf16(x[0], x[1]), pack_bf16(x[2], x[3]), pack_bf16(x[4], x[5]), pack_bf16(x[6], x[7]));
}

template <int D>
__global__ __launch_bounds__(kRowsThreads) void k_cache_read(CacheReadArgs a) {
  using B = CacheBlock<D>;
  constexpr int LPT = D / 8;
  constexpr int kPasses = kCacheBlock * LPT / kRowsThreads;
  __shared__ uint32_t words[4 * D];
  const int heads = a.c.L * a.c.Hkv;
  const int lh = (int)blockIdx.x % heads, b = blockIdx.y;
  const int64_t first = a.first[b], n = a.off[b + 1] - a.off[b];
  const int64_t j = (first >> 5) + (int)blockIdx.x / heads;
  if (j * kCacheBlock >= first + n) return;
  const int32_t raw = a.c.lens[b];
  const int32_t len = raw < 0 || raw > a.c.max_len ? 0 : raw;
  const uint8_t* blk = j * kCacheBlock < len ? cache_block<D>(a.c, lh / a.c.Hkv, lh % a.c.Hkv, b, (int)j) : nullptr;
  if (blk != nullptr)
    for (int i = threadIdx.x; i < D; i += kRowsThreads)
      *((uint4*)words + i) = *((const uint4*)(blk + B::kValues) + i);
  __syncthreads();
  const int piece = threadIdx.x % LPT;
#pragma unroll
  for (int p = 0; p < kPasses; ++p) {
    const int slot = (int)threadIdx.x / LPT + p * (kRowsThreads / LPT);
    const int64_t t = j * kCacheBlock + slot;
    if (t < first || t >= first + n) continue;
    uint4 k = make_uint4(0, 0, 0, 0), v = k;
    if (blk != nullptr && t < len) {
      const uint32_t w = *((const uint32_t*)(blk + B::kKeys) + slot * LPT + (piece & 3) * (D / 32) + (piece >> 2));
      const uint32_t ks = *((const uint16_t*)(blk + B::kKeyScales) + slot * (D / 32) + (piece >> 2));
      float c[8];
#pragma unroll
      for (int e = 0; e < 8; ++e) c[e] = (float)((int)((w >> (4 * nibble_of(e))) & 0xFu) - 8);
      k = held_row(c, __uint_as_float(ks << 16));
      const int g = (slot >> 2) & 3, e = (slot >> 4) * 4 + (slot & 3);
#pragma unroll
      for (int i = 0; i < 8; ++i) {
        const int x = piece * 8 + i;
        const uint32_t vw = words[(x >> 6) * 256 + (g * 16 + (x & 15)) * 4 + ((x >> 4) & 3)];
        c[i] = (float)((int)((vw >> (4 * nibble_of(e))) & 0xFu) - 8);
      }
      v = held_row(c, *((const float*)(blk + B::kValueScales) + slot));
    }
    const int64_t to = (int64_t)lh * a.off[a.c.batch] + a.off[b] + (t - first);
    *((uint4*)(a.k + to * D) + piece) = k;
    *((uint4*)(a.v + to * D) + piece) = v;
  }
}

}  // namespace

hipError_t launch_cache_append(const CacheWriteArgs& a, int head_dim, hipStream_t stream) {
  const int units = a.c.L * a.c.Hkv * a.blocks * a.c.batch;
  const unsigned grid = (unsigned)units + (a.q.data != nullptr ? (unsigned)(a.c.L * a.s.total) : 0u);
  if (head_dim == 128)
    hipLaunchKernelGGL((k_cache_write<128, false>), dim3(grid), dim3(kRowsThreads), 0, stream, a, units);
  else
    hipLaunchKernelGGL((k_cache_write<64, false>), dim3(grid), dim3(kRowsThreads), 0, stream, a, units);
  return hipGetLastError();
}

hipError_t launch_cache_load(const CacheWriteArgs& a, int head_dim, hipStream_t stream) {
  const int units = a.c.L * a.c.Hkv * a.blocks;
  const dim3 grid((unsigned)units, (unsigned)a.c.batch);
  if (head_dim == 128)
    hipLaunchKernelGGL((k_cache_write<128, true>), grid, dim3(kRowsThreads), 0, stream, a, units);
  else
    hipLaunchKernelGGL((k_cache_write<64, true>), grid, dim3(kRowsThreads), 0, stream, a, units);
  return hipGetLastError();
}

hipError_t launch_cache_read(const CacheReadArgs& a, int head_dim, hipStream_t stream) {
  const dim3 grid((unsigned)(a.c.L * a.c.Hkv * a.blocks), (unsigned)a.c.batch);
  if (head_dim == 128)
    hipLaunchKernelGGL(k_cache_read<128>, grid, dim3(kRowsThreads), 0, stream, a);
  else
    hipLaunchKernelGGL(k_cache_read<64>, grid, dim3(kRowsThreads), 0, stream, a);
  return hipGetLastError();
}

}  // namespace tp

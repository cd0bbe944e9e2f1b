// Attention over the paged 8-bit cache (tp_cache8_attention): the newest tokens of each sequence, from one (decoding)
// to a prompt's chunk, against all its tokens.
//
// A row's output is sum_t p_t v_t / sum_t p_t with p_t = exp(softmax_scale q . k_t - m), in one pass with a running
// reference m and sum.  attend_blocks does that for 16 to 64 query rows of one (sequence, KV head) and a range of its
// blocks of 32 tokens; its four or eight waves take every fourth or eighth block and join through LDS.  Both products
// are on v_mfma_f32_16x16x32_f16 with the cache as the A operand:
//   scores  S^T = C Q^T of the keys' codes, exact in fp16 (integers up to 127; e4m3 numbers, the smallest 2^-9);
//           the block's key scale goes into the factor that turns a sum into an exponent, one number a block;
//   output  O^T += C^T P^T of the values' codes, with the values' scales multiplied into the weights P.
// Codes become fp16 operands in registers: 0x6400 | u is 1024 + u for a byte u = c + 128 (one byte permutation makes
// two of them, one packed addition takes 1152 off), and an e4m3 pair is one conversion instruction.  Queries are exact
// in fp16 after a power of two of their row's.  Scores, reference, sum and outputs are fp32; the weights times the
// values' scales are rounded to fp16, 2^-11, below the output's own 2^-8 (bf16 operands would add as much again).
//
// What a workgroup takes:
//  - decoding and drafted tokens (up to 32 rows) that have to be split: equal shares of all the call's blocks, cut on the
//    device (k_cache8_shares, k_cache8_join_shares);
//  - short ones: whole sequences (k_cache8_attention);
//  - prompts: 64 rows, whole sequences or chunks that the host plans (k_cache8_attention, k_cache_merge).
//
// Measured at d = 128, 8 KV heads, kernels alone (a bare nontemporal read reaches 7.1 TB/s on this card).  One row tile is bound by
// HBM: 48 decoding sequences of 5201 to 23457 tokens, 64 query heads, 1.14 GB: 174 us, 6.5 TB/s, and 5 to join (in chunks that the
// host plans 213 together); two of 200003 and 98305: 93 and 5.  Two tiles: 16 sequences of 1 to 8 drafted tokens against 2208 to
// 11710: 46, of which HBM needs 33; the start (lengths, pages, queries: dependent loads) and the waves' join take the rest.
// Four tiles: chunks of 1024 and 300 tokens, 14001 and 4096 with those before them, 32 query heads: 246 GFLOP in 246 to 267 us by
// the card, 0.92 to 1.0 PFLOP/s; the issue of vector instructions beside the matrix core's bounds them: 271 and 64 products a wave and
// block, the matrix core 48 % busy (a stream of products leaves a neighbouring wave 40 % of the vector ALU's issue).
#include <algorithm>

#include "cache8_block.h"
#include "cache_join.h"

namespace tp {
namespace {

// Eight codes as fp16 numbers c; magic: 0x64646464.
template <bool FP8>
__device__ inline Frag codes8(uint32_t lo, uint32_t hi, uint32_t magic) {
  Frag f;
  if (FP8) {
    f.w[0] = __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_f16_fp8(lo, 1.0f, false));
    f.w[1] = __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_f16_fp8(lo, 1.0f, true));
    f.w[2] = __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_f16_fp8(hi, 1.0f, false));
    f.w[3] = __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_f16_fp8(hi, 1.0f, true));
  } else {
    const f16x2 off = {(_Float16)-1152.0f, (_Float16)-1152.0f};
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      const uint32_t two = __builtin_amdgcn_perm(magic, i < 2 ? lo : hi, (i & 1) ? 0x04030402u : 0x04010400u);
      f.w[i] = __builtin_bit_cast(uint32_t, __builtin_bit_cast(f16x2, two) + off);
    }
  }
  return f;
}

// Copies straight into LDS, 16 or 4 bytes a lane: lane i's land at lds + 16 i (4 i).  In assembly, because the compiler
// would wait for all of them before every LDS read that follows; the kernel waits for those that it needs.
template <bool ONCE>
__device__ inline void copy16(uint32_t offset, const uint8_t* from, uint32_t lds) {
  if (ONCE)
    asm volatile("s_mov_b32 m0, %2\n\ts_nop 0\n\tglobal_load_lds_dwordx4 %0, %1 nt" ::"v"(offset), "s"(from), "s"(lds) : "memory", "m0");
  else
    asm volatile("s_mov_b32 m0, %2\n\ts_nop 0\n\tglobal_load_lds_dwordx4 %0, %1" ::"v"(offset), "s"(from), "s"(lds) : "memory", "m0");
}
template <bool ONCE>
__device__ inline void copy4(uint32_t offset, const uint8_t* from, uint32_t lds) {
  if (ONCE)
    asm volatile("s_mov_b32 m0, %2\n\ts_nop 0\n\tglobal_load_lds_dword %0, %1 nt" ::"v"(offset), "s"(from), "s"(lds) : "memory", "m0");
  else
    asm volatile("s_mov_b32 m0, %2\n\ts_nop 0\n\tglobal_load_lds_dword %0, %1" ::"v"(offset), "s"(from), "s"(lds) : "memory", "m0");
}
template <int N>
__device__ inline void wait_copies_but() {
  asm volatile("s_waitcnt vmcnt(%0)" ::"n"(N) : "memory");
}
__device__ inline void wait_lds_reads() { asm volatile("s_waitcnt lgkmcnt(0)" ::: "memory"); }

// Division of a decoding call's work on the device, where the lengths are known: the (sequence, head) pairs in a row
// (sequences, then heads), each as long as its blocks and what starting on it costs, are cut into equal shares, one a
// workgroup.  A share holds several short pairs or a part of a long one; a pair whose blocks lie in several shares has a
// partial result in each, which k_cache8_join_shares joins.  So what a call costs goes by what its sequences hold and not
// by the bounds it was given.
//
// Times here are of both kernels, each call on a cache that the last ones did not read.  A share is a workgroup of four waves, one a
// CU.  Two a CU: 48 sequences of 5000 to 24000 tokens, 64 query heads, 1.32 GB, 210 -> 216 us, the 1.14 GB above 183 -> 190, one
// sequence of 131072 52.1 -> 55.9, of 13215 14.5 -> 15.3, drafted tokens unchanged; 320, 384 or 640 workgroups, which do not divide
// among the CUs, cost 10 to 25 %.  kStart: a share that begins a pair waits for lengths, pages, queries and a first block, one
// after another, and joins its waves at the end.  With 4, 8, 12, 16, 24, 32 blocks counted for that (before loads were
// nontemporal from 16 MB on): 24 sequences of 100 to 9000 tokens 58.1, 53.4, 50.2, 47.2, 47.2, 48.5 us; one of 13215 18.0, 16.9,
// 15.9, 15.8, 15.8, 15.8; four of 6000 18.5, 20.2, 20.4, 20.1, 20.1, 20.0.  Shares of at least kLeastShare blocks, one a wave: one
// sequence of 2000 tokens with 4, 8, 16: 9.8, 11.9, 12.9 us, of 1024 9.1, 9.6, 12.3.  Above kMostSequences every workgroup's sum over the lengths costs more than shares
// save (2000 sequences of 4500, one KV head: 430 us, in the plan's chunks 423; 1024 of 5000: 231, 236).
constexpr int kStart = 16;            // blocks that a pair's start and end cost
constexpr int kLeastShare = 4;
constexpr int kMostSequences = 1024;  // whose lengths every workgroup adds up

// Length of a pair of sequence b: its blocks (one, which writes the zeros, where it has rows and no tokens) and kStart, or 0.
// All positions are below 2^31 (cache8_plan).
__device__ inline int pair_length(const CacheAttnArgs& a, int b) {
  if (b >= a.c.batch) return 0;
  int32_t count = 1;
  if (a.s.offsets != nullptr) {
    const int32_t lo = a.s.offsets[b], hi = a.s.offsets[b + 1];
    count = step_range(a.s, lo, hi) ? hi - lo : 0;
  }
  const int32_t len = a.c.lens[b];
  if (count == 0) return 0;
  return max((len < 0 || len > a.c.max_len ? 0 : len) + kCacheBlock - 1, kCacheBlock) / kCacheBlock + kStart;
}
// Sums over the lanes up to each, of 64 numbers >= 0.
__device__ inline int wave_scan(int x) {
  // row_shr 1, 2, 4, 8, then the last lane of a row into the next, and that of the first two rows into the others
  x += __builtin_amdgcn_update_dpp(0, x, 0x111, 0xF, 0xF, true);
  x += __builtin_amdgcn_update_dpp(0, x, 0x112, 0xF, 0xF, true);
  x += __builtin_amdgcn_update_dpp(0, x, 0x114, 0xF, 0xF, true);
  x += __builtin_amdgcn_update_dpp(0, x, 0x118, 0xF, 0xF, true);
  x += __builtin_amdgcn_update_dpp(0, x, 0x142, 0xA, 0xF, false);
  x += __builtin_amdgcn_update_dpp(0, x, 0x143, 0xC, 0xF, false);
  return x;
}
// The pairs' lengths of 64 sequences from b0 on, one a lane, and their sums.
struct SequenceSums {
  int mine, upto, all;
};
__device__ inline SequenceSums sum_sequences(const CacheAttnArgs& a, int b0) {
  SequenceSums s;
  s.mine = pair_length(a, b0 + (int)(threadIdx.x & 63));
  s.upto = wave_scan(s.mine);
  s.all = __builtin_amdgcn_readlane(s.upto, 63);
  return s;
}
// Of one head of all sequences; `head`: the sums of the first 64.
__device__ inline int sum_all(const CacheAttnArgs& a, const SequenceSums& head) {
  int sum = head.all;
  for (int b0 = 64; b0 < a.c.batch; b0 += 64) sum += sum_sequences(a, b0).all;
  return sum;
}
__device__ inline int share_of(int all, int shares) {
  const int each = __builtin_amdgcn_readfirstlane((int)(((uint32_t)all + (uint32_t)shares - 1) / (uint32_t)shares));
  return max((each + 3) & ~3, kLeastShare);  // whole blocks for each of four waves
}
// A position in the row of pairs: `in` of the `length` of head lh of sequence b.
struct ShareAt {
  int b, lh, in, length;
};
// Position x < all.  (No length where there is none: lengths that change while the call runs end it.)
__device__ inline ShareAt share_at(const CacheAttnArgs& a, const SequenceSums& head, int x) {
  const int heads = (int)a.heads.d;
  SequenceSums s = head;
  int base = 0;
  for (int b0 = 0; b0 < a.c.batch;) {
    const uint64_t behind = __builtin_amdgcn_ballot_w64((base + s.upto) * heads > x);
    if (behind != 0) {
      const int i = __builtin_ctzll(behind);
      ShareAt p;
      p.b = b0 + i;
      p.length = __builtin_amdgcn_readlane(s.mine, i);
      const int rest = x - (base + __builtin_amdgcn_readlane(s.upto, i) - p.length) * heads;
      p.lh = __builtin_amdgcn_readfirstlane((int)((uint32_t)rest / (uint32_t)p.length));
      p.in = rest - p.lh * p.length;
      return p;
    }
    base += s.all;
    b0 += 64;
    s = sum_sequences(a, b0);
  }
  return {0, 0, 0, 0};
}
// Where workgroup w keeps a row of its part of a pair: it has at most one part with the pair's first block, at its end,
// and one without it, at its start.
__device__ inline int64_t share_row(const CacheAttnArgs& a, int w, bool begins, int row) {
  return (int64_t)(w * 2 + (begins ? 1 : 0)) * (16 * a.tiles) + row;
}

// The rows of one (sequence, head) pair, or a group of them, on its blocks `first` to `stop` - 1: the outputs, where these are
// all, or the partial results from row `base` of the workspace on.  NR tiles of 16 rows, W waves.  ONCE: the cache is read
// once and is not found in a cache by the next call (loads leave it out).
template <int D, bool FP8, int NR, int W, bool ONCE>
__device__ inline void attend_blocks(const CacheAttnArgs& a, int b, int lh, int group, int first, int stop, int64_t base) {
  using B = Cache8Block<D>;
  constexpr int KS = D / 32;  // products of a score: channels in steps of 32
  constexpr int ND = D / 16;  // output tiles: channels in steps of 16
  constexpr int kStride = D + 4;
  constexpr int kPolicy = ONCE ? 2 : 0;  // nontemporal
  // Four tiles leave no registers for a block ahead: it waits in LDS.  (In registers they spilled, and each reload waited
  // for all loads in flight: prompts 345 us, staged 257.  Rings of three blocks: 259; tiles of 32 rows, 32x32x16 products:
  // 263 to 296.)
  constexpr bool kStaged = NR == 4;
  constexpr int kCodes = 32 * D, kScales = 256, kWaveStage = kStaged ? 2 * kCodes + kScales : 0;
  constexpr int kJoin = 16 * kStride * 4;  // bytes of a wave's outputs of a tile
  constexpr int kWaveLds = kWaveStage > kJoin ? kWaveStage : kJoin;
  __shared__ alignas(16) uint8_t lds_wave[W * kWaveLds];
  __shared__ float2 lds_stat[W][16 * NR];
  const auto lds_o = [&](int w, int row, int x) { return (float*)(lds_wave + w * kWaveLds) + row * kStride + x; };

  int lane = threadIdx.x & 63;
  asm volatile("" : "+v"(lane));  // nothing that is formed from it is kept from one pair to the next
  const int wave = __builtin_amdgcn_readfirstlane((int)threadIdx.x >> 6), g = lane >> 4, n = lane & 15;
  const int layer = a.by_Hkv.div(lh), head = a.by_Hkv.mod(lh, layer);
  // 64 of the pair's pages from page0 on, one a lane
  int page0 = first >> a.c.page_shift;
  const int32_t* row_pages = a.c.table + (int64_t)b * a.c.max_pages;
  const auto load_pages = [&] {
    const uint32_t i = (uint32_t)(page0 + lane);
    const int page = (int)i < a.c.max_pages ? *(const int32_t*)((const char*)row_pages + 4 * (uint64_t)i) : -1;
    return page < a.c.num_pages ? page : -1;
  };
  int pages = load_pages();
  const StepSeq q = step_sequence(a.c, a.s, b);
  const RowGroup rg = row_group(a, q, group, 16 * NR);
  if (rg.row0 >= rg.rows || (first > 0 && first * kCacheBlock >= rg.keys)) return;

  uint32_t magic = 0x64646464u;
  asm("" : "+v"(magic));

  const int j0 = first + wave, j1 = min(stop, (rg.keys + kCacheBlock - 1) / kCacheBlock);  // every W-th block
  const int all_seen = rg.before + a.R.div(rg.row0) + 1;  // keys before this one are seen by every row of the group

  // Block j's part of the lane: keys' bytes and scale, values' bytes and scales, in registers or in LDS.
  u32x4 kw[2][D / 64], vw[D / 32], vs[2];
  uint32_t ks = 0;
  uint8_t* const stage = lds_wave + wave * kWaveLds;
  const uint32_t stage_at = __builtin_amdgcn_readfirstlane((int)(uintptr_t)(__attribute__((address_space(3))) uint8_t*)stage);
  constexpr int kCopies = D / 32;  // of a block's keys, and of its values
  // Block j of the wave, in turn; whether it has no page (then it is that of any page).
  const auto block_at = [&](int j, bool& missing) {
    if ((j >> a.c.page_shift) - page0 >= 64) {
      page0 = j >> a.c.page_shift;
      pages = load_pages();
    }
    int page = __builtin_amdgcn_readlane(pages, (j >> a.c.page_shift) - page0);
    missing = page < 0;
    page = max(page, 0);
    const int64_t at = (((int64_t)layer * a.c.num_pages + page) * a.c.Hkv + head) << a.c.page_shift;
    return a.c.pages + (at + (j & ((1 << a.c.page_shift) - 1))) * B::kBytes;
  };
  const auto buffer = [&](uint8_t* blk) { return __builtin_amdgcn_make_buffer_rsrc(blk, 0, B::kBytes, 0x00020000); };
  const auto load_keys = [&](uint8_t* blk) {
    if (kStaged) {
#pragma unroll
      for (int i = 0; i < kCopies; ++i) copy16<ONCE>(lane * 16, blk + B::kKeys + i * 1024, stage_at + i * 1024);
      return;
    }
    const auto r = buffer(blk);
#pragma unroll
    for (int u = 0; u < 2; ++u)
#pragma unroll
      for (int i = 0; i < D / 64; ++i)
        kw[u][i] = __builtin_amdgcn_raw_buffer_load_b128(r, lane * 16, B::kKeys + u * 16 * D + i * 1024, kPolicy);
    ks = __builtin_amdgcn_raw_buffer_load_b32(r, 0, B::kKeyScale, kPolicy);
  };
  const auto load_values = [&](uint8_t* blk) {
    if (kStaged) {
#pragma unroll
      for (int i = 0; i < kCopies; ++i) copy16<ONCE>(lane * 16, blk + B::kValues + i * 1024, stage_at + kCodes + i * 1024);
      copy4<ONCE>(min(lane, 32) * 4, blk + B::kValueScales, stage_at + 2 * kCodes);  // the values', then the keys'
      return;
    }
    const auto r = buffer(blk);
#pragma unroll
    for (int x = 0; x < D / 32; ++x) vw[x] = __builtin_amdgcn_raw_buffer_load_b128(r, lane * 16, B::kValues + x * 1024, kPolicy);
#pragma unroll
    for (int u = 0; u < 2; ++u) vs[u] = __builtin_amdgcn_raw_buffer_load_b128(r, g * 16, B::kValueScales + u * 64, kPolicy);
  };
  // What is staged, from LDS into registers.
  const auto read_keys = [&] {
#pragma unroll
    for (int u = 0; u < 2; ++u)
#pragma unroll
      for (int i = 0; i < D / 64; ++i) kw[u][i] = *(const u32x4*)(stage + u * 16 * D + i * 1024 + lane * 16);
  };
  const auto read_values = [&] {
#pragma unroll
    for (int x = 0; x < D / 32; ++x) vw[x] = *(const u32x4*)(stage + kCodes + x * 1024 + lane * 16);
  };
  const auto key = [&](int u, int s) {
    const u32x4 w = kw[u][s >> 1];
    return codes8<FP8>((s & 1) ? w.z : w.x, (s & 1) ? w.w : w.y, magic);
  };
  const auto value = [&](int x) {
    const u32x4 w = vw[x >> 1];
    return codes8<FP8>((x & 1) ? w.z : w.x, (x & 1) ? w.w : w.y, magic);
  };
  bool missing = false, next_missing = false;
  uint8_t* next = nullptr;
  if (j0 < j1) {
    next = block_at(j0, missing);
    next_missing = missing;
    load_keys(next);
    load_values(next);
  }

  // Queries as the products' B operand, each row brought near 2^14 by a power of two: in registers, or, for several
  // tiles, in LDS, one copy for the waves.
  constexpr bool kShared = NR > 1;
  __shared__ u32x4 lds_q[kShared ? NR * KS * 64 : 1];
  Frag qf[kShared ? 1 : NR][KS];
  __shared__ int lds_shift[kShared ? 16 * NR : 1];  // the powers of two that the rows were multiplied by
  int shift = 0;                                    // (one tile: the lane's row's)
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
    const bool finite = top < 0x7F80u;
    const int e = 15 - __builtin_amdgcn_frexp_expf(__uint_as_float(top << 16));  // the largest comes to [2^14, 2^15)
    shift = e;
    if (kShared && g == 0) lds_shift[r * 16 + n] = e;
#pragma unroll
    for (int s = 0; s < KS; ++s) {
      const uint32_t w[4] = {x[s].x, x[s].y, x[s].z, x[s].w};
      Frag f;
#pragma unroll
      for (int i = 0; i < 4; ++i) {
        f.w[i] = pack_h(__builtin_amdgcn_ldexpf(__uint_as_float(w[i] << 16), e),
                        __builtin_amdgcn_ldexpf(__uint_as_float(w[i] & 0xFFFF0000u), e));
        if (!finite) f.w[i] = 0x7E007E00u;  // every score of the row is NaN, also where a code is 0
      }
      if (!kShared)
        qf[kShared ? 0 : r][s] = f;
      else
        lds_q[(r * KS + s) * 64 + lane] = (u32x4){f.w[0], f.w[1], f.w[2], f.w[3]};
    }
  }
  if (kShared) __syncthreads();
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

  f32x4 acc[NR][ND];
  float m[NR], l[NR];
#pragma unroll
  for (int r = 0; r < NR; ++r) {
    m[r] = -kFar;
    l[r] = 0.0f;
#pragma unroll
    for (int x = 0; x < ND; ++x) acc[r][x] = (f32x4){0, 0, 0, 0};
  }

  if (kStaged && j0 < j1) {
    if (j0 + W < j1) next = block_at(j0 + W, next_missing);
    wait_copies_but<kCopies + 1>();
    read_keys();
    wait_lds_reads();
    load_keys(next);
  }
  // the group's tiles: a decoding sequence beside a prompt's chunk has one, whose weights alone are formed
  const int tiles = (rg.rows - rg.row0 + 15) / 16;
  for (int j = j0; j < j1; j += W) {
    const bool masked = missing || (j + 1) * kCacheBlock > all_seen;
    f32x4 xs[2][NR];
#pragma unroll
    for (int u = 0; u < 2; ++u)
#pragma unroll
      for (int r = 0; r < NR; ++r) xs[u][r] = (f32x4){0, 0, 0, 0};
    if (kStaged) {
      // Operands are read and formed a product ahead: the LDS's latency and the conversions pass beside the products
      // (257 -> 253 us).
      Frag qn[NR], kn[2];
#pragma unroll
      for (int r = 0; r < NR; ++r) qn[r] = query(r, 0);
#pragma unroll
      for (int u = 0; u < 2; ++u) kn[u] = key(u, 0);
#pragma unroll
      for (int s = 0; s < KS; ++s) {
        Frag q[NR], k[2];
#pragma unroll
        for (int r = 0; r < NR; ++r) q[r] = qn[r];
#pragma unroll
        for (int u = 0; u < 2; ++u) k[u] = kn[u];
        if (s + 1 < KS) {
#pragma unroll
          for (int r = 0; r < NR; ++r) qn[r] = query(r, s + 1);
        }
        __builtin_amdgcn_sched_barrier(0);
        if (s + 1 < KS) {
#pragma unroll
          for (int u = 0; u < 2; ++u) kn[u] = key(u, s + 1);
        }
#pragma unroll
        for (int u = 0; u < 2; ++u)
#pragma unroll
          for (int r = 0; r < NR; ++r) xs[u][r] = mfma(k[u], q[r], xs[u][r]);
        __builtin_amdgcn_sched_barrier(0);
      }
      wait_copies_but<kCopies>();  // the values and scales are there
#pragma unroll
      for (int u = 0; u < 2; ++u) vs[u] = *(const u32x4*)(stage + 2 * kCodes + u * 64 + g * 16);
      ks = *(const uint32_t*)(stage + 2 * kCodes + 128);
    } else {
#pragma unroll
      for (int u = 0; u < 2; ++u)
#pragma unroll
        for (int s = 0; s < KS; ++s) {
          const Frag k = key(u, s);
#pragma unroll
          for (int r = 0; r < NR; ++r) xs[u][r] = mfma(k, query(r, s), xs[u][r]);
        }
      // (after the last block, that block once more: no branch, so the registers stay in place)
      next = block_at(j + W < j1 ? j + W : j, next_missing);
      __builtin_amdgcn_sched_barrier(0);
    }
    if (masked) {  // scales that no row sees may be anything, those that one does not see must be finite
      if (missing) ks = 0;
#pragma unroll
      for (int u = 0; u < 2; ++u)
#pragma unroll
        for (int i = 0; i < 4; ++i)
          vs[u][i] = __float_as_uint(__builtin_amdgcn_fmed3f(__uint_as_float(vs[u][i]), 0.0f, -kNoMax));
    }
    // softmax_scale * log2(e) * the keys' scale, as a number near softmax_scale's and a power of two
    const float factor1 = a.scale_log2 * __builtin_amdgcn_frexp_mantf(__uint_as_float(ks));
    const int power = __builtin_amdgcn_frexp_expf(__uint_as_float(ks));
    if (!kStaged) load_keys(next);  // (the keys' scale is used)

    Frag pf[NR] = {};
#pragma unroll
    for (int r = 0; r < NR; ++r) {
      if (r > 0 && r >= tiles) break;
      float w[8], p[8], sum, top;
      // above 0 and finite, so that an unseen token's -infinity and a score of 0 stay that
      const float factor = __builtin_amdgcn_fmed3f(
          __builtin_amdgcn_ldexpf(factor1, power - (kShared ? lds_shift[r * 16 + n] : shift)), 0x1p-149f, -kNoMax);
#pragma unroll
      for (int i = 0; i < 8; ++i) w[i] = __uint_as_float(vs[i >> 2][i & 3]);
      if (masked) {
        const int row = rg.row0 + r * 16 + n;
        int seen = missing || row >= rg.rows ? 0 : rg.before + a.R.div(row) + 1;
        seen -= j * kCacheBlock + g * 4;
        asm volatile("" : "+v"(seen));
#pragma unroll
        for (int i = 0; i < 8; ++i)
          if ((i >> 2) * 16 + (i & 3) >= seen) xs[i >> 2][r][i & 3] = -INFINITY;
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
      if (__builtin_expect(__builtin_amdgcn_ballot_w64(fmaxf(top, sum * kLeastScale) > kLimit) != 0, false)) {
        float next = kNoMax;
#pragma unroll
        for (int i = 0; i < 8; ++i) {
          float v = w[i];
          asm volatile("" : "+v"(v));
          next = fmaxf(next, fmaf(xs[i >> 2][r][i & 3], factor, __builtin_amdgcn_logf(fmaxf(v, kLeastScale)) - kSet));
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
      if (kStaged && r == 0) {
        read_values();
        __builtin_amdgcn_sched_barrier(0);
      }
    }
    if (kStaged) {
      wait_lds_reads();
      load_values(next);
      wait_copies_but<kCopies + 1>();  // the next block's keys are there
      read_keys();
      __builtin_amdgcn_sched_barrier(0);
    }
    if (FP8 && masked) {  // e4m3 has NaN: bytes of tokens behind the last seen one are zeros
      uint32_t keep[2];
#pragma unroll
      for (int u = 0; u < 2; ++u) {
        const int first = j * kCacheBlock + u * 16 + g * 4, count = missing ? 0 : min(max(rg.keys - first, 0), 4);
        keep[u] = count == 4 ? 0xFFFFFFFFu : (1u << (8 * count)) - 1u;
      }
#pragma unroll
      for (int x = 0; x < D / 32; ++x)
#pragma unroll
        for (int i = 0; i < 4; ++i) vw[x][i] &= keep[i & 1];
    }
#pragma unroll
    for (int x = 0; x < ND; ++x) {
      const Frag v = value(x);
#pragma unroll
      for (int r = 0; r < NR; ++r) acc[r][x] = mfma(v, pf[r], acc[r][x]);
    }
    __builtin_amdgcn_sched_barrier(0);
    missing = next_missing;
    if (kStaged) {
      if (j + 2 * W < j1) next = block_at(j + 2 * W, next_missing);
      wait_lds_reads();
      load_keys(next);
    } else {
      load_values(next);
    }
  }
  if (kStaged) wait_copies_but<0>();  // the last ones land before the outputs take their place

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
      *(f32x4*)lds_o(wave, n, x * 16 + g * 4) = o;
    }
    __syncthreads();
    // a row's channels by 4 W threads
    constexpr int CH = D / (4 * W);
    const int row16 = (wave * 64 + lane) / (4 * W), c0 = (lane % (4 * W)) * CH;
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
        for (int w = 0; w < W; ++w) o[i] += *lds_o(w, row16, c0 + i);
      }
      const int t = a.R.div(row), hq = head * (int)a.R.d + a.R.mod(row, t);
      const int64_t token = q.row + t;
      if (first == 0 && stop * kCacheBlock >= rg.keys) {
        store_output<CH>(a, layer, token, hq, c0, o, st);
      } else {
        if (c0 == 0) a.stat[base + row] = st;
#pragma unroll
        for (int i = 0; i < CH; ++i) a.part[(base + row) * D + c0 + i] = o[i];
      }
    }
  }
}

// A workgroup a chunk of a pair's tokens and group of its rows.
template <int D, bool FP8, int NR, int W, bool ONCE>
__global__ __launch_bounds__(64 * W, (NR == 1 ? 4 : NR == 2 ? 3 : 2) + (D == 64)) void k_cache8_attention(CacheAttnArgs a) {
  const int rest = a.heads.div((int)blockIdx.x), lh = a.heads.mod((int)blockIdx.x, rest), b = blockIdx.y;
  const int chunk = a.by_groups.div(rest), group = a.by_groups.mod(rest, chunk), blocks = a.chunk / kCacheBlock;
  attend_blocks<D, FP8, NR, W, ONCE>(a, b, lh, group, chunk * blocks, (chunk + 1) * blocks, partial_row(a, chunk, b, lh, 0));
}

// A workgroup a share.
template <int D, bool FP8, int NR, bool ONCE>
__global__ __launch_bounds__(256, 2) void k_cache8_shares(CacheAttnArgs a) {
  const SequenceSums head = sum_sequences(a, 0);
  const int all = sum_all(a, head) * (int)a.heads.d, share = share_of(all, a.chunks);
  if ((int64_t)blockIdx.x * share >= all) return;
  int at = (int)blockIdx.x * share;
  const int end = (int)min((uint32_t)at + (uint32_t)share, (uint32_t)all);
  ShareAt pair = share_at(a, head, at);
  while (pair.length > 0) {
    const int ends = min(pair.length, pair.in + (end - at)), first = max(pair.in - kStart, 0), stop = ends - kStart;
    if (stop <= first) return;  // (the share ends before the pair's first block)
    attend_blocks<D, FP8, NR, 4, ONCE>(a, pair.b, pair.lh, 0, first, stop, share_row(a, (int)blockIdx.x, first == 0, 0));
    at += ends - pair.in;
    if (at >= end) return;
    pair.in = 0;
    if (++pair.lh == (int)a.heads.d) {
      pair.lh = 0;
      do pair.length = __builtin_amdgcn_readfirstlane(pair_length(a, ++pair.b));
      while (pair.length == 0 && pair.b < a.c.batch);
    }
    __syncthreads();
  }
}

// Joins the parts of a row whose pair lies in several shares: by WPR waves, whose groups of D / 4 lanes take every kGroups-th
// part, four channels a lane, each with a reference of its own.  A workgroup has several rows of a pair.  A launch and
// dependent loads (lengths, statistics, parts) bound it: 4.5 to 5 us.  One wave a row for few parts: 16 sequences' drafts 4.85
// us (four: 5.4), 48 sequences 4.9 (6.5).
template <int D, int WPR>
__global__ __launch_bounds__(kMergeThreads) void k_cache8_join_shares(CacheAttnArgs a) {
  constexpr int kLanes = D / 4;
  constexpr int kGroups = WPR * 64 / kLanes;
  constexpr int kRows = kMergeThreads / 64 / WPR;
  __shared__ f32x4 lds_o[kRows][kGroups][kLanes];
  __shared__ float2 lds_stat[kRows][kGroups];
  const int rest = a.heads.div((int)blockIdx.x), lh = a.heads.mod((int)blockIdx.x, rest), b = blockIdx.y;
  const int mine = threadIdx.x / (WPR * 64);  // row of the workgroup
  const int row = rest * kRows + mine;
  const int part = threadIdx.x % (WPR * 64) / kLanes, lane = threadIdx.x % kLanes;
  const StepSeq q = step_sequence(a.c, a.s, b);
  // where the pair lies among all
  SequenceSums s64 = sum_sequences(a, 0);
  const int heads = (int)a.heads.d, share = share_of(sum_all(a, s64) * heads, a.chunks);
  int before = 0;
  for (int b0 = 64; b0 <= b; b0 += 64) {
    before += s64.all;
    s64 = sum_sequences(a, b0);
  }
  const int length = __builtin_amdgcn_readlane(s64.mine, b & 63);
  const int from = (before + __builtin_amdgcn_readlane(s64.upto, b & 63) - length) * heads + lh * length;
  const int w0 = (uint32_t)(from + kStart) / (uint32_t)share, w1 = (uint32_t)(from + length - 1) / (uint32_t)share;
  const bool in = row < q.count * (int)a.R.d && w0 != w1;
  float2 st = make_float2(kNoMax, 0.0f);
  f32x4 o = {0, 0, 0, 0};
  if (in) {
#pragma unroll 4
    for (int w = w0 + part; w <= w1; w += kGroups) {
      const int64_t i = share_row(a, w, w == w0, row);
      const float2 s = a.stat[i];
      const f32x4 p = *(const f32x4*)(a.part + i * D + lane * 4);
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
  const int layer = a.by_Hkv.div(lh), head = a.by_Hkv.mod(lh, layer);
  const int t = a.R.div(row), hq = head * (int)a.R.d + a.R.mod(row, t);
  const float x[4] = {o.x, o.y, o.z, o.w};
  store_output<4>(a, layer, q.row + t, hq, lane * 4, x, st);
}

}  // namespace

// Bytes of a cache (by the call's bounds) from which on its loads are nontemporal: a step's other layers and their weights push
// it out of the chip's 256 MB before the next call on it.  Found in no cache, with and without: 32 sequences of about 2300 tokens
// 30.8 us, 33.6; eight of 13000 44.2, 49.9; one of 13215 14.6, 15.8; one of 2000 (4 MB) 10.5, 10.2.  Where one layer is called again
// and again, or a model's layers and weights stay below that together, they mostly cost: 32 of 300 (20 MB) 8.5, 7.3; one of 13107
// 14.0, 12.7; 32 of 2300 26.3, 25.3; 48 of 2000 (200 MB) 38.1, 32.4, the most seen; one of 40000 19.6, 20.6.  A call whose bound is
// far above what its sequences hold is streamed too (eight of 1000 with a bound of 131072: 12.0 either way).
constexpr int64_t kStreamed = 16 << 20;

// The 4-bit cache's division into rows and chunks, but that decoding calls which it would split are cut into shares on the
// device (chunk 0), one a CU.  Whole sequences stay whole: 32 of 2300 tokens take 25.1 us in
// eight waves each, in shares 27.8; 64 of 1024 29.2, 35.9; 64 of 20 to 3000 52.3, 47.8.
CachePlan cache8_plan(int32_t L, int32_t Hq, int32_t Hkv, int32_t head_dim, int32_t batch, int32_t max_new,
                      int32_t max_len) {
  constexpr int64_t kCus = 256;
  CachePlan p = cache_plan(L, Hq, Hkv, head_dim, batch, max_new, max_len);
  const int64_t heads = (int64_t)L * Hkv * batch, length = ((int64_t)max_len + kCacheBlock - 1) / kCacheBlock + kStart;
  p.once = p.row_groups == 1 && (double)heads * max_len * (double)cache8_block_bytes(head_dim) / kCacheBlock >
                                    (double)kStreamed;
  if (p.tiles < 4 && p.chunks > 1 && batch <= kMostSequences && heads * length < (int64_t)1 << 31) {
    p.chunk = 0;
    p.chunks = (int32_t)kCus;
  }
  // A workgroup's two partial results, of 32 rows at most, in the bound of cache_plan, which never falls.
  if (max_len > 512) {
    const int64_t rows = 32 * 2 * std::min(kCus, heads * length / kLeastShare + 1);
    const size_t o_off = ((size_t)rows * sizeof(float2) + 255) / 256 * 256;
    const size_t total = o_off + (size_t)rows * head_dim * sizeof(float);
    if (p.chunk == 0) p.o_off = o_off;
    p.total = std::max(p.total, total);
  }
  return p;
}

namespace {

template <int D, bool FP8, int NR, int W>
void launch_chunks(const CacheAttnArgs& a, dim3 grid, hipStream_t stream) {
  if (a.once)
    hipLaunchKernelGGL((k_cache8_attention<D, FP8, NR, W, true>), grid, dim3(64 * W), 0, stream, a);
  else
    hipLaunchKernelGGL((k_cache8_attention<D, FP8, NR, W, false>), grid, dim3(64 * W), 0, stream, a);
}

template <int D, bool FP8, int NR>
void launch_shares(const CacheAttnArgs& a, hipStream_t stream) {
  if (a.once)
    hipLaunchKernelGGL((k_cache8_shares<D, FP8, NR, true>), dim3(a.chunks), dim3(256), 0, stream, a);
  else
    hipLaunchKernelGGL((k_cache8_shares<D, FP8, NR, false>), dim3(a.chunks), dim3(256), 0, stream, a);
}

template <int D, bool FP8>
hipError_t launch_attention(const CacheAttnArgs& a, hipStream_t stream) {
  const unsigned heads = (unsigned)(a.c.L * a.c.Hkv), batch = (unsigned)a.c.batch;
  const bool shares = a.chunk == 0;
  const dim3 grid(heads * a.row_groups * a.chunks, batch);
  if (shares && a.tiles == 1) launch_shares<D, FP8, 1>(a, stream);
  else if (shares) launch_shares<D, FP8, 2>(a, stream);
  else if (a.tiles == 1 && a.waves == 8) launch_chunks<D, FP8, 1, 8>(a, grid, stream);
  else if (a.tiles == 1) launch_chunks<D, FP8, 1, 4>(a, grid, stream);
  else if (a.tiles == 2) launch_chunks<D, FP8, 2, 4>(a, grid, stream);
  else launch_chunks<D, FP8, 4, 4>(a, grid, stream);
  const hipError_t e = hipGetLastError();
  if (e != hipSuccess || a.chunks == 1) return e;
  const unsigned rows = heads * a.row_groups * a.tiles * 16;  // 16 a tile
  const unsigned pair_rows = a.R.d * (unsigned)a.s.max_new;
  if (shares && (unsigned)a.chunks <= 8 * heads * batch)  // few parts of a pair
    hipLaunchKernelGGL((k_cache8_join_shares<D, 1>), dim3(heads * ((pair_rows + 3) / 4), batch), dim3(kMergeThreads), 0, stream, a);
  else if (shares)
    hipLaunchKernelGGL((k_cache8_join_shares<D, 4>), dim3(heads * pair_rows, batch), dim3(kMergeThreads), 0, stream, a);
  else if (a.chunks >= 8)
    hipLaunchKernelGGL((k_cache_merge<D, 4>), dim3(rows, batch), dim3(kMergeThreads), 0, stream, a);
  else
    hipLaunchKernelGGL((k_cache_merge<D, 1>), dim3(rows / 4, batch), dim3(kMergeThreads), 0, stream, a);
  return hipGetLastError();
}

}  // namespace

hipError_t launch_cache8_attention(const CacheAttnArgs& a, bool fp8, int head_dim, hipStream_t stream) {
  if (head_dim == 128) return fp8 ? launch_attention<128, true>(a, stream) : launch_attention<128, false>(a, stream);
  return fp8 ? launch_attention<64, true>(a, stream) : launch_attention<64, false>(a, stream);
}

}  // namespace tp

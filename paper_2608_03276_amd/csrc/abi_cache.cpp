// C-ABI layer of the paged 4-bit cache: validation and dispatch.  Nothing is enqueued unless every
// host argument is valid; what lies on the device (lengths, page table, offsets, positions) is checked
// by the kernels, which leave out what is out of range.
#include <limits.h>
#include <math.h>
#include <string.h>

#include <algorithm>

#include "abi_internal.h"
#include "cache_block.h"

namespace {

using tp::aligned16;
using tp::check_dims;
using tp::fail;
using tp::hip_fail;
using tp::ok;

bool aligned4(const void* p) { return ((uintptr_t)p & 3u) == 0; }

int page_shift_of(int32_t page_tokens) {
  for (int s = 0; s < 4; ++s)
    if (page_tokens == (tp::kCacheBlock << s)) return s;
  return -1;
}

// `d` has passed check_dims.
tp_status check_cache(const tp_dims* d, const tp_cache* c, bool need_lens, tp::CacheArgs& a) {
  if (!c) return fail(TP_ERR_NULL, "cache is NULL");
  if (!c->pages || !c->page_table || (need_lens && !c->lens))
    return fail(TP_ERR_NULL, "the cache's pages, page_table and lens must be non-NULL");
  if (!aligned16(c->pages)) return fail(TP_ERR_PARAM, "pages must be 16-byte aligned");
  if (!aligned4(c->page_table) || !aligned4(c->lens))
    return fail(TP_ERR_PARAM, "page_table and lens must be 4-byte aligned");
  const int shift = page_shift_of(c->page_tokens);
  if (shift < 0) return fail(TP_ERR_UNSUPPORTED, "page_tokens %d not supported (32, 64, 128 or 256)", c->page_tokens);
  if (c->batch < 1 || c->max_pages < 1 || c->num_pages < 1)
    return fail(TP_ERR_SHAPE, "the cache's batch, max_pages and num_pages must be >= 1");
  if (c->batch > 65535) return fail(TP_ERR_UNSUPPORTED, "batch %d exceeds 65535", c->batch);
  if (c->num_pages > INT32_MAX) return fail(TP_ERR_UNSUPPORTED, "num_pages exceeds 2^31 - 1");
  if ((int64_t)c->max_pages * c->page_tokens > ((int64_t)1 << 30))
    return fail(TP_ERR_UNSUPPORTED, "max_pages * page_tokens exceeds 2^30");
  a.pages = (uint8_t*)c->pages;
  a.table = c->page_table;
  a.lens = c->lens;
  a.num_pages = c->num_pages;
  a.max_pages = c->max_pages;
  a.batch = c->batch;
  a.page_shift = shift;
  a.max_len = c->max_pages * c->page_tokens;
  a.L = d->num_layers;
  a.Hkv = d->num_kv_heads;
  return TP_OK;
}

tp_status check_step(const tp_cache* c, const tp_step* s, tp::StepArgs& a) {
  if (!s) return fail(TP_ERR_NULL, "step is NULL");
  if (s->total < 1 || s->max_new < 1) return fail(TP_ERR_SHAPE, "the step's total and max_new must be >= 1");
  if (!s->offsets && (s->max_new != 1 || s->total < c->batch))
    return fail(TP_ERR_SHAPE, "a step without offsets has max_new = 1 and total >= batch");
  if (!aligned4(s->offsets)) return fail(TP_ERR_PARAM, "the step's offsets must be 4-byte aligned");
  a.offsets = s->offsets;
  a.total = s->total;
  a.max_new = s->max_new;
  return TP_OK;
}

// Rows [L][total][heads][d].  An output's rows must not overlap: ordered by stride, each dimension's
// stride covers the extent of those before it.
tp_status check_rows(const tp_dims* d, int32_t heads, int32_t total, const tp_rows* r, bool output, const char* what,
                     tp::RowsArgs& a) {
  if (!r || !r->data) return fail(TP_ERR_NULL, "%s must be non-NULL", what);
  if (!aligned16(r->data)) return fail(TP_ERR_PARAM, "%s must be 16-byte aligned", what);
  struct Dim {
    int64_t stride, count;
  } dims[3] = {{r->layer_stride, d->num_layers}, {r->token_stride, total}, {r->head_stride, heads}};
  for (const Dim& x : dims) {
    if (x.stride < 0 || x.stride % 8 != 0)
      return fail(TP_ERR_PARAM, "%s: strides must be multiples of 8 elements, >= 0", what);
    if (x.count > 1 && x.stride > ((int64_t)1 << 60) / x.count)
      return fail(TP_ERR_UNSUPPORTED, "%s: strides reach beyond 2^60 elements", what);
  }
  if (output) {
    std::sort(dims, dims + 3, [](const Dim& x, const Dim& y) { return x.stride < y.stride; });
    int64_t extent = d->head_dim;
    for (const Dim& x : dims) {
      if (x.count == 1) continue;
      if (x.stride < extent) return fail(TP_ERR_SHAPE, "%s: rows overlap", what);
      extent += (x.count - 1) * x.stride;
    }
  }
  a.data = (uint16_t*)r->data;
  a.layer = r->layer_stride;
  a.token = r->token_stride;
  a.head = r->head_stride;
  return TP_OK;
}

// Rows of q heads written where they are read: every row in its own place.
bool in_place_or_apart(const tp_dims* d, int32_t total, const tp_rows* from, const tp_rows* to) {
  return from->data != to->data || ((d->num_layers == 1 || from->layer_stride == to->layer_stride) &&
                                    (total == 1 || from->token_stride == to->token_stride) &&
                                    (d->num_q_heads == 1 || from->head_stride == to->head_stride));
}

// A launch's x dimension holds fewer than 2^32 work-items.
bool fits_grid(double workgroups, double threads = 256.0) { return workgroups * threads < 0x1p32; }

// Makes the stream's device current for the launch, and the caller's again afterwards.
class OnDevice {
 public:
  explicit OnDevice(hipStream_t st) {
    int dev = 0;
    if (st == nullptr) return;
    if (hipStreamGetDevice(st, &dev) != hipSuccess || hipGetDevice(&cur_) != hipSuccess || dev == cur_) return;
    changed_ = hipSetDevice(dev) == hipSuccess;
  }
  ~OnDevice() {
    if (changed_) (void)hipSetDevice(cur_);
  }
  OnDevice(const OnDevice&) = delete;

 private:
  int cur_ = 0;
  bool changed_ = false;
};

}  // namespace

extern "C" {

size_t tp_cache_page_bytes(const tp_dims* dims, int32_t page_tokens) {
  if (check_dims(dims) != TP_OK) return 0;
  const int shift = page_shift_of(page_tokens);
  if (shift < 0) {
    fail(TP_ERR_UNSUPPORTED, "page_tokens %d not supported (32, 64, 128 or 256)", page_tokens);
    return 0;
  }
  ok();
  return (size_t)tp::cache_block_bytes(dims->head_dim) << shift;
}

tp_status tp_cache_load(const tp_dims* dims, const tp_cache* cache, const int64_t* kept_offsets, const void* k,
                        const void* v_q, const float* scales, int32_t bits, void* stream) {
  tp::CacheWriteArgs a;
  memset(&a, 0, sizeof a);
  tp_status s = check_dims(dims);
  if (s == TP_OK) s = check_cache(dims, cache, false, a.c);
  if (s != TP_OK) return s;
  if (cache->batch > TP_MAX_BATCH)
    return fail(TP_ERR_UNSUPPORTED, "batch %d exceeds TP_MAX_BATCH (%d)", cache->batch, TP_MAX_BATCH);
  s = tp::check_offsets(kept_offsets, cache->batch, "kept_offsets", true);
  if (s != TP_OK) return s;
  if (!k || !v_q || !scales) return fail(TP_ERR_NULL, "k, v_q and scales must be non-NULL");
  if (!aligned16(k) || !aligned16(v_q) || !aligned16(scales))
    return fail(TP_ERR_PARAM, "tensor pointers must be 16-byte aligned");
  if (bits < 2 || bits > 8) return fail(TP_ERR_PARAM, "bits %d outside [2, 8]", bits);
  if (bits > 4) return fail(TP_ERR_UNSUPPORTED, "the pages hold codes of at most 4 bits (got %d)", bits);
  int64_t most = 0;
  for (int b = 0; b <= cache->batch; ++b) {
    a.kept_off[b] = kept_offsets[b];
    if (b == 0) continue;
    const int64_t n = kept_offsets[b] - kept_offsets[b - 1];
    if (n > a.c.max_len)
      return fail(TP_ERR_SHAPE, "sequence %d holds %lld tokens, its pages %d", b - 1, (long long)n, a.c.max_len);
    most = std::max(most, n);
  }
  if (most == 0) return ok();
  const int64_t d = dims->head_dim, tot = kept_offsets[cache->batch];
  a.blocks = (int32_t)((most + tp::kCacheBlock - 1) / tp::kCacheBlock);
  if (!fits_grid((double)a.blocks * dims->num_layers * dims->num_kv_heads))
    return fail(TP_ERR_UNSUPPORTED, "kept_offsets: sequences too long for one launch");
  a.k = {(uint16_t*)k, dims->num_kv_heads * tot * d, d, tot * d};
  a.v_q = (const uint8_t*)v_q;
  a.v_scales = scales;
  OnDevice on((hipStream_t)stream);
  const hipError_t e = tp::launch_cache_load(a, dims->head_dim, (hipStream_t)stream);
  if (e != hipSuccess) return hip_fail(e, "tp_cache_load launch");
  return ok();
}

tp_status tp_cache_append(const tp_dims* dims, const tp_cache* cache, const tp_step* step, const tp_rows* k,
                          const tp_rows* v, const int32_t* positions, const tp_rope* rope, const tp_rows* q,
                          const tp_rows* q_out, void* stream) {
  tp::CacheWriteArgs a;
  memset(&a, 0, sizeof a);
  tp_status s = check_dims(dims);
  if (s == TP_OK) s = check_cache(dims, cache, true, a.c);
  if (s == TP_OK) s = check_step(cache, step, a.s);
  if (s == TP_OK) s = check_rows(dims, dims->num_kv_heads, step->total, k, false, "k", a.k);
  if (s == TP_OK) s = check_rows(dims, dims->num_kv_heads, step->total, v, false, "v", a.v);
  if (s != TP_OK) return s;
  if ((q == nullptr) != (q_out == nullptr)) return fail(TP_ERR_NULL, "q and q_out must both be given or both NULL");
  if (q && !rope) return fail(TP_ERR_NULL, "q is rotated: rope must be non-NULL");
  if (rope) {
    if (!rope->cos_sin || !positions) return fail(TP_ERR_NULL, "the rope's cos_sin and positions must be non-NULL");
    if (!aligned16(rope->cos_sin)) return fail(TP_ERR_PARAM, "cos_sin must be 16-byte aligned");
    if (!aligned4(positions)) return fail(TP_ERR_PARAM, "positions must be 4-byte aligned");
    if (rope->num_positions < 1) return fail(TP_ERR_SHAPE, "num_positions must be >= 1");
    if (rope->style != TP_ROPE_HALVES && rope->style != TP_ROPE_PAIRS)
      return fail(TP_ERR_PARAM, "unknown rope style %d", rope->style);
    if (rope->rotary_dim < 16 || rope->rotary_dim % 16 != 0 || rope->rotary_dim > dims->head_dim)
      return fail(TP_ERR_PARAM, "rotary_dim %d is not a multiple of 16 in [16, %d]", rope->rotary_dim, dims->head_dim);
    a.positions = positions;
    a.cos_sin = rope->cos_sin;
    a.num_positions = std::min<int64_t>(rope->num_positions, (int64_t)INT32_MAX + 1);
    a.rotary_dim = rope->rotary_dim;
    a.pairs = rope->style == TP_ROPE_PAIRS;
  }
  if (q) {
    s = check_rows(dims, dims->num_q_heads, step->total, q, false, "q", a.q);
    if (s == TP_OK) s = check_rows(dims, dims->num_q_heads, step->total, q_out, true, "q_out", a.q_out);
    if (s != TP_OK) return s;
    if (!in_place_or_apart(dims, step->total, q, q_out))
      return fail(TP_ERR_SHAPE, "q_out on q's memory must have q's strides");
  }
  a.Hq = dims->num_q_heads;
  // n consecutive tokens lie in at most (n + 30) / 32 + 1 blocks
  a.blocks = (int32_t)(((int64_t)step->max_new + tp::kCacheBlock - 2) / tp::kCacheBlock + 1);
  const double heads = (double)dims->num_layers * dims->num_kv_heads;
  if (!fits_grid(heads * a.blocks * cache->batch + (q ? (double)dims->num_layers * step->total : 0.0), 512.0))
    return fail(TP_ERR_UNSUPPORTED, "step too long for one launch");
  OnDevice on((hipStream_t)stream);
  const hipError_t e = tp::launch_cache_append(a, dims->head_dim, (hipStream_t)stream);
  if (e != hipSuccess) return hip_fail(e, "tp_cache_append launch");
  return ok();
}

}  // extern "C"

// The attention's arguments without its tensors, and its plan.
static tp_status prepare_attention(const tp_dims* dims, const tp_cache* cache, const tp_step* step, int64_t max_len,
                                   tp::CacheAttnArgs& a, tp::CachePlan& plan) {
  memset(&a, 0, sizeof a);
  tp_status s = check_dims(dims);
  if (s == TP_OK) s = check_cache(dims, cache, true, a.c);
  if (s == TP_OK) s = check_step(cache, step, a.s);
  if (s != TP_OK) return s;
  if (max_len < 1 || max_len > a.c.max_len)
    return fail(TP_ERR_SHAPE, "max_len %lld outside [1, %d]", (long long)max_len, a.c.max_len);
  a.c.max_len = (int32_t)max_len;
  a.Hq = dims->num_q_heads;
  a.R = tp::Divisor::of(dims->num_q_heads / dims->num_kv_heads);
  const double rows = (double)dims->num_layers * dims->num_q_heads * step->max_new * cache->batch;
  if ((double)a.R.d * step->max_new > 0x1p26 || rows > 0x1p32)
    return fail(TP_ERR_UNSUPPORTED, "step of %d tokens too long for these dims", step->total);
  plan = tp::cache_plan(a.c.L, a.Hq, a.c.Hkv, dims->head_dim, a.c.batch, a.s.max_new, a.c.max_len);
  if (!fits_grid((double)dims->num_layers * dims->num_kv_heads * plan.row_groups * plan.chunks) ||
      !fits_grid((double)dims->num_layers * dims->num_kv_heads * plan.row_groups * plan.tiles * 16.0))
    return fail(TP_ERR_UNSUPPORTED, "step or sequences too long for one launch");
  a.heads = tp::Divisor::of((int64_t)dims->num_layers * dims->num_kv_heads);
  a.by_Hkv = tp::Divisor::of(dims->num_kv_heads);
  a.by_groups = tp::Divisor::of(plan.row_groups);
  a.by_chunk = tp::Divisor::of(plan.chunk);
  a.tiles = plan.tiles;
  a.row_groups = plan.row_groups;
  a.chunk = plan.chunk;
  a.chunks = plan.chunks;
  a.waves = plan.waves;
  a.once = plan.once;
  return TP_OK;
}

extern "C" {

tp_status tp_cache_workspace_size(const tp_dims* dims, const tp_cache* cache, const tp_step* step, int64_t max_len,
                                  size_t* bytes) {
  if (!bytes) return fail(TP_ERR_NULL, "bytes is NULL");
  tp::CacheAttnArgs a;
  tp::CachePlan plan;
  const tp_status s = prepare_attention(dims, cache, step, max_len, a, plan);
  if (s != TP_OK) return s;
  *bytes = plan.total;
  return ok();
}

tp_status tp_cache_attention(const tp_dims* dims, const tp_cache* cache, const tp_step* step, const tp_rows* q,
                             float softmax_scale, int64_t max_len, const tp_rows* o, float* lse, void* workspace,
                             size_t ws_bytes, void* stream) {
  tp::CacheAttnArgs a;
  tp::CachePlan plan;
  tp_status s = prepare_attention(dims, cache, step, max_len, a, plan);
  if (s == TP_OK) s = check_rows(dims, dims->num_q_heads, step->total, q, false, "q", a.q);
  if (s == TP_OK) s = check_rows(dims, dims->num_q_heads, step->total, o, true, "o", a.o);
  if (s != TP_OK) return s;
  if (!aligned4(lse)) return fail(TP_ERR_PARAM, "lse must be 4-byte aligned");
  a.scale_log2 = (float)((double)softmax_scale * 1.4426950408889634);
  if (!(softmax_scale > 0.0f) || !isfinite(a.scale_log2))
    return fail(TP_ERR_PARAM, "softmax_scale must be finite and > 0");
  if (plan.total > 0 && (!workspace || ws_bytes < plan.total))
    return fail(TP_ERR_WORKSPACE, "workspace needs %zu bytes (got %zu%s)", plan.total, ws_bytes,
                workspace ? "" : ", NULL");
  if (((uintptr_t)workspace & 255u) != 0) return fail(TP_ERR_WORKSPACE, "workspace must be 256-byte aligned");
  if (!in_place_or_apart(dims, step->total, q, o)) return fail(TP_ERR_SHAPE, "o on q's memory must have q's strides");
  a.lse = lse;
  a.stat = (float2*)((char*)workspace + plan.stat_off);
  a.part = (float*)((char*)workspace + plan.o_off);
  OnDevice on((hipStream_t)stream);
  const hipError_t e = tp::launch_cache_attention(a, dims->head_dim, (hipStream_t)stream);
  if (e != hipSuccess) return hip_fail(e, "tp_cache_attention launch");
  return ok();
}

tp_status tp_cache_read(const tp_dims* dims, const tp_cache* cache, const tp_batch* batch, const int64_t* first,
                        void* k_out, void* v_out, void* stream) {
  tp::CacheReadArgs a;
  memset(&a, 0, sizeof a);
  tp_status s = check_dims(dims);
  if (s == TP_OK) s = check_cache(dims, cache, true, a.c);
  if (s != TP_OK) return s;
  if (!batch) return fail(TP_ERR_NULL, "batch is NULL");
  if (batch->batch != cache->batch)
    return fail(TP_ERR_SHAPE, "batch of %d sequences for a cache of %d", batch->batch, cache->batch);
  if (batch->batch > TP_MAX_BATCH)
    return fail(TP_ERR_UNSUPPORTED, "batch %d exceeds TP_MAX_BATCH (%d)", batch->batch, TP_MAX_BATCH);
  s = tp::check_offsets(batch->ctx_offsets, batch->batch, "ctx_offsets", true);
  if (s != TP_OK) return s;
  if (!k_out || !v_out) return fail(TP_ERR_NULL, "k_out and v_out must be non-NULL");
  if (!aligned16(k_out) || !aligned16(v_out)) return fail(TP_ERR_PARAM, "tensor pointers must be 16-byte aligned");
  int64_t most = 0;
  for (int b = 0; b <= batch->batch; ++b) {
    a.off[b] = batch->ctx_offsets[b];
    if (b == batch->batch) break;
    const int64_t n = batch->ctx_offsets[b + 1] - batch->ctx_offsets[b], f = first ? first[b] : 0;
    if (f < 0 || f > ((int64_t)1 << 30) || n > ((int64_t)1 << 30) - f)
      return fail(TP_ERR_SHAPE, "range of sequence %d (%lld tokens from %lld) outside [0, 2^30]", b, (long long)n,
                  (long long)f);
    a.first[b] = f;
    if (n > 0) most = std::max(most, (f + n - 1) / tp::kCacheBlock - f / tp::kCacheBlock + 1);
  }
  if (most == 0) return ok();
  a.blocks = (int32_t)most;
  if (!fits_grid((double)a.blocks * dims->num_layers * dims->num_kv_heads))
    return fail(TP_ERR_UNSUPPORTED, "ctx_offsets: ranges too long for one launch");
  a.k = (uint16_t*)k_out;
  a.v = (uint16_t*)v_out;
  OnDevice on((hipStream_t)stream);
  const hipError_t e = tp::launch_cache_read(a, dims->head_dim, (hipStream_t)stream);
  if (e != hipSuccess) return hip_fail(e, "tp_cache_read launch");
  return ok();
}

}  // extern "C"

// C-ABI layer of the paged 8-bit cache: validation and dispatch, as abi_cache.cpp's for the 4-bit one.
#include "abi_cache.h"
#include "cache8_block.h"

namespace {

using tp::check_dims;
using tp::fail;
using tp::hip_fail;
using tp::ok;
using namespace tp::cache_abi;

// The cache's code format; dims and the rest of the cache are checked with the call.
tp_status check_format(const tp_cache8* c) {
  if (!c) return fail(TP_ERR_NULL, "cache is NULL");
  if (c->qfmt != TP_QFMT_INT && c->qfmt != TP_QFMT_FP8_E4M3) return fail(TP_ERR_PARAM, "unknown qfmt %d", c->qfmt);
  return TP_OK;
}

bool fp8_of(const tp_cache8* c) { return c->qfmt == TP_QFMT_FP8_E4M3; }

}  // namespace

extern "C" {

size_t tp_cache8_page_bytes(const tp_dims* dims, int32_t page_tokens) {
  if (check_dims(dims) != TP_OK) return 0;
  const int shift = page_shift_of(page_tokens);
  if (shift < 0) {
    fail(TP_ERR_UNSUPPORTED, "page_tokens %d not supported (32, 64, 128 or 256)", page_tokens);
    return 0;
  }
  ok();
  return (size_t)tp::cache8_block_bytes(dims->head_dim) << shift;
}

tp_status tp_cache8_load(const tp_dims* dims, const tp_cache8* cache, const int64_t* kept_offsets, const void* k,
                         const void* v_q, const float* scales, int32_t bits, void* stream) {
  tp::Cache8WriteArgs a;
  tp_status s = check_format(cache);
  if (s == TP_OK) s = prepare_load(dims, &cache->cache, kept_offsets, k, v_q, scales, a);
  if (s != TP_OK) return s;
  a.fp8 = fp8_of(cache);
  if (!a.fp8 && (bits < 2 || bits > 8)) return fail(TP_ERR_PARAM, "bits %d outside [2, 8]", bits);
  a.nibbles = !a.fp8 && bits <= 4;
  if (a.blocks == 0) return ok();
  OnDevice on((hipStream_t)stream);
  const hipError_t e = tp::launch_cache8_load(a, dims->head_dim, (hipStream_t)stream);
  if (e != hipSuccess) return hip_fail(e, "tp_cache8_load launch");
  return ok();
}

tp_status tp_cache8_append(const tp_dims* dims, const tp_cache8* cache, const tp_step* step, const tp_rows* k,
                           const tp_rows* v, const int32_t* positions, const tp_rope* rope, const tp_rows* q,
                           const tp_rows* q_out, void* stream) {
  tp::Cache8WriteArgs a;
  tp_status s = check_format(cache);
  if (s == TP_OK) s = prepare_append(dims, &cache->cache, step, k, v, positions, rope, q, q_out, a);
  if (s != TP_OK) return s;
  a.fp8 = fp8_of(cache);
  a.nibbles = 0;
  OnDevice on((hipStream_t)stream);
  const hipError_t e = tp::launch_cache8_append(a, dims->head_dim, (hipStream_t)stream);
  if (e != hipSuccess) return hip_fail(e, "tp_cache8_append launch");
  return ok();
}

tp_status tp_cache8_workspace_size(const tp_dims* dims, const tp_cache8* cache, const tp_step* step, int64_t max_len,
                                   size_t* bytes) {
  if (!bytes) return fail(TP_ERR_NULL, "bytes is NULL");
  tp::CacheAttnArgs a;
  tp::CachePlan plan;
  tp_status s = check_format(cache);
  if (s == TP_OK) s = prepare_attention(tp::cache8_plan, dims, &cache->cache, step, max_len, a, plan);
  if (s != TP_OK) return s;
  *bytes = plan.total;
  return ok();
}

tp_status tp_cache8_attention(const tp_dims* dims, const tp_cache8* cache, const tp_step* step, const tp_rows* q,
                              float softmax_scale, int64_t max_len, const tp_rows* o, float* lse, void* workspace,
                              size_t ws_bytes, void* stream) {
  tp::CacheAttnArgs a;
  tp::CachePlan plan;
  tp_status s = check_format(cache);
  if (s == TP_OK) s = prepare_attention(tp::cache8_plan, dims, &cache->cache, step, max_len, a, plan);
  if (s == TP_OK) s = prepare_tensors(dims, step, plan, q, softmax_scale, o, lse, workspace, ws_bytes, a);
  if (s != TP_OK) return s;
  OnDevice on((hipStream_t)stream);
  const hipError_t e = tp::launch_cache8_attention(a, fp8_of(cache), dims->head_dim, (hipStream_t)stream);
  if (e != hipSuccess) return hip_fail(e, "tp_cache8_attention launch");
  return ok();
}

tp_status tp_cache8_read(const tp_dims* dims, const tp_cache8* cache, const tp_batch* batch, const int64_t* first,
                         void* k_out, void* v_out, void* stream) {
  tp::CacheReadArgs a;
  tp_status s = check_format(cache);
  if (s == TP_OK) s = prepare_read(dims, &cache->cache, batch, first, k_out, v_out, a);
  if (s != TP_OK) return s;
  if (a.blocks == 0) return ok();
  OnDevice on((hipStream_t)stream);
  const hipError_t e = tp::launch_cache8_read(a, fp8_of(cache), dims->head_dim, (hipStream_t)stream);
  if (e != hipSuccess) return hip_fail(e, "tp_cache8_read launch");
  return ok();
}

}  // extern "C"

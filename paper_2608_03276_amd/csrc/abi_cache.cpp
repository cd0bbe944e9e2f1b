// C-ABI layer of the paged 4-bit cache: validation and dispatch.  Nothing is enqueued unless every
// host argument is valid; what lies on the device (lengths, page table, offsets, positions) is checked
// by the kernels, which leave out what is out of range.
#include "abi_cache.h"

namespace {

using tp::check_dims;
using tp::fail;
using tp::hip_fail;
using tp::ok;
using namespace tp::cache_abi;

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
  const tp_status s = prepare_load(dims, cache, kept_offsets, k, v_q, scales, a);
  if (s != TP_OK) return s;
  if (bits < 2 || bits > 8) return fail(TP_ERR_PARAM, "bits %d outside [2, 8]", bits);
  if (bits > 4) return fail(TP_ERR_UNSUPPORTED, "the pages hold codes of at most 4 bits (got %d)", bits);
  if (a.blocks == 0) return ok();
  OnDevice on((hipStream_t)stream);
  const hipError_t e = tp::launch_cache_load(a, dims->head_dim, (hipStream_t)stream);
  if (e != hipSuccess) return hip_fail(e, "tp_cache_load launch");
  return ok();
}

tp_status tp_cache_append(const tp_dims* dims, const tp_cache* cache, const tp_step* step, const tp_rows* k,
                          const tp_rows* v, const int32_t* positions, const tp_rope* rope, const tp_rows* q,
                          const tp_rows* q_out, void* stream) {
  tp::CacheWriteArgs a;
  const tp_status s = prepare_append(dims, cache, step, k, v, positions, rope, q, q_out, a);
  if (s != TP_OK) return s;
  OnDevice on((hipStream_t)stream);
  const hipError_t e = tp::launch_cache_append(a, dims->head_dim, (hipStream_t)stream);
  if (e != hipSuccess) return hip_fail(e, "tp_cache_append launch");
  return ok();
}

tp_status tp_cache_workspace_size(const tp_dims* dims, const tp_cache* cache, const tp_step* step, int64_t max_len,
                                  size_t* bytes) {
  if (!bytes) return fail(TP_ERR_NULL, "bytes is NULL");
  tp::CacheAttnArgs a;
  tp::CachePlan plan;
  const tp_status s = prepare_attention(tp::cache_plan, dims, cache, step, max_len, a, plan);
  if (s != TP_OK) return s;
  *bytes = plan.total;
  return ok();
}

tp_status tp_cache_attention(const tp_dims* dims, const tp_cache* cache, const tp_step* step, const tp_rows* q,
                             float softmax_scale, int64_t max_len, const tp_rows* o, float* lse, void* workspace,
                             size_t ws_bytes, void* stream) {
  tp::CacheAttnArgs a;
  tp::CachePlan plan;
  tp_status s = prepare_attention(tp::cache_plan, dims, cache, step, max_len, a, plan);
  if (s == TP_OK) s = prepare_tensors(dims, step, plan, q, softmax_scale, o, lse, workspace, ws_bytes, a);
  if (s != TP_OK) return s;
  OnDevice on((hipStream_t)stream);
  const hipError_t e = tp::launch_cache_attention(a, dims->head_dim, (hipStream_t)stream);
  if (e != hipSuccess) return hip_fail(e, "tp_cache_attention launch");
  return ok();
}

tp_status tp_cache_read(const tp_dims* dims, const tp_cache* cache, const tp_batch* batch, const int64_t* first,
                        void* k_out, void* v_out, void* stream) {
  tp::CacheReadArgs a;
  const tp_status s = prepare_read(dims, cache, batch, first, k_out, v_out, a);
  if (s != TP_OK) return s;
  if (a.blocks == 0) return ok();
  OnDevice on((hipStream_t)stream);
  const hipError_t e = tp::launch_cache_read(a, dims->head_dim, (hipStream_t)stream);
  if (e != hipSuccess) return hip_fail(e, "tp_cache_read launch");
  return ok();
}

}  // extern "C"

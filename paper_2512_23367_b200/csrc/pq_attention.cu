// Attention of a step's tokens over the paged key/value cache.  See include/pq.h for the contract.
#include <cuda_fp16.h>

#include <algorithm>
#include <cmath>

#include "pq_attention.h"

using namespace pq;

extern "C" {

int pq_paged_attention(const void* q_f16, int64_t q_stride, int32_t heads, const pq_kv_cache* cache,
                       const int32_t* block_table, int64_t width, const int32_t* q_start, const int32_t* kv_len,
                       int64_t requests, int64_t tokens, int64_t max_q, int64_t max_kv, float scale, int32_t window,
                       void* out_f16, void* workspace, size_t workspace_bytes, void* stream) {
  int rc = check_kv_cache(cache);
  if (rc != PQ_OK) return rc;
  if (heads < 1 || heads % cache->heads != 0 || heads / cache->heads > kMostGroup) return PQ_ERR_SHAPE;
  if (requests < 0 || requests > 0x7fffffff || tokens < 0 || tokens > 0x7fffffff) return PQ_ERR_SHAPE;
  if (width < 1 || width > 0x7fffffff || max_q < 0 || max_kv < 0 || window < 0 || !std::isfinite(scale)) return PQ_ERR_SHAPE;
  if (q_stride < static_cast<int64_t>(heads) * cache->dim || q_stride % 8 != 0) return PQ_ERR_SHAPE;
  if (requests > PQ_MAX_REQUESTS) return PQ_ERR_LIMIT;
  if (requests == 0 || tokens == 0) return PQ_OK;
  if (!q_f16 || !block_table || !q_start || !kv_len || !out_f16) return PQ_ERR_NULL;
  if (!aligned16(q_f16) || !aligned16(out_f16) || !aligned256(workspace)) return PQ_ERR_ALIGN;
  if ((rc = check_arch()) != PQ_OK) return rc;
  // Up to 16 rows per request and key/value head go to the row kernel, more to the tile kernel; which of them a request
  // takes is decided on the device.  A single request of many rows needs no row kernel, nor do groups of more than 16
  // heads, where a single token is more rows than it serves.
  const int group = heads / cache->heads;
  // No request has more rows than the step, nor keys beyond its table: larger bounds say no more.
  max_q = std::min(max_q, tokens);
  max_kv = bounded_keys(std::min(max_kv, width * cache->page));
  const bool wide = max_q * group > kAttnRows, narrow = group <= kAttnRows && (!wide || requests > 1);
  AttnArgs a{static_cast<const __half*>(q_f16), q_stride, *cache, block_table, width, q_start, kv_len,
             static_cast<__half*>(out_f16), tokens, static_cast<int>(requests), heads, window,
             narrow ? kAttnRows / group : 0, scale * 1.44269504f, 0, nullptr, nullptr};
  const Scratch sc = scratch_from(workspace, workspace_bytes);
  a.counters = sc.counters;
  a.partials = reinterpret_cast<float*>(sc.partials);
  cudaStream_t st = static_cast<cudaStream_t>(stream);
  if (narrow) {
    const AttnPlan plan = plan_attn_rows(requests, max_q, max_kv, window, cache->heads, cache->dim, cache->type == PQ_KV_INT8,
                                         sm_count(), sc.partial_bytes);
    a.part_keys = plan.part_keys;
    rc = launch_attn_rows(a, plan, max_q, st);
    if (rc != PQ_OK) return rc;
  }
  if (!wide) return PQ_OK;
  const TilePlan tile = plan_attn_tile(requests, tokens, max_q, max_kv, window, group, cache->heads, cache->dim,
                                       sm_count(), sc.partial_bytes);
  return launch_attn_tile(a, tile, st);
}

size_t pq_attention_workspace_bytes(int64_t requests, int64_t tokens, int64_t max_q, int64_t max_kv, int32_t heads,
                                    int32_t kv_heads, int32_t dim, int32_t sms) {
  return pq_attention_workspace_bytes_window(requests, tokens, max_q, max_kv, heads, kv_heads, dim, sms, 0);
}

size_t pq_attention_workspace_bytes_window(int64_t requests, int64_t tokens, int64_t max_q, int64_t max_kv, int32_t heads,
                                           int32_t kv_heads, int32_t dim, int32_t sms, int32_t window) {
  if (requests < 1 || requests > PQ_MAX_REQUESTS || tokens < 1 || tokens > 0x7fffffff || max_q < 1 || max_kv < 1 || kv_heads < 1 ||
      kv_heads > kMostKvHeads || heads < kv_heads || heads % kv_heads != 0 || heads / kv_heads > kMostGroup || (dim != 64 && dim != 128) || sms < 1 || window < 0) {
    return 0;
  }
  max_q = std::min(max_q, tokens);
  max_kv = bounded_keys(max_kv);
  size_t bytes = 0;   // for either type of cache
  const int group = heads / kv_heads;
  for (int int8 = 0; int8 < 2 && group <= kAttnRows; ++int8) {
    const AttnPlan plan = plan_attn_rows(requests, max_q, max_kv, window, kv_heads, dim, int8 != 0, sms, ~size_t(0));
    bytes = bytes > plan.partial_bytes ? bytes : plan.partial_bytes;
  }
  if (max_q * group > kAttnRows) {
    const TilePlan tile = plan_attn_tile(requests, tokens, max_q, max_kv, window, group, kv_heads, dim, sms, ~size_t(0));
    bytes = bytes > tile.partial_bytes ? bytes : tile.partial_bytes;   // the two kernels follow each other
  }
  return bytes > 0 ? kScratchHeaderBytes + bytes : 0;
}

}  // extern "C"

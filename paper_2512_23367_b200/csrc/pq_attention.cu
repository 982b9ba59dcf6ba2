// Attention of a step's tokens over the paged key/value cache.  See include/pq.h for the contract.
#include <cuda_fp16.h>

#include <cmath>

#include "pq_attention.h"
#include "pq_ptx.cuh"

namespace pq {

namespace {

// One warp per (row, head); a lane holds dim / 32 values of the query and of the sum; keys one after the other
// with a running maximum and sum.
template <bool kInt8, int D>
__global__ void __launch_bounds__(128) attention_kernel(const AttnArgs a) {
  constexpr int E = D / 32;
  grid_dep_launch();
  grid_dep_wait();
  const int lane = threadIdx.x & 31;
  const int64_t unit = static_cast<int64_t>(blockIdx.x) * 4 + (threadIdx.x >> 5);
  const int64_t t = unit / a.heads;
  const int h = static_cast<int>(unit - t * a.heads);
  if (t >= a.tokens || a.requests < 1 || t < a.q_start[0] || t >= a.q_start[a.requests]) return;
  int lo = 0, hi = a.requests - 1;
  while (lo < hi) {
    const int mid = (lo + hi + 1) >> 1;
    if (a.q_start[mid] <= t) lo = mid; else hi = mid - 1;
  }
  const int q0 = a.q_start[lo], n = a.q_start[lo + 1] - q0, L = a.kv_len[lo];
  if (static_cast<int64_t>(n) * (a.heads / a.c.heads) <= kAttnRows) return;   // the row kernel's
  const int64_t p = static_cast<int64_t>(L) - n + (t - q0);
  const int64_t end = min(p + 1, a.width * a.c.page);
  const int64_t begin = a.window > 0 ? max(static_cast<int64_t>(0), p + 1 - a.window) : 0;
  const int hk = h / (a.heads / a.c.heads);
  float q[E], o[E];
#pragma unroll
  for (int e = 0; e < E; ++e) q[e] = __half2float(a.q[t * a.q_stride + h * D + lane * E + e]) * a.scale_log2, o[e] = 0.0f;
  float m = -INFINITY, l = 0.0f;
  for (int64_t j = begin; j < end; ++j) {
    const int id = a.table[lo * a.width + j / a.c.page];
    const bool there = id >= 0 && id < a.c.pages;
    const int64_t vec = there ? (static_cast<int64_t>(id) * a.c.heads + hk) * a.c.page + j % a.c.page : 0;
    float k[E], v[E];
    float ks = there ? 1.0f : 0.0f, vs = ks;
    if constexpr (kInt8) {
      ks *= a.c.k_scale[vec];
      vs *= a.c.v_scale[vec];
#pragma unroll
      for (int e = 0; e < E; ++e) {
        k[e] = static_cast<const int8_t*>(a.c.k)[vec * D + lane * E + e];
        v[e] = static_cast<const int8_t*>(a.c.v)[vec * D + lane * E + e];
      }
    } else {
#pragma unroll
      for (int e = 0; e < E; ++e) {
        k[e] = __half2float(static_cast<const __half*>(a.c.k)[vec * D + lane * E + e]);
        v[e] = __half2float(static_cast<const __half*>(a.c.v)[vec * D + lane * E + e]);
      }
    }
    float s = 0.0f;
#pragma unroll
    for (int e = 0; e < E; ++e) s = fmaf(q[e], k[e], s);
#pragma unroll
    for (int d = 16; d > 0; d >>= 1) s += __shfl_xor_sync(0xffffffffu, s, d);
    s = there ? s * ks : 0.0f;
    const float mn = fmaxf(m, s);
    const float f = exp2f(m - mn), w = exp2f(s - mn);
    l = fmaf(l, f, w);
#pragma unroll
    for (int e = 0; e < E; ++e) o[e] = fmaf(o[e], f, there ? w * vs * v[e] : 0.0f);
    m = mn;
  }
#pragma unroll
  for (int e = 0; e < E; ++e) a.out[(t * a.heads + h) * D + lane * E + e] = __float2half_rn(l > 0.0f ? o[e] / l : 0.0f);
}

}  // namespace
}  // namespace pq

using namespace pq;

extern "C" {

int pq_paged_attention(const void* q_f16, int64_t q_stride, int32_t heads, const pq_kv_cache* cache,
                       const int32_t* block_table, int64_t width, const int32_t* q_start, const int32_t* kv_len,
                       int64_t requests, int64_t tokens, int64_t max_q, int64_t max_kv, float scale, int32_t window,
                       void* out_f16, void* workspace, size_t workspace_bytes, void* stream) {
  int rc = check_kv_cache(cache);
  if (rc != PQ_OK) return rc;
  if (heads < 1 || heads % cache->heads != 0 || heads / cache->heads > 64) return PQ_ERR_SHAPE;
  if (requests < 0 || requests > 0x7fffffff || tokens < 0 || tokens > 0x7fffffff) return PQ_ERR_SHAPE;
  if (width < 1 || width > 0x7fffffff || max_q < 0 || max_kv < 0 || window < 0 || !std::isfinite(scale)) return PQ_ERR_SHAPE;
  if (q_stride < static_cast<int64_t>(heads) * cache->dim || q_stride % 8 != 0) return PQ_ERR_SHAPE;
  if (requests > PQ_MAX_REQUESTS) return PQ_ERR_LIMIT;
  if (requests == 0 || tokens == 0) return PQ_OK;
  if (!q_f16 || !block_table || !q_start || !kv_len || !out_f16) return PQ_ERR_NULL;
  if (!aligned16(q_f16) || !aligned16(out_f16) || !aligned256(workspace)) return PQ_ERR_ALIGN;
  if ((rc = check_arch()) != PQ_OK) return rc;
  AttnArgs a{static_cast<const __half*>(q_f16), q_stride, *cache, block_table, width, q_start, kv_len,
             static_cast<__half*>(out_f16), tokens, static_cast<int>(requests), heads, window, scale * 1.44269504f,
             0, nullptr, nullptr};
  const Scratch sc = scratch_from(workspace, workspace_bytes);
  const AttnPlan plan = plan_attn_rows(requests, max_kv, cache->heads, cache->dim, sm_count(), sc.partial_bytes);
  a.part_keys = plan.part_keys;
  a.counters = sc.counters;
  a.partials = reinterpret_cast<float*>(sc.partials);
  rc = launch_attn_rows(a, plan, static_cast<cudaStream_t>(stream));
  if (rc != PQ_OK || max_q * (heads / cache->heads) <= kAttnRows) return rc;
  if (cache->type == PQ_KV_F16) {
    const TilePlan tile = plan_attn_tile(requests, tokens, max_q, max_kv, heads / cache->heads, cache->heads, cache->dim,
                                         sm_count(), sc.partial_bytes);
    return launch_attn_tile(a, tile, static_cast<cudaStream_t>(stream));
  }
  const int64_t blocks = (tokens * heads + 3) / 4;
  if (blocks > 0x7fffffff) return PQ_ERR_SHAPE;
  const dim3 grid(static_cast<unsigned>(blocks)), block(128);
  cudaStream_t st = static_cast<cudaStream_t>(stream);
  if (cache->type == PQ_KV_INT8) {
    return cache->dim == 128 ? launch_dependent(attention_kernel<true, 128>, grid, block, 0, st, a)
                             : launch_dependent(attention_kernel<true, 64>, grid, block, 0, st, a);
  }
  return cache->dim == 128 ? launch_dependent(attention_kernel<false, 128>, grid, block, 0, st, a)
                           : launch_dependent(attention_kernel<false, 64>, grid, block, 0, st, a);
}

size_t pq_attention_workspace_bytes(int64_t requests, int64_t tokens, int64_t max_q, int64_t max_kv, int32_t heads,
                                    int32_t kv_heads, int32_t dim, int32_t sms) {
  if (requests < 1 || requests > PQ_MAX_REQUESTS || tokens < 1 || max_q < 1 || max_kv < 1 || kv_heads < 1 ||
      heads < kv_heads || heads % kv_heads != 0 || (dim != 64 && dim != 128) || sms < 1) {
    return 0;
  }
  const AttnPlan plan = plan_attn_rows(requests, max_kv, kv_heads, dim, sms, ~size_t(0));
  size_t bytes = plan.partial_bytes;
  if (max_q * (heads / kv_heads) > kAttnRows) {
    const TilePlan tile = plan_attn_tile(requests, tokens, max_q, max_kv, heads / kv_heads, kv_heads, dim, sms, ~size_t(0));
    bytes = bytes > tile.partial_bytes ? bytes : tile.partial_bytes;   // the two kernels follow each other
  }
  return bytes > 0 ? kScratchHeaderBytes + bytes : 0;
}

}  // extern "C"

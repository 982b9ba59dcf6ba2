// Paged key/value cache: block tables and slot map of a step, the write of the step's keys and values, and their
// read-back.  See include/pq.h for the contract of every call.
#include <cuda_fp16.h>

#include <type_traits>

#include "pq_internal.h"
#include "pq_ptx.cuh"
#include "pq_quant_math.cuh"

namespace pq {

int check_kv_cache(const pq_kv_cache* c) {
  if (c == nullptr || c->k == nullptr || c->v == nullptr) return PQ_ERR_NULL;
  if (c->type != PQ_KV_F16 && c->type != PQ_KV_INT8) return PQ_ERR_SHAPE;
  if (c->type == PQ_KV_INT8 && (c->k_scale == nullptr || c->v_scale == nullptr)) return PQ_ERR_NULL;
  if (c->dim != 64 && c->dim != 128) return PQ_ERR_SHAPE;
  if (c->page < 16 || c->page > 1024 || c->page % 16 != 0) return PQ_ERR_SHAPE;
  if (c->heads < 1 || c->heads > kMostKvHeads || c->pages < 1 || c->pages > 0x7fffffff) return PQ_ERR_SHAPE;
  if (c->pages * c->heads * c->page > 0x7fffffff) return PQ_ERR_SHAPE;
  if (!aligned16(c->k) || !aligned16(c->v)) return PQ_ERR_ALIGN;
  if (c->type == PQ_KV_INT8 && (!aligned16(c->k_scale) || !aligned16(c->v_scale))) return PQ_ERR_ALIGN;
  return PQ_OK;
}

namespace {

constexpr int kThreads = 256;

// ---------------------------------------------------------------------------------------- block tables
struct TableArgs {
  const int* kv_len;
  const int* new_len;
  int* table;
  const int* free_list;
  const int* free_head;
  int* q_start;
  int* kv_total;
  int64_t* slots;
  int* pos;
  int* free_next;
  int64_t width, free_count;
  int requests, page, tokens;
};

// Every CTA scans the requests' lengths by itself (two exclusive sums held in shared memory: rows and fresh
// pages) and then serves its share of the rows: the request of a row by bisection over the row sums, its page
// from the table (pages that were there) or straight from the free list (fresh ones), so that no CTA waits for
// another's table entries.  The row that begins a fresh page enters it in the table.
// Latency bound: one read of 8 B per request, one dependent read per row, 12 B written per row.
__global__ void __launch_bounds__(kThreads) block_tables_kernel(const TableArgs a) {
  __shared__ int s_row[PQ_MAX_REQUESTS + 1];
  __shared__ int s_page[PQ_MAX_REQUESTS + 1];
  __shared__ int s_sum[2][kThreads / 32];
  grid_dep_launch();
  grid_dep_wait();
  const int tid = threadIdx.x, lane = tid & 31, warp = tid >> 5;
  const int per = (a.requests + kThreads - 1) / kThreads;   // requests of one thread, consecutive
  const int b0 = min(tid * per, a.requests), b1 = min(b0 + per, a.requests);
  const int head = *a.free_head;

  int rows = 0, fresh = 0;
  for (int b = b0; b < b1; ++b) {
    const int kv = max(a.kv_len[b], 0), n = max(a.new_len[b], 0);
    s_row[b] = rows;       // sums inside the thread's own run; the offset of the run is added below
    s_page[b] = fresh;
    rows += n;
    fresh += (kv + n + a.page - 1) / a.page - (kv + a.page - 1) / a.page;
    if (blockIdx.x == 0) a.kv_total[b] = kv + n;
  }
  int row_in = rows, page_in = fresh;
#pragma unroll
  for (int o = 1; o < 32; o <<= 1) {
    const int r = __shfl_up_sync(0xffffffffu, row_in, o), p = __shfl_up_sync(0xffffffffu, page_in, o);
    if (lane >= o) row_in += r, page_in += p;
  }
  if (lane == 31) s_sum[0][warp] = row_in, s_sum[1][warp] = page_in;
  __syncthreads();
  int row_off = row_in - rows, page_off = page_in - fresh, row_all = 0, page_all = 0;
#pragma unroll
  for (int w = 0; w < kThreads / 32; ++w) {
    if (w < warp) row_off += s_sum[0][w], page_off += s_sum[1][w];
    row_all += s_sum[0][w], page_all += s_sum[1][w];
  }
  for (int b = b0; b < b1; ++b) {
    s_row[b] += row_off;
    s_page[b] += page_off;
    if (blockIdx.x == 0) a.q_start[b] = s_row[b];
  }
  if (tid == 0) {
    s_row[a.requests] = row_all;
    if (blockIdx.x == 0) {
      a.q_start[a.requests] = row_all;
      *a.free_next = head + page_all;
    }
  }
  __syncthreads();

  for (int64_t t = static_cast<int64_t>(blockIdx.x) * kThreads + tid; t < a.tokens; t += static_cast<int64_t>(gridDim.x) * kThreads) {
    if (t >= row_all) {
      a.slots[t] = -1;
      a.pos[t] = -1;
      continue;
    }
    int lo = 0, hi = a.requests - 1;   // the last request whose first row is <= t (empty requests before it share that row)
    while (lo < hi) {
      const int mid = (lo + hi + 1) >> 1;
      if (s_row[mid] <= t) lo = mid; else hi = mid - 1;
    }
    const int kv = max(a.kv_len[lo], 0);
    const int pos = kv + static_cast<int>(t) - s_row[lo];
    const int col = pos / a.page, off = pos - col * a.page;
    const int have = (kv + a.page - 1) / a.page;
    int id = -1;
    if (pos >= 0 && col < a.width) {
      int* entry = a.table + static_cast<int64_t>(lo) * a.width + col;
      if (col < have) {
        id = *entry;
      } else {
        const int64_t take = static_cast<int64_t>(head) + s_page[lo] + (col - have);
        if (take >= 0 && take < a.free_count) id = a.free_list[take];
        if (off == 0) *entry = id;
      }
    }
    a.slots[t] = id < 0 ? -1 : static_cast<int64_t>(id) * a.page + off;
    a.pos[t] = pos;
  }
}

// ---------------------------------------------------------------------------------------- append, read
struct RowArgs {
  pq_kv_cache c;
  const void* k;
  const void* v;
  int64_t k_stride, v_stride;
  const int64_t* slots;
  int64_t tokens;
  void* k_out;
  void* v_out;
  int rows_per_block;   // tokens that a block of kThreads serves side by side
};

// Element offset of (slot, head) in the cache's value arrays, in units of one vector; -1 for a slot outside it.
__device__ __forceinline__ int64_t vector_of(const pq_kv_cache& c, int64_t slot, int head) {
  if (slot < 0 || slot >= c.pages * c.page) return -1;
  const uint32_t s = static_cast<uint32_t>(slot);   // pages * page < 2^31
  const uint32_t id = s / static_cast<uint32_t>(c.page), off = s - id * c.page;
  return (static_cast<int64_t>(id) * c.heads + head) * c.page + off;
}

// A thread owns one 16-byte chunk (8 values) of a token's key and of its value, of kTokens tokens; all its loads are in
// flight together, the slots' among them.  The 8 or 16 threads of a vector are neighbours in a warp.
//   kInt8: the vector's maximum by lane exchanges inside those 8 or 16 threads, then the codes of Eq. 1-2.
// HBM bound beyond a few hundred tokens, latency below (64 tokens, 8 heads of 128: 1.7 us FP16, 2.0 INT8).
template <bool kInt8, int D, int kTokens>
__global__ void __launch_bounds__(kThreads) kv_append_kernel(const RowArgs a) {
  constexpr int kChunks = D / 8;   // threads per vector
  grid_dep_launch();
  grid_dep_wait();
  const int chunks = a.c.heads * kChunks;
  const int sub = threadIdx.x / chunks;
  const int first = threadIdx.x - sub * chunks;
  if (sub >= a.rows_per_block) return;   // whole vectors leave together
  const int64_t t0 = static_cast<int64_t>(blockIdx.x) * (a.rows_per_block * kTokens) + sub;
  const int step = a.rows_per_block > 1 ? chunks : kThreads;
  for (int c = first; c < chunks; c += step) {
    uint4 k[kTokens], v[kTokens];
    int64_t vec[kTokens];
#pragma unroll
    for (int i = 0; i < kTokens; ++i) {
      const int64_t t = t0 + i * a.rows_per_block;
      vec[i] = -1;
      if (t < a.tokens) {
        k[i] = __ldg(reinterpret_cast<const uint4*>(static_cast<const __half*>(a.k) + t * a.k_stride) + c);
        v[i] = __ldg(reinterpret_cast<const uint4*>(static_cast<const __half*>(a.v) + t * a.v_stride) + c);
        vec[i] = a.slots[t];
      }
    }
    const int head = c / kChunks, part = c % kChunks;
#pragma unroll
    for (int i = 0; i < kTokens; ++i) {
      vec[i] = vector_of(a.c, vec[i], head);
      if (vec[i] < 0) continue;            // the same for all threads of a vector
      if constexpr (!kInt8) {
        reinterpret_cast<uint4*>(a.c.k)[vec[i] * kChunks + part] = k[i];
        reinterpret_cast<uint4*>(a.c.v)[vec[i] * kChunks + part] = v[i];
      } else {
        const uint32_t lane = threadIdx.x & 31;
        const uint32_t mask = (kChunks == 16 ? 0xffffu : 0xffu) << (lane & ~(kChunks - 1));
        float ka = absmax8(k[i]), va = absmax8(v[i]);
#pragma unroll
        for (int o = kChunks / 2; o > 0; o >>= 1) {
          ka = fmaxf(ka, __shfl_xor_sync(mask, ka, o));
          va = fmaxf(va, __shfl_xor_sync(mask, va, o));
        }
        float ks, kf, vs, vf;
        act_scale(ka, &ks, &kf);
        act_scale(va, &vs, &vf);
        const __half* kh = reinterpret_cast<const __half*>(&k[i]);
        const __half* vh = reinterpret_cast<const __half*>(&v[i]);
        float x[8], y[8];
#pragma unroll
        for (int j = 0; j < 8; ++j) x[j] = __half2float(kh[j]), y[j] = __half2float(vh[j]);
        reinterpret_cast<uint2*>(a.c.k)[vec[i] * kChunks + part] =
            make_uint2(codes4<false>(x[0], x[1], x[2], x[3], kf), codes4<false>(x[4], x[5], x[6], x[7], kf));
        reinterpret_cast<uint2*>(a.c.v)[vec[i] * kChunks + part] =
            make_uint2(codes4<false>(y[0], y[1], y[2], y[3], vf), codes4<false>(y[4], y[5], y[6], y[7], vf));
        if (part == 0) {
          a.c.k_scale[vec[i]] = ks;
          a.c.v_scale[vec[i]] = vs;
        }
      }
    }
  }
}

__device__ __forceinline__ uint4 values_of(const uint2& codes, float s) {
  const int8_t* c = reinterpret_cast<const int8_t*>(&codes);
  uint4 out;
  __half2* h = reinterpret_cast<__half2*>(&out);
#pragma unroll
  for (int i = 0; i < 4; ++i)
    h[i] = __floats2half2_rn(__fmul_rn(static_cast<float>(c[2 * i]), s), __fmul_rn(static_cast<float>(c[2 * i + 1]), s));
  return out;
}

template <bool kInt8, int D, int kTokens>
__global__ void __launch_bounds__(kThreads) kv_read_kernel(const RowArgs a) {
  constexpr int kChunks = D / 8;
  using Piece = std::conditional_t<kInt8, uint2, uint4>;   // 8 values as they lie in the cache
  grid_dep_launch();
  grid_dep_wait();
  const int chunks = a.c.heads * kChunks;
  const int sub = threadIdx.x / chunks;
  const int first = threadIdx.x - sub * chunks;
  if (sub >= a.rows_per_block) return;
  const int64_t t0 = static_cast<int64_t>(blockIdx.x) * (a.rows_per_block * kTokens) + sub;
  const int step = a.rows_per_block > 1 ? chunks : kThreads;
  for (int c = first; c < chunks; c += step) {
    const int head = c / kChunks, part = c % kChunks;
    Piece k[kTokens] = {}, v[kTokens] = {};
    float ks[kTokens] = {}, vs[kTokens] = {};
#pragma unroll
    for (int i = 0; i < kTokens; ++i) {
      const int64_t t = t0 + i * a.rows_per_block;
      const int64_t vec = t < a.tokens ? vector_of(a.c, a.slots[t], head) : -1;
      if (vec >= 0) {
        k[i] = static_cast<const Piece*>(a.c.k)[vec * kChunks + part];
        v[i] = static_cast<const Piece*>(a.c.v)[vec * kChunks + part];
        if constexpr (kInt8) ks[i] = a.c.k_scale[vec], vs[i] = a.c.v_scale[vec];
      }
    }
#pragma unroll
    for (int i = 0; i < kTokens; ++i) {
      const int64_t t = t0 + i * a.rows_per_block;
      if (t >= a.tokens) continue;
      if constexpr (kInt8) {
        static_cast<uint4*>(a.k_out)[t * chunks + c] = values_of(k[i], ks[i]);
        static_cast<uint4*>(a.v_out)[t * chunks + c] = values_of(v[i], vs[i]);
      } else {
        static_cast<uint4*>(a.k_out)[t * chunks + c] = k[i];
        static_cast<uint4*>(a.v_out)[t * chunks + c] = v[i];
      }
    }
  }
}

// Tokens side by side in a block; a token wider than a block is walked by all its threads.
int rows_per_block(int chunks) { return chunks >= kThreads ? 1 : kThreads / chunks; }

// Two tokens per thread where the grid still fills the machine a few times over (32768 tokens, 8 heads of 128, INT8:
// append 46.9 us with one, 41.4 with two, 44.3 with four; read 47.4, 34.5, 38.3).
constexpr int kManyTokens = 2;
template <bool kAppend, bool kInt8, int D>
int launch_rows(const RowArgs& a, cudaStream_t stream) {
  const int64_t blocks = (a.tokens + a.rows_per_block - 1) / a.rows_per_block;
  const bool many = blocks >= static_cast<int64_t>(kManyTokens) * 8 * sm_count();
  const unsigned grid = static_cast<unsigned>(many ? (blocks + kManyTokens - 1) / kManyTokens : blocks);
  if constexpr (kAppend) {
    return launch_dependent(many ? kv_append_kernel<kInt8, D, kManyTokens> : kv_append_kernel<kInt8, D, 1>, dim3(grid), dim3(kThreads), 0, stream, a);
  } else {
    return launch_dependent(many ? kv_read_kernel<kInt8, D, kManyTokens> : kv_read_kernel<kInt8, D, 1>, dim3(grid), dim3(kThreads), 0, stream, a);
  }
}
template <bool kAppend>
int launch_rows(const RowArgs& a, cudaStream_t stream) {
  if (a.c.type == PQ_KV_INT8) return a.c.dim == 128 ? launch_rows<kAppend, true, 128>(a, stream) : launch_rows<kAppend, true, 64>(a, stream);
  return a.c.dim == 128 ? launch_rows<kAppend, false, 128>(a, stream) : launch_rows<kAppend, false, 64>(a, stream);
}

}  // namespace
}  // namespace pq

using namespace pq;

extern "C" {

int pq_block_tables(const int32_t* kv_len, const int32_t* new_len, int64_t requests, int32_t* block_table,
                    int64_t width, const int32_t* free_list, int64_t free_count, const int32_t* free_head,
                    int32_t page, int64_t tokens, int32_t* q_start, int32_t* kv_total, int64_t* slots,
                    int32_t* pos, int32_t* free_next, void* stream) {
  if (requests < 0 || tokens < 0 || tokens > 0x7fffffff || width < 1 || width > 0x7fffffff || free_count < 0) return PQ_ERR_SHAPE;
  if (page < 16 || page > 1024 || page % 16 != 0) return PQ_ERR_SHAPE;
  if (requests > PQ_MAX_REQUESTS) return PQ_ERR_LIMIT;
  if (!free_head || !q_start || !free_next || (!free_list && free_count > 0)) return PQ_ERR_NULL;
  if (requests > 0 && (!kv_len || !new_len || !block_table || !kv_total)) return PQ_ERR_NULL;
  if (tokens > 0 && (!slots || !pos)) return PQ_ERR_NULL;
  if (free_next == free_head || (requests > 0 && kv_total == kv_len)) return PQ_ERR_SHAPE;
  const int rc = check_arch();
  if (rc != PQ_OK) return rc;
  const TableArgs a{kv_len, new_len, block_table, free_list, free_head, q_start, kv_total, slots, pos, free_next,
                    width, free_count, static_cast<int>(requests), page, static_cast<int>(tokens)};
  const int64_t want = (tokens + kThreads - 1) / kThreads, most = sm_count();
  const unsigned grid = static_cast<unsigned>(want < 1 ? 1 : (want < most ? want : most));
  return launch_dependent(block_tables_kernel, dim3(grid), dim3(kThreads), 0, static_cast<cudaStream_t>(stream), a);
}

int pq_kv_append(const pq_kv_cache* cache, const void* k_f16, int64_t k_stride, const void* v_f16, int64_t v_stride,
                 const int64_t* slots, int64_t tokens, void* stream) {
  int rc = check_kv_cache(cache);
  if (rc != PQ_OK) return rc;
  const int64_t row = static_cast<int64_t>(cache->heads) * cache->dim;
  if (tokens < 0 || tokens > 0x7fffffff || k_stride < row || v_stride < row || k_stride % 8 != 0 || v_stride % 8 != 0) return PQ_ERR_SHAPE;
  if (tokens == 0) return PQ_OK;
  if (!k_f16 || !v_f16 || !slots) return PQ_ERR_NULL;
  if (!aligned16(k_f16) || !aligned16(v_f16)) return PQ_ERR_ALIGN;
  if ((rc = check_arch()) != PQ_OK) return rc;
  const int per = rows_per_block(static_cast<int>(row / 8));
  const RowArgs a{*cache, k_f16, v_f16, k_stride, v_stride, slots, tokens, nullptr, nullptr, per};
  return launch_rows<true>(a, static_cast<cudaStream_t>(stream));
}

int pq_kv_read(const pq_kv_cache* cache, const int64_t* slots, int64_t tokens, void* k_f16, void* v_f16, void* stream) {
  int rc = check_kv_cache(cache);
  if (rc != PQ_OK) return rc;
  if (tokens < 0 || tokens > 0x7fffffff) return PQ_ERR_SHAPE;
  if (tokens == 0) return PQ_OK;
  if (!k_f16 || !v_f16 || !slots) return PQ_ERR_NULL;
  if (!aligned16(k_f16) || !aligned16(v_f16)) return PQ_ERR_ALIGN;
  if ((rc = check_arch()) != PQ_OK) return rc;
  const int per = rows_per_block(cache->heads * cache->dim / 8);
  const RowArgs a{*cache, nullptr, nullptr, 0, 0, slots, tokens, k_f16, v_f16, per};
  return launch_rows<false>(a, static_cast<cudaStream_t>(stream));
}

}  // extern "C"

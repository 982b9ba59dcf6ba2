// Rotary positions: queries and keys turned pair by pair by an angle proportional to the token's position, by themselves
// and on the way into a paged cache.  See include/pq.h for the contract of every call.
#include <cuda_fp16.h>

#include <cmath>

#include "pq_internal.h"
#include "pq_ptx.cuh"
#include "pq_quant_math.cuh"

namespace pq {

int check_latent_cache(const pq_latent_cache* c) {
  if (c == nullptr || c->data == nullptr) return PQ_ERR_NULL;
  if (c->latent != 256 && c->latent != 512) return PQ_ERR_SHAPE;
  if (c->page < 16 || c->page > 1024 || c->page % 16 != 0) return PQ_ERR_SHAPE;
  if (c->pages < 1 || c->pages > 0x7fffffff || c->pages * c->page > 0x7fffffff) return PQ_ERR_SHAPE;
  return aligned16(c->data) ? PQ_OK : PQ_ERR_ALIGN;
}

namespace {

constexpr int kThreads = 256;
constexpr int kItem = 16;   // values of one work item: two 16-byte chunks, 8 pairs

enum Target { kRotate, kKvF16, kKvInt8, kLatent };

// n / d for n below 2^20 and d up to 2^20: n * ceil(2^40 / d) exceeds n / d * 2^40 by less than n <= 2^20, less than the 2^40 / d that
// the next whole number is away.
struct Divisor {
  uint32_t d;
  uint64_t mul;
  Divisor() = default;
  explicit Divisor(int by) : d(by), mul(((uint64_t(1) << 40) + by - 1) / by) {}
  __device__ __forceinline__ int divide(int n) const { return static_cast<int>(static_cast<uint64_t>(n) * mul >> 40); }
};

// Rows of one operand: head h of token t at p + t * stride + h * head_stride.
struct Rows {
  const __half* p;
  int64_t stride, head_stride;
  int heads;
  int items;   // of a head: its values / 16
  Divisor by_items;
};

struct TurnArgs {
  pq_rotary r;
  const int* pos;
  const int64_t* slots;
  int64_t tokens;
  int per_token;    // items of a token: queries', keys', values'
  Divisor by_token;
  int turned;       // of a head: its first dim / 16 items are turned (0: none)
  Rows q, k, v;     // kLatent: k the rotary key, v the latent vector
  __half* out;      // of the queries
  int64_t out_stride, out_head_stride;
  pq_kv_cache kv;
  pq_latent_cache latent;
};

__device__ __forceinline__ void unpack8(const uint4& v, float* x) {
  const __half2* h = reinterpret_cast<const __half2*>(&v);
#pragma unroll
  for (int i = 0; i < 4; ++i) {
    const float2 f = __half22float2(h[i]);
    x[2 * i] = f.x, x[2 * i + 1] = f.y;
  }
}
__device__ __forceinline__ uint4 pack8(const float* x) {
  uint4 v;
  __half2* h = reinterpret_cast<__half2*>(&v);
#pragma unroll
  for (int i = 0; i < 4; ++i) h[i] = __floats2half2_rn(x[2 * i], x[2 * i + 1]);
  return v;
}

// One thread serves kItems items of 16 values: 8 pairs, whose two sides are chunks i and i + dim / 16 (kHalf) or neighbours
// inside the chunks 2i and 2i + 1; behind the turned part of a head, and for values, two neighbouring chunks.  A block's
// items lie one after the other in (token, operand, head, item) order, so that neighbours share lines.
//
// The angle of pair i at position p is p * freq[i] turns, an integer product modulo 2^64: exact modulo a turn at
// every 32-bit position, where FP32 radians would be off by 2^-24 p.  A block's cosines and sines are computed once per
// (token, pair) into shared memory, for all heads; in FP32, as the products are.  FP16 results are rounded once; an INT8 key is
// quantized from its FP32 values, so that it is rounded once, too.
//
// HBM bound beyond a few hundred tokens, latency below: 8192 tokens of 40 heads of 128, half of each turned, 27 us in a row (6.2 TB/s)
// and 31 alone; one token 1.5 and 3.7.  8192 tokens of 32 query and 8 key/value heads into an FP16 cache 34 and 38.5, where the bytes take 31.
// Into an INT8 cache 38.5 and 44 (44 and 49 with one item per thread), where they take 28: quantization makes it nearest to instructions,
// 75 % of the issue slots, while memory is at 43 %; a warp that does not issue waits for its loads, for the block's cosines or for a fixed latency.
// Five blocks an SM, 48 registers, of which the kernels with two items spill a few: with four and 64 registers the calls for 8192 tokens
// took 2 to 4 us more, with six 1 to 8.
template <Target kTarget, bool kHalf, int kItems>
__global__ void __launch_bounds__(kThreads, 5) rotary_kernel(const TurnArgs a) {
  extern __shared__ float s_cos[];
  grid_dep_launch();
  const int tid = threadIdx.x;
  const int64_t base = static_cast<int64_t>(blockIdx.x) * (kThreads * kItems);
  const int64_t tok0 = base / a.per_token;
  const int lead = static_cast<int>(base - tok0 * a.per_token);   // items of token tok0 that are an earlier block's
  const int pairs = a.r.dim / 2;
  const int toks = static_cast<int>(min(a.tokens - tok0, static_cast<int64_t>((lead + kThreads * kItems - 1) / a.per_token + 1)));
  float* s_sin = s_cos + toks * pairs;
  grid_dep_wait();

  // every load that depends on nothing else first
  uint4 lo[kItems], hi[kItems];
  int tok[kItems], head[kItems], item[kItems], part[kItems];
#pragma unroll
  for (int u = 0; u < kItems; ++u) {
    const int flat = lead + tid + u * kThreads;
    tok[u] = a.by_token.divide(flat);
    int rest = flat - tok[u] * a.per_token;
    part[u] = tok[u] >= toks ? -1 : 0;
    Rows r = a.q;
    if (kTarget != kRotate && rest >= a.q.heads * a.q.items) {
      rest -= a.q.heads * a.q.items;
      r = a.k, part[u] = tok[u] >= toks ? -1 : 1;
      if (rest >= a.k.heads * a.k.items) {
        rest -= a.k.heads * a.k.items;
        r = a.v, part[u] = tok[u] >= toks ? -1 : 2;
      }
    }
    head[u] = r.by_items.divide(rest), item[u] = rest - head[u] * r.items;
    lo[u] = hi[u] = make_uint4(0, 0, 0, 0);
    if (part[u] >= 0) {
      const uint4* p = reinterpret_cast<const uint4*>(r.p + (tok0 + tok[u]) * r.stride + head[u] * r.head_stride);
      const bool apart = kHalf && part[u] != 2 && item[u] < a.turned;
      lo[u] = p[apart ? item[u] : 2 * item[u]];
      hi[u] = p[apart ? item[u] + a.turned : 2 * item[u] + 1];
    }
  }
  for (int i = tid; i < toks * pairs; i += kThreads) {
    const int t = i / pairs, j = i - t * pairs;
    const uint64_t turn = static_cast<uint64_t>(static_cast<int64_t>(a.pos[tok0 + t])) * a.r.freq[j];
    float s, c;
    sincospif(__ll2float_rn(static_cast<int64_t>(turn)) * 0x1p-63f, &s, &c);   // in half turns, within [-1, 1]
    s_cos[i] = c * a.r.amplitude;
    s_sin[i] = s * a.r.amplitude;
  }
  __syncthreads();

#pragma unroll
  for (int u = 0; u < kItems; ++u) {
    if (part[u] < 0) continue;   // whole heads leave together
    const bool turn = part[u] != 2 && item[u] < a.turned;
    const bool apart = kHalf && turn;
    float x[kItem];
    if (turn || (kTarget == kKvInt8 && part[u] > 0)) unpack8(lo[u], x), unpack8(hi[u], x + 8);
    if (turn) {
      float c[8], s[8];
      const float4* cp = reinterpret_cast<const float4*>(s_cos + tok[u] * pairs) + 2 * item[u];
      const float4* sp = reinterpret_cast<const float4*>(s_sin + tok[u] * pairs) + 2 * item[u];
      *reinterpret_cast<float4*>(c) = cp[0], *reinterpret_cast<float4*>(c + 4) = cp[1];
      *reinterpret_cast<float4*>(s) = sp[0], *reinterpret_cast<float4*>(s + 4) = sp[1];
#pragma unroll
      for (int j = 0; j < 8; ++j) {
        float& p = x[kHalf ? j : 2 * j];
        float& q = x[kHalf ? j + 8 : 2 * j + 1];
        const float e = fmaf(p, c[j], -(q * s[j])), f = fmaf(q, c[j], p * s[j]);
        p = e, q = f;
      }
    }
    if (part[u] == 0) {
      uint4* p = reinterpret_cast<uint4*>(a.out + (tok0 + tok[u]) * a.out_stride + head[u] * a.out_head_stride);
      p[apart ? item[u] : 2 * item[u]] = turn ? pack8(x) : lo[u];
      p[apart ? item[u] + a.turned : 2 * item[u] + 1] = turn ? pack8(x + 8) : hi[u];
      continue;
    }
    if constexpr (kTarget == kLatent) {
      const int64_t slot = a.slots[tok0 + tok[u]];
      if (slot < 0 || slot >= a.latent.pages * a.latent.page) continue;
      uint4* p = reinterpret_cast<uint4*>(static_cast<__half*>(a.latent.data) + slot * (a.latent.latent + PQ_LATENT_ROPE) +
                                          (part[u] == 1 ? a.latent.latent : 0));
      p[apart ? item[u] : 2 * item[u]] = turn ? pack8(x) : lo[u];
      p[apart ? item[u] + a.turned : 2 * item[u] + 1] = turn ? pack8(x + 8) : hi[u];
    } else if constexpr (kTarget != kRotate) {
      const int64_t slot = a.slots[tok0 + tok[u]];
      if (slot < 0 || slot >= a.kv.pages * a.kv.page) continue;   // the same for all threads of a vector
      const uint32_t s = static_cast<uint32_t>(slot), id = s / static_cast<uint32_t>(a.kv.page);   // pages * page < 2^31
      const int64_t vec = (static_cast<int64_t>(id) * a.kv.heads + head[u]) * a.kv.page + (s - id * a.kv.page);
      void* to = part[u] == 1 ? a.kv.k : a.kv.v;
      const int c0 = apart ? item[u] : 2 * item[u], c1 = apart ? item[u] + a.turned : 2 * item[u] + 1;
      if constexpr (kTarget == kKvF16) {
        uint4* p = static_cast<uint4*>(to) + vec * (a.kv.dim / 8);
        p[c0] = turn ? pack8(x) : lo[u];
        p[c1] = turn ? pack8(x + 8) : hi[u];
      } else {   // the maximum over the vector's 4 or 8 threads, then the codes of Eq. 1-2
        const int lanes = a.kv.dim / kItem;
        const uint32_t mask = ((1u << lanes) - 1u) << ((tid & 31) & ~(lanes - 1));
        float top = 0.0f;
#pragma unroll
        for (int j = 0; j < kItem; ++j) top = fmaxf(top, fabsf(x[j]));
        for (int o = lanes / 2; o > 0; o >>= 1) top = fmaxf(top, __shfl_xor_sync(mask, top, o));
        float scale, f;
        act_scale(top, &scale, &f);
        uint2* p = static_cast<uint2*>(to) + vec * (a.kv.dim / 8);
        p[c0] = make_uint2(codes4<false>(x[0], x[1], x[2], x[3], f), codes4<false>(x[4], x[5], x[6], x[7], f));
        p[c1] = make_uint2(codes4<false>(x[8], x[9], x[10], x[11], f), codes4<false>(x[12], x[13], x[14], x[15], f));
        if (item[u] == 0) (part[u] == 1 ? a.kv.k_scale : a.kv.v_scale)[vec] = scale;
      }
    }
  }
}

// Two items per thread where the grid still fills the machine several times over.
constexpr int kManyItems = 2;
template <Target kTarget, bool kHalf>
int launch_items(TurnArgs a, cudaStream_t stream) {
  a.by_token = Divisor(a.per_token);
  const int64_t items = a.tokens * a.per_token;
  const bool many = items >= static_cast<int64_t>(kThreads) * kManyItems * 8 * sm_count();
  const int64_t block = kThreads * (many ? kManyItems : 1), grid = (items + block - 1) / block;
  if (grid > 0x7fffffff) return PQ_ERR_LIMIT;
  // Tokens that a block's items may belong to, and their cosines and sines: at most 2 (dim / 2) per 16 values of `dim`.
  const int64_t toks = (block + a.per_token - 2) / a.per_token + 1;
  const size_t smem = static_cast<size_t>(toks < a.tokens ? toks : a.tokens) * a.r.dim * sizeof(float);
  return many ? launch_dependent(rotary_kernel<kTarget, kHalf, kManyItems>, dim3(static_cast<unsigned>(grid)), dim3(kThreads), smem, stream, a)
              : launch_dependent(rotary_kernel<kTarget, kHalf, 1>, dim3(static_cast<unsigned>(grid)), dim3(kThreads), smem, stream, a);
}
template <Target kTarget>
int launch_turn(const TurnArgs& a, cudaStream_t stream) {
  return a.r.layout == PQ_ROTARY_HALF ? launch_items<kTarget, true>(a, stream) : launch_items<kTarget, false>(a, stream);
}

// The rules for a rotation of heads of `width` values.
int check_rotary(const pq_rotary* r, int width) {
  if (r == nullptr || r->freq == nullptr) return PQ_ERR_NULL;
  if (r->layout != PQ_ROTARY_HALF && r->layout != PQ_ROTARY_PAIRS) return PQ_ERR_SHAPE;
  if (r->dim < 16 || r->dim > 256 || r->dim % 16 != 0 || r->dim > width) return PQ_ERR_SHAPE;
  if (!(r->amplitude >= 0x1p-16f && r->amplitude <= 0x1p16f)) return PQ_ERR_SHAPE;
  return (reinterpret_cast<uintptr_t>(r->freq) & 7u) == 0 ? PQ_OK : PQ_ERR_ALIGN;
}
// Rows of heads that can be read and written in 16-byte chunks.
bool strides_ok(int64_t stride, int64_t head_stride, int heads, int width) {
  if (stride % 8 != 0 || stride < 0) return false;
  return heads == 1 || (head_stride % 8 == 0 && head_stride >= width);
}

struct QueryRows {   // the optional queries of an append
  const void* q;
  int64_t stride, head_stride;
  int heads;
  void* out;
  int64_t out_stride, out_head_stride;
};
int set_queries(TurnArgs& a, const QueryRows& q, int width) {
  if (q.heads < 0 || q.heads > 1024) return PQ_ERR_SHAPE;
  a.q = Rows{static_cast<const __half*>(q.q), q.stride, q.head_stride, q.heads, width / kItem, Divisor(width / kItem)};
  a.out = static_cast<__half*>(q.out), a.out_stride = q.out_stride, a.out_head_stride = q.out_head_stride;
  if (q.heads == 0) return PQ_OK;
  if (!strides_ok(q.stride, q.head_stride, q.heads, width) || !strides_ok(q.out_stride, q.out_head_stride, q.heads, width)) return PQ_ERR_SHAPE;
  if (a.tokens > 1 && q.out_stride < width) return PQ_ERR_SHAPE;   // rows on top of each other
  if (a.tokens > 0 && (!q.q || !q.out)) return PQ_ERR_NULL;
  return aligned16(q.q) && aligned16(q.out) ? PQ_OK : PQ_ERR_ALIGN;
}

// Copies latent vectors and rotary keys out of the cache: 16-byte chunks, a thread each.
struct ReadArgs {
  pq_latent_cache c;
  const int64_t* slots;
  int64_t tokens;
  uint4* latent;
  uint4* rope;
};
__global__ void __launch_bounds__(kThreads) latent_read_kernel(const ReadArgs a) {
  grid_dep_launch();
  grid_dep_wait();
  const int wide = a.c.latent / 8, chunks = wide + PQ_LATENT_ROPE / 8;
  const int64_t i = static_cast<int64_t>(blockIdx.x) * kThreads + threadIdx.x;
  const int64_t t = i / chunks;
  const int c = static_cast<int>(i - t * chunks);
  if (t >= a.tokens) return;
  const int64_t slot = a.slots[t];
  uint4 v = make_uint4(0, 0, 0, 0);
  if (slot >= 0 && slot < a.c.pages * a.c.page) v = static_cast<const uint4*>(a.c.data)[slot * chunks + c];
  if (c < wide) a.latent[t * wide + c] = v; else a.rope[t * (PQ_LATENT_ROPE / 8) + (c - wide)] = v;
}

}  // namespace
}  // namespace pq

using namespace pq;

extern "C" {

int pq_rotary_frequencies(int32_t dim, double base, int32_t scaling, double factor, double original, double low, double high,
                          uint64_t* freq, float* amplitude) {
  if (dim < 16 || dim > 256 || dim % 16 != 0 || !(base > 1.0) || !std::isfinite(base)) return PQ_ERR_SHAPE;
  if (scaling < PQ_ROTARY_PLAIN || scaling > PQ_ROTARY_WAVES) return PQ_ERR_SHAPE;
  if (scaling != PQ_ROTARY_PLAIN && !(factor >= 1.0 && factor <= 1e6)) return PQ_ERR_SHAPE;
  const bool ranged = scaling == PQ_ROTARY_BANDS || scaling == PQ_ROTARY_WAVES;
  if (ranged && !(original >= 1.0 && original <= 2147483648.0 && low > 0.0 && high > low && high <= 1e9)) return PQ_ERR_SHAPE;
  if (!freq || !amplitude) return PQ_ERR_NULL;
  const double two_pi = 6.283185307179586476925286766559, d = dim;
  if (scaling == PQ_ROTARY_BASE) base *= std::pow(factor, d / (d - 2.0));
  // bands: pairs that make more than `high` turns over the original length keep their frequency, below `low` they are stretched
  auto pair_of = [&](double turns) { return d * std::log(original / (turns * two_pi)) / (2.0 * std::log(base)); };
  double first = 0.0, last = 0.0;
  if (scaling == PQ_ROTARY_BANDS) {
    first = std::fmax(std::floor(pair_of(high)), 0.0);
    last = std::fmin(std::ceil(pair_of(low)), d - 1.0);
  }
  for (int i = 0; i < dim / 2; ++i) {
    double f = std::pow(base, -2.0 * i / d), stretched = 0.0;   // radians per position; share of the stretched frequency
    if (scaling == PQ_ROTARY_LINEAR) stretched = 1.0;
    if (scaling == PQ_ROTARY_BANDS) stretched = (i - first) / std::fmax(last - first, 0.001);
    if (scaling == PQ_ROTARY_WAVES) stretched = 1.0 - (original * f / two_pi - low) / (high - low);
    stretched = std::fmin(std::fmax(stretched, 0.0), 1.0);
    f = f / (scaling == PQ_ROTARY_PLAIN ? 1.0 : factor) * stretched + f * (1.0 - stretched);
    freq[i] = static_cast<uint64_t>(std::llrint(f / two_pi * 0x1p62)) << 2;   // f <= 1: below 2^60 before the shift
  }
  *amplitude = scaling == PQ_ROTARY_BANDS ? static_cast<float>(0.1 * std::log(factor) + 1.0) : 1.0f;
  return PQ_OK;
}

int pq_rotate(const pq_rotary* rotary, const void* x_f16, int64_t x_stride, int64_t x_head_stride, int32_t heads, int32_t width,
              const int32_t* pos, int64_t tokens, void* out_f16, int64_t out_stride, int64_t out_head_stride, void* stream) {
  if (width < 16 || width > 1024 || width % 16 != 0 || heads < 1 || heads > 1024 || tokens < 0 || tokens > 0x7fffffff) return PQ_ERR_SHAPE;
  int rc = check_rotary(rotary, width);
  if (rc != PQ_OK) return rc;
  TurnArgs a = {};
  a.r = *rotary, a.pos = pos, a.tokens = tokens, a.turned = rotary->dim / kItem;
  if ((rc = set_queries(a, {x_f16, x_stride, x_head_stride, heads, out_f16, out_stride, out_head_stride}, width)) != PQ_OK) return rc;
  if (tokens == 0) return PQ_OK;
  if (!pos) return PQ_ERR_NULL;
  if ((rc = check_arch()) != PQ_OK) return rc;
  a.per_token = heads * a.q.items;
  return launch_turn<kRotate>(a, static_cast<cudaStream_t>(stream));
}

int pq_kv_append_rotated(const pq_kv_cache* cache, const pq_rotary* rotary, const void* k_f16, int64_t k_stride, const void* v_f16,
                         int64_t v_stride, const int64_t* slots, const int32_t* pos, int64_t tokens, const void* q_f16,
                         int64_t q_stride, int64_t q_head_stride, int32_t q_heads, void* out_f16, int64_t out_stride,
                         int64_t out_head_stride, void* stream) {
  int rc = check_kv_cache(cache);
  if (rc != PQ_OK || (rc = check_rotary(rotary, cache->dim)) != PQ_OK) return rc;
  const int64_t row = static_cast<int64_t>(cache->heads) * cache->dim;
  if (tokens < 0 || tokens > 0x7fffffff || k_stride < row || v_stride < row || k_stride % 8 != 0 || v_stride % 8 != 0) return PQ_ERR_SHAPE;
  TurnArgs a = {};
  a.r = *rotary, a.pos = pos, a.slots = slots, a.tokens = tokens, a.turned = rotary->dim / kItem, a.kv = *cache;
  if ((rc = set_queries(a, {q_f16, q_stride, q_head_stride, q_heads, out_f16, out_stride, out_head_stride}, cache->dim)) != PQ_OK) return rc;
  if (tokens == 0) return PQ_OK;
  if (!k_f16 || !v_f16 || !slots || !pos) return PQ_ERR_NULL;
  if (!aligned16(k_f16) || !aligned16(v_f16)) return PQ_ERR_ALIGN;
  if ((rc = check_arch()) != PQ_OK) return rc;
  const int items = cache->dim / kItem;
  a.k = Rows{static_cast<const __half*>(k_f16), k_stride, cache->dim, cache->heads, items, Divisor(items)};
  a.v = Rows{static_cast<const __half*>(v_f16), v_stride, cache->dim, cache->heads, items, Divisor(items)};
  a.per_token = (q_heads + 2 * cache->heads) * items;
  return cache->type == PQ_KV_INT8 ? launch_turn<kKvInt8>(a, static_cast<cudaStream_t>(stream))
                                   : launch_turn<kKvF16>(a, static_cast<cudaStream_t>(stream));
}

int pq_latent_append(const pq_latent_cache* cache, const pq_rotary* rotary, const void* c_f16, int64_t c_stride,
                     const void* k_rope_f16, int64_t k_rope_stride, const int64_t* slots, const int32_t* pos, int64_t tokens,
                     const void* q_f16, int64_t q_stride, int64_t q_head_stride, int32_t q_heads, void* out_f16,
                     int64_t out_stride, int64_t out_head_stride, void* stream) {
  int rc = check_latent_cache(cache);
  if (rc != PQ_OK || (rc = check_rotary(rotary, PQ_LATENT_ROPE)) != PQ_OK) return rc;
  if (tokens < 0 || tokens > 0x7fffffff || c_stride < cache->latent || k_rope_stride < PQ_LATENT_ROPE || c_stride % 8 != 0 || k_rope_stride % 8 != 0) return PQ_ERR_SHAPE;
  TurnArgs a = {};
  a.r = *rotary, a.pos = pos, a.slots = slots, a.tokens = tokens, a.turned = rotary->dim / kItem, a.latent = *cache;
  if ((rc = set_queries(a, {q_f16, q_stride, q_head_stride, q_heads, out_f16, out_stride, out_head_stride}, PQ_LATENT_ROPE)) != PQ_OK) return rc;
  if (tokens == 0) return PQ_OK;
  if (!c_f16 || !k_rope_f16 || !slots || !pos) return PQ_ERR_NULL;
  if (!aligned16(c_f16) || !aligned16(k_rope_f16)) return PQ_ERR_ALIGN;
  if ((rc = check_arch()) != PQ_OK) return rc;
  a.k = Rows{static_cast<const __half*>(k_rope_f16), k_rope_stride, PQ_LATENT_ROPE, 1, PQ_LATENT_ROPE / kItem, Divisor(PQ_LATENT_ROPE / kItem)};
  a.v = Rows{static_cast<const __half*>(c_f16), c_stride, cache->latent, 1, cache->latent / kItem, Divisor(cache->latent / kItem)};
  a.per_token = q_heads * a.q.items + a.k.items + a.v.items;
  return launch_turn<kLatent>(a, static_cast<cudaStream_t>(stream));
}

int pq_latent_read(const pq_latent_cache* cache, const int64_t* slots, int64_t tokens, void* c_f16, void* k_rope_f16, void* stream) {
  int rc = check_latent_cache(cache);
  if (rc != PQ_OK) return rc;
  if (tokens < 0 || tokens > 0x7fffffff) return PQ_ERR_SHAPE;
  if (tokens == 0) return PQ_OK;
  if (!slots || !c_f16 || !k_rope_f16) return PQ_ERR_NULL;
  if (!aligned16(c_f16) || !aligned16(k_rope_f16)) return PQ_ERR_ALIGN;
  if ((rc = check_arch()) != PQ_OK) return rc;
  const int64_t grid = (tokens * ((cache->latent + PQ_LATENT_ROPE) / 8) + kThreads - 1) / kThreads;
  if (grid > 0x7fffffff) return PQ_ERR_LIMIT;
  const ReadArgs a{*cache, slots, tokens, static_cast<uint4*>(c_f16), static_cast<uint4*>(k_rope_f16)};
  return launch_dependent(latent_read_kernel, dim3(static_cast<unsigned>(grid)), dim3(kThreads), 0, static_cast<cudaStream_t>(stream), a);
}

}  // extern "C"

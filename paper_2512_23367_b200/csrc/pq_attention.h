// What the attention kernels share: arguments, the split of the keys over CTAs and the joining of the parts.
#pragma once
#include <cuda_fp16.h>

#include <cstdint>

#include "pq_internal.h"

namespace pq {

struct AttnArgs {
  const __half* q;
  int64_t q_stride;
  pq_kv_cache c;
  const int* table;
  int64_t width;
  const int* q_start;
  const int* kv_len;
  __half* out;
  int64_t tokens;
  int requests, heads, window;
  int row_tokens;            // requests of up to so many tokens are the row kernel's (0: it is not launched)
  float scale_log2;          // scale * log2(e): scores are powers of two
  int part_keys;             // keys of one part, a multiple of 128
  unsigned int* counters;    // row kernel: arrivals per unit, zero between calls
  float* partials;           // per unit and part: rows x dim sums, then rows x (maximum, sum)
};

// Rows of a (request, key/value head) that the row kernel takes: two 8-wide tiles of the warp's matrix instruction.
// Requests with more rows go to the tile kernel.
constexpr int kAttnRows = 16;

constexpr int kMostGroup = 64;   // query heads of one key/value head

// Lengths are 32 bits wide, and the schedules round up to parts of 128 keys in 32 bits: 2^30 keys are as good as more
// (the last part of a unit takes the keys that are left).
constexpr int64_t kMostKeys = int64_t(1) << 30;
inline int64_t bounded_keys(int64_t max_kv) { return max_kv < kMostKeys ? max_kv : kMostKeys; }

// Schedule of a call, from sizes that the host knows: how many parts a unit's keys may be cut into.
struct AttnPlan {
  int64_t units = 0;      // units of the row kernel: requests x key/value heads
  int parts = 1;          // grid parts per unit
  int part_keys = 128;
  size_t partial_bytes = 0;
};
AttnPlan plan_attn_rows(int64_t requests, int64_t max_q, int64_t max_kv, int window, int kv_heads, int dim, bool int8, int sms, size_t room);

int launch_attn_rows(const AttnArgs& a, const AttnPlan& plan, int64_t max_q, cudaStream_t stream);

// The tile kernel's schedule: a unit is one tile of 2 x (128 / group) tokens of one key/value head.
struct TilePlan {
  int64_t whole = 0;      // units that one CTA serves whole
  int64_t split = 0;      // units after those, whose keys are cut into up to `parts` parts; both are upper bounds
  int parts = 1;
  int part_keys = 128;
  size_t partial_bytes = 0;
};
TilePlan plan_attn_tile(int64_t requests, int64_t tokens, int64_t max_q, int64_t max_kv, int window, int group, int kv_heads,
                        int dim, int sms, size_t room);
int launch_attn_tile(const AttnArgs& a, const TilePlan& plan, cudaStream_t stream);

__device__ __forceinline__ float exp2_approx(float x) {
  float y;
  asm("ex2.approx.ftz.f32 %0, %1;" : "=f"(y) : "f"(x));
  return y;
}

__device__ __forceinline__ float log2_approx(float x) {
  float y;
  asm("lg2.approx.ftz.f32 %0, %1;" : "=f"(y) : "f"(x));
  return y;
}

__device__ __forceinline__ uint32_t pack_f16(float a, float b) {
  const __half2 h = __floats2half2_rn(a, b);
  return *reinterpret_cast<const uint32_t*>(&h);
}
// Four INT8 codes, offset by 128 (bytes u = code + 128), as FP16: 0x6400 | u is 1024 + u, and 1024 + u - 1152 is the
// code, exactly.  sel picks the two bytes.
__device__ __forceinline__ uint32_t codes_f16(uint32_t u, uint32_t sel) {
  const uint32_t h = __byte_perm(u, 0x64646464u, sel);
  const __half2 r = __hsub2(*reinterpret_cast<const __half2*>(&h), __half2(__ushort_as_half(0x6480), __ushort_as_half(0x6480)));
  return *reinterpret_cast<const uint32_t*>(&r);
}
__device__ __forceinline__ float power_of_two(int e) { return __uint_as_float(static_cast<uint32_t>(127 + e) << 23); }   // |e| <= 126
// The exponent of an INT8 value scale, within [-40, 60]: scales of FP16 values lie in [2^-31, 2^10), and with a range of
// 100 no weight that counts leaves FP32's on the way to its sum, nor does a sum of them.
__device__ __forceinline__ int scale_exponent(float v) { return min(max(static_cast<int>(__float_as_uint(v) << 1 >> 24) - 127, -40), 60); }
__device__ __forceinline__ float scale_log(float v) { return fminf(fmaxf(log2_approx(v), -40.0f), 60.0f); }   // within the same range
// The smallest power of two >= v, within the same range: the unit that a run of INT8 value scales is taken in.
__device__ __forceinline__ float scale_unit(float v) {
  return __uint_as_float((__float_as_uint(fminf(fmaxf(v, 0x1p-40f), 0x1p60f)) + 0x7fffffu) & 0x7f800000u);
}

// First key that a row at position p sees.  In 64 bits: p may be negative (a row before its request's first key) and
// the window up to 2^31 - 1.
__device__ __forceinline__ int first_key(int p, int window) {
  const int64_t first = static_cast<int64_t>(p) + 1 - window;
  return window > 0 && first > 0 ? static_cast<int>(first) : 0;
}

// Keys [lo, hi) that a request's rows may see: lo from the window of its first row, hi from its length and its table.
struct AttnRange {
  int n, L, lo, hi;
};
__device__ __forceinline__ AttnRange attn_range(const AttnArgs& a, int rows, int cached) {
  AttnRange r;
  r.n = rows;
  r.L = max(cached, 0);   // positions from -n on stay within 32 bits
  const int64_t cap = a.width * a.c.page;
  r.hi = static_cast<int>(min(static_cast<int64_t>(r.L), cap));
  r.lo = first_key(r.L - r.n, a.window);
  return r;
}

}  // namespace pq

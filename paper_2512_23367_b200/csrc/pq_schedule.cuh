// The schedule of the latent attention kernels: how one CTA per SM finds its share of a step's work on the device, from
// the requests' lengths.
//
// A UNIT is a tile of a request's query rows (for one head, where heads have keys of their own) with the STEPS of keys that
// its last row sees.  Two ways to hand units out:
//   shares   the steps of all units, in order, are cut into runs of one length, one per CTA, so that every SM takes the same
//            share whatever the lengths are.  A share may begin and end inside a unit: that unit's parts are joined later.
//   turns    whole units, a request's last tile, which sees most keys, first: CTA c of n takes the units c, 2n - 1 - c, 2n + c, ...,
//            there and back again, so that who has the largest of one turn has the smallest of the next (512 units of a prompt of
//            4096: the longest CTA has 3 % more than its share; with c, n + c, 2n + c, ... it had 26).
#pragma once
#include <cstdint>

#include "pq_attention.h"
#include "pq_attn_mma.cuh"
#include "pq_ptx.cuh"

namespace pq {

// sum over 0 <= i < n of floor((a i + b) / m), by the Euclidean algorithm.
__device__ inline uint64_t floor_sum(uint64_t n, uint64_t m, uint64_t a, uint64_t b) {
  uint64_t sum = 0;
  while (n > 0) {
    if (a >= m) sum += (n - 1) * n / 2 * (a / m), a %= m;
    if (b >= m) sum += n * (b / m), b %= m;
    const uint64_t top = a * n + b;
    if (top < m) break;
    n = top / m, b = top % m;
    const uint64_t x = a;
    a = m, m = x;
  }
  return sum;
}

constexpr int kFewSteps = 6;   // of a unit at most: shares are not worth their joining

struct UnitShape {
  int rows;      // query rows of a tile
  int heads;     // rows per token: row r of a request is of token r / heads
  int keys;      // keys of a step
  int copies;    // units per tile
};

struct Request {
  int q0, n;              // first token, tokens (n * heads, and units over all requests, below 2^31)
  int k0, L, hi;          // first key (where keys are ragged rows), keys, keys that can be read
  UnitShape s;
  uint32_t all;           // rows: below 2^31
  int tiles;
  int same;               // > 0: steps of every unit (fewer keys than rows, or than the table holds)
  __device__ __forceinline__ void settle() {
    all = static_cast<uint32_t>(n) * static_cast<uint32_t>(s.heads);
    tiles = static_cast<int>((all + s.rows - 1) / static_cast<uint32_t>(s.rows));
    same = L < n || hi < L ? max((hi + s.keys - 1) / s.keys, 1) : 0;
  }
  __device__ __forceinline__ int units() const { return tiles * s.copies; }
  __device__ __forceinline__ int steps(int tile) const {
    if (same) return same;
    const uint32_t last = min(static_cast<uint32_t>(tile + 1) * s.rows, all) - 1;
    return (L - n + static_cast<int>(last / static_cast<uint32_t>(s.heads))) / s.keys + 1;
  }
  __device__ __forceinline__ int64_t before_tile(int tile) const {   // steps of one copy of the tiles before; tile < tiles
    if (same) return static_cast<int64_t>(same) * tile;
    if (tile == 0) return 0;
    return static_cast<int64_t>(floor_sum(tile, static_cast<uint64_t>(s.keys) * s.heads, s.rows, s.rows - 1 + static_cast<uint64_t>(L - n) * s.heads)) + tile;
  }
  __device__ __forceinline__ int64_t before(int unit) const {        // unit < units()
    const int tile = unit / s.copies, copy = unit - tile * s.copies;
    return before_tile(tile) * s.copies + static_cast<int64_t>(copy) * (copy ? steps(tile) : 0);
  }
  __device__ __forceinline__ int64_t total() const { return tiles == 0 ? 0 : (before_tile(tiles - 1) + steps(tiles - 1)) * s.copies; }
};

// Shares: `left` steps from step `step` of unit `unit` of request `b` on.
struct Share {
  int b, unit, step, per;
  int64_t left;
};

// By the whole block; sums: one word per warp.
template <int kThreads, class Args>
__device__ __forceinline__ void find_share(const Args& a, int worker, int workers, int least, Share* share, int64_t* sums) {
  const int tid = threadIdx.x, lane = tid & 31, warp = tid >> 5;
  const int each = (a.requests + kThreads - 1) / kThreads;
  const int b0 = min(tid * each, a.requests), b1 = min(b0 + each, a.requests);
  int64_t mine = 0;
  for (int b = b0; b < b1; ++b) mine += a.request(b).total();
  int64_t in = mine;
#pragma unroll
  for (int o = 1; o < 32; o <<= 1) {
    const int64_t x = __shfl_up_sync(0xffffffffu, in, o);
    if (lane >= o) in += x;
  }
  if (lane == 31) sums[warp] = in;
  if (tid == 0) share->left = 0, share->b = a.requests, share->unit = 0, share->step = 0;
  __syncthreads();
  int64_t off = in - mine, all = 0;
#pragma unroll
  for (int w = 0; w < kThreads / 32; ++w) {
    if (w < warp) off += sums[w];
    all += sums[w];
  }
  int64_t per = (all + workers - 1) / workers;
  if (per < least) per = least;
  const int64_t first = per * worker;
  if (first < all && first >= off && first < off + mine) {
    int64_t at = first - off;
    for (int b = b0; b < b1; ++b) {
      const Request r = a.request(b);
      const int64_t t = r.total();
      if (at >= t) {
        at -= t;
        continue;
      }
      int lo = 0, hi = r.units() - 1;   // the last unit that begins at or before the step
      while (lo < hi) {
        const int mid = lo + (hi - lo + 1) / 2;
        if (r.before(mid) <= at) lo = mid; else hi = mid - 1;
      }
      share->b = b, share->unit = lo, share->step = static_cast<int>(at - r.before(lo));
      share->left = min(per, all - first);
      break;
    }
  }
  if (tid == 0) share->per = static_cast<int>(min(per, static_cast<int64_t>(0x7fffffff)));
  __syncthreads();
}

// Walks the units of one CTA, as every warp of it does for itself; all lanes together.  By turns, a lane keeps one of 32
// requests, so that going on to the next unit reads no memory (it took 3000 cycles between a unit's end and the next one's begin).
template <class Args>
struct Walk {
  const Args& a;
  const bool shares;
  int step_there, step_back;        // turns: to the next unit
  int b;                            // request
  int unit;                         // shares: as in Share; turns: counted from request `base`'s first
  int64_t left;                     // turns: 1 as long as there are any
  int step, count, all_steps;       // the unit's steps: first, how many, of all
  int tile, copy;
  Request r;
  Request mine;                     // turns: the lane's, base + lane
  int base, in;                     // units of the requests from base to the lane's, its own included
  __device__ __forceinline__ Walk(const Args& args, const Share& s, bool by_shares, int worker, int of)
      : a(args), shares(by_shares), step_there(2 * (of - 1 - worker) + 1), step_back(2 * worker + 1), b(by_shares ? s.b : -1), unit(by_shares ? s.unit : worker), left(by_shares ? s.left : 1),
        step(by_shares ? s.step : 0), base(0) {
    if (shares) {
      if (left > 0) r = a.request(b);
    } else {
      fetch();
    }
    find();
  }
  __device__ __forceinline__ bool more() const { return left > 0; }
  __device__ __forceinline__ bool whole() const { return count == all_steps; }
  __device__ __forceinline__ void next() {
    if (shares) {
      left -= count, ++unit;
    } else {
      const int x = step_there;
      unit += x, step_there = step_back, step_back = x;
    }
    step = 0;
    find();
  }
  __device__ __forceinline__ void fetch() {
    const int lane = threadIdx.x & 31;
    in = 0;
    if (base + lane < a.requests) mine = a.request(base + lane), in = mine.units();
#pragma unroll
    for (int o = 1; o < 32; o <<= 1) {
      const int x = __shfl_up_sync(0xffffffffu, in, o);
      if (lane >= o) in += x;
    }
  }
  __device__ __forceinline__ void find() {
    if (left <= 0) return;
    if (shares) {
      while (unit >= r.units()) {
        if (++b >= a.requests) {
          left = 0;
          return;
        }
        r = a.request(b), unit = 0;
      }
      return take(unit);
    }
    for (;;) {
      const uint32_t behind = __ballot_sync(0xffffffffu, in > unit);
      if (behind) {
        const int at = __ffs(behind) - 1;
        const int before = __shfl_sync(0xffffffffu, in, max(at - 1, 0));
        b = base + at;
        r.q0 = __shfl_sync(0xffffffffu, mine.q0, at), r.n = __shfl_sync(0xffffffffu, mine.n, at);
        r.k0 = __shfl_sync(0xffffffffu, mine.k0, at), r.L = __shfl_sync(0xffffffffu, mine.L, at), r.hi = __shfl_sync(0xffffffffu, mine.hi, at);
        r.s = a.shape();
        r.settle();
        return take(unit - (at > 0 ? before : 0));
      }
      unit -= __shfl_sync(0xffffffffu, in, 31);
      base += 32;
      if (base >= a.requests) break;
      fetch();
    }
    left = 0;
  }
  __device__ __forceinline__ void take(int of_request) {
    tile = of_request / r.s.copies, copy = of_request - tile * r.s.copies;
    if (!shares) tile = r.tiles - 1 - tile;
    all_steps = r.steps(tile);
    count = shares ? static_cast<int>(min(static_cast<int64_t>(all_steps - step), left)) : all_steps;
  }
};

// Joins the parts of a unit that was cut: a thread has 16 values of one row, lanes along the rows.  A part is [values / 4][kRows]
// x 4 sums, then [kRows] x (reference, sum of weights); part(i) is the i-th of `parts`, `first` the thread's first value, `to` where
// its row has them (nullptr: there is no such row).  All of four parts is loaded at once: L2 latency bounds it.
// kGroups > 1: so many threads of a block share a row's parts, in blocks of kGroups x kRows threads.  One request of 52000 tokens
// in 148 parts: 49 us with one group, 36 with four; 64 requests in two or three parts each, where four times the blocks
// come in waves: 141 and 155.
// many_parts: whether a unit may be in more than 16, from bounds of the units and of the steps of one.
inline bool many_parts(int64_t units, int workers, int64_t steps, int least) {
  return units * 16 < workers && steps > 16 * least;
}
template <int kRows, int kValues, int kGroups, class Part>
__device__ __forceinline__ void join_parts(const Part& part, int parts, int first, __half* to) {
  __shared__ float s_join[kGroups > 1 ? kGroups - 1 : 1][18][kGroups > 1 ? kRows : 1];
  const int row = threadIdx.x % kRows, group = kGroups > 1 ? threadIdx.x / kRows : 0;
  float M = -INFINITY, L = 0.0f;
  float v[16];
#pragma unroll
  for (int j = 0; j < 16; ++j) v[j] = 0.0f;
  constexpr int kBatch = 4;
  for (int i0 = group; to != nullptr && i0 < parts; i0 += kBatch * kGroups) {
    float2 ml[kBatch];
    float4 x[kBatch][4];
#pragma unroll
    for (int i = 0; i < kBatch; ++i) {
      ml[i] = make_float2(-INFINITY, 0.0f);
#pragma unroll
      for (int j = 0; j < 4; ++j) x[i][j] = make_float4(0.0f, 0.0f, 0.0f, 0.0f);
      if (i0 + i * kGroups >= parts) continue;
      const float* p = part(i0 + i * kGroups);
      ml[i] = __ldcg(reinterpret_cast<const float2*>(p + kRows * kValues) + row);
#pragma unroll
      for (int j = 0; j < 4; ++j) x[i][j] = __ldcg(reinterpret_cast<const float4*>(p) + (first / 4 + j) * kRows + row);
    }
    float top = M;
#pragma unroll
    for (int i = 0; i < kBatch; ++i) top = fmaxf(top, ml[i].x);
    const float ref = top == -INFINITY ? 0.0f : top, f = exp2_approx(M - ref);
    M = top;
    L *= f;
#pragma unroll
    for (int j = 0; j < 16; ++j) v[j] *= f;
#pragma unroll
    for (int i = 0; i < kBatch; ++i) {
      const float w = exp2_approx(ml[i].x - ref);   // 0 for a part that is not there, or whose row saw nothing
      L = fmaf(ml[i].y, w, L);
#pragma unroll
      for (int j = 0; j < 4; ++j) {
        v[4 * j] = fmaf(x[i][j].x, w, v[4 * j]), v[4 * j + 1] = fmaf(x[i][j].y, w, v[4 * j + 1]);
        v[4 * j + 2] = fmaf(x[i][j].z, w, v[4 * j + 2]), v[4 * j + 3] = fmaf(x[i][j].w, w, v[4 * j + 3]);
      }
    }
  }
  if constexpr (kGroups > 1) {
    if (group > 0 && group < parts) {
      float (*mine)[kRows] = s_join[group - 1];
      mine[0][row] = M, mine[1][row] = L;
#pragma unroll
      for (int j = 0; j < 16; ++j) mine[2 + j][row] = v[j];
    }
    __syncthreads();
    if (group > 0) return;
    for (int g = 1; g < min(parts, kGroups); ++g) {
      const float (*other)[kRows] = s_join[g - 1];
      const float m = other[0][row], top = fmaxf(M, m), ref = top == -INFINITY ? 0.0f : top;
      const float f = exp2_approx(M - ref), w = exp2_approx(m - ref);
      M = top, L = fmaf(other[1][row], w, L * f);
#pragma unroll
      for (int j = 0; j < 16; ++j) v[j] = fmaf(other[2 + j][row], w, v[j] * f);
    }
  }
  if (to == nullptr) return;
  const float inv = L > 0.0f ? 1.0f / L : 0.0f;
  uint32_t h[8];
#pragma unroll
  for (int j = 0; j < 8; ++j) h[j] = pack_f16(v[2 * j] * inv, v[2 * j + 1] * inv);
  store_32_bytes(to, h[0], h[1], h[2], h[3], h[4], h[5], h[6], h[7]);
}

}  // namespace pq

// The schedule of the latent attention kernels: how one CTA per SM finds its share of a step's work on the device, from
// the requests' lengths.
//
// A UNIT is a tile of a request's query rows (for one head, where heads have keys of their own) with the STEPS of keys that
// its last row sees.  Two ways to hand units out:
//   shares   the steps of all units, in order, are cut into runs of one length, one per CTA, so that every SM takes the same
//            share whatever the lengths are.  A share may begin and end inside a unit: that unit's parts are joined later.
//   turns    CTA c takes the units c, c + CTAs, ...: whole units, a request's last tile, which sees most keys, first.
#pragma once
#include <cstdint>

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

// Walks the units of one CTA, as every warp of it does for itself; all lanes together.
template <class Args>
struct Walk {
  const Args& a;
  const bool shares;
  const int workers;
  int b;
  int unit;                         // shares: as in Share; turns: counted from request b's first
  int64_t left;                     // turns: 1 as long as there are any
  int step, count, all_steps;       // the unit's steps: first, how many, of all
  int tile, copy;
  Request r;
  __device__ __forceinline__ Walk(const Args& args, const Share& s, bool by_shares, int worker, int of)
      : a(args), shares(by_shares), workers(of), b(by_shares ? s.b : 0), unit(by_shares ? s.unit : worker), left(by_shares ? s.left : 1),
        step(by_shares ? s.step : 0) {
    find();
  }
  __device__ __forceinline__ bool more() const { return left > 0; }
  __device__ __forceinline__ bool whole() const { return count == all_steps; }
  __device__ __forceinline__ void next() {
    if (shares) left -= count, ++unit; else unit += workers;
    step = 0;
    find();
  }
  __device__ __forceinline__ void find() {
    if (left <= 0) return;
    if (shares) {
      for (; b < a.requests; ++b, unit = 0) {
        r = a.request(b);
        if (unit < r.units()) return take();
      }
      left = 0;
      return;
    }
    const int lane = threadIdx.x & 31;
    for (; b < a.requests; b += 32) {   // 32 requests at a time
      int in = b + lane < a.requests ? a.request(b + lane).units() : 0;
#pragma unroll
      for (int o = 1; o < 32; o <<= 1) {
        const int x = __shfl_up_sync(0xffffffffu, in, o);
        if (lane >= o) in += x;
      }
      const uint32_t behind = __ballot_sync(0xffffffffu, in > unit);
      if (behind) {
        const int at = __ffs(behind) - 1;
        const int before = __shfl_sync(0xffffffffu, in, max(at - 1, 0));
        if (at > 0) unit -= before;
        b += at;
        r = a.request(b);
        return take();
      }
      unit -= __shfl_sync(0xffffffffu, in, 31);
    }
    left = 0;
  }
  __device__ __forceinline__ void take() {
    tile = unit / r.s.copies, copy = unit - tile * r.s.copies;
    if (!shares) tile = r.tiles - 1 - tile;
    all_steps = r.steps(tile);
    count = shares ? static_cast<int>(min(static_cast<int64_t>(all_steps - step), left)) : all_steps;
  }
};

}  // namespace pq

// The schedule of the latent attention kernels: how one CTA per SM finds its share of a step's work on the device, from
// the requests' lengths.
//
// A UNIT is a tile of a request's query rows (for one head, where heads have keys of their own) with the STEPS of keys that
// its last row sees.  A request's last tile may have no more than half of a tile's rows; its steps take less than twice the time per
// row then, in a way of the kernel's own (HALVES).  Two ways to hand units out:
//   shares   the steps of all units, in order, weighed by what they take (COST), are cut into runs of one cost, one per CTA, so that
//            every SM takes the same share whatever the lengths are.  A share may begin and end inside a unit, a step being its
//            who has the step's begin: that unit's parts are joined later.
//   turns    whole units, a request's last tile, which sees most keys, first: CTA c of n takes the units c, 2n - 1 - c, 2n + c, ...,
//            there and back again, so that who has the largest of one turn has the smallest of the next (512 units of a prompt of
//            4096: the longest CTA has 3 % more than its share; with c, n + c, 2n + c, ... it had 26).
#pragma once
#include <cstdint>

#include "pq_attention.h"
#include "pq_attn_mma.cuh"
#include "pq_ptx.cuh"

namespace pq {

// sum over 0 <= i < n of floor((a i + b) / m), by the Euclidean algorithm.  a n + b only falls: in 32 bits if it fits them at first
// (a 64-bit division is some hundred instructions).
template <typename T>
__device__ __forceinline__ uint64_t floor_sum_in(T n, T m, T a, T b) {
  uint64_t sum = 0;
  while (n > 0) {
    if (a >= m) sum += static_cast<uint64_t>(n - 1) * n / 2 * (a / m), a %= m;
    if (b >= m) sum += static_cast<uint64_t>(n) * (b / m), b %= m;
    const T top = a * n + b;
    if (top < m) break;
    n = top / m, b = top % m;
    const T x = a;
    a = m, m = x;
  }
  return sum;
}
__device__ inline uint64_t floor_sum(uint64_t n, uint64_t m, uint64_t a, uint64_t b) {
  if (m <= 0xffffffffu && a * n + b <= 0xffffffffu)   // n >= 1: a and b, too
    return floor_sum_in(static_cast<uint32_t>(n), static_cast<uint32_t>(m), static_cast<uint32_t>(a), static_cast<uint32_t>(b));
  return floor_sum_in(n, m, a, b);
}

constexpr int kFewSteps = 6;   // of a unit at most: shares are not worth their joining

// The same where a and m are constants and a n + b is below 2^32: without a division but by them.
template <uint32_t m, uint32_t a>
__device__ __forceinline__ uint64_t floor_sum_of(uint32_t n, uint32_t b) {
  uint64_t sum = static_cast<uint64_t>(n - 1) * n / 2 * (a / m) + static_cast<uint64_t>(n) * (b / m);   // n >= 1
  b %= m;
  if constexpr (a % m != 0) {
    const uint32_t top = a % m * n + b;
    if (top >= m) sum += floor_sum_of<a % m, m>(top / m, top % m);
  }
  return sum;
}

// A kernel's units.  Shape has
//   rows     query rows of a tile
//   heads    rows per token: row r of a request is of token r / heads
//   keys     keys of a step;  half_keys: of one of a half
//   copies   units per tile
//   halves   whether a last tile of half the rows has steps of its own kind
//   cost, half_cost, unit_cost   of a step, of the beginning and the end of a unit
//   uint64_t floors(n, b)   sum over 0 <= i < n of floor((rows i + b) / (keys heads)), n >= 1
template <class Shape>
struct Request {
  int q0, n;              // first token, tokens (n * heads, and units over all requests, below 2^31)
  int k0, L, hi;          // first key (where keys are ragged rows), keys, keys that can be read (below 2^31 - 2 half_keys)
  Shape s;
  uint32_t all;           // rows: below 2^31
  int tiles;
  int half;               // the tile that is a half (none: -1)
  __device__ __forceinline__ void settle(bool halves) {
    all = static_cast<uint32_t>(n) * static_cast<uint32_t>(s.heads);
    tiles = static_cast<int>((all + s.rows - 1) / static_cast<uint32_t>(s.rows));
    half = halves && may_halve() ? tiles - 1 : -1;
  }
  __device__ __forceinline__ bool may_halve() const { return s.halves && tiles > 0 && all - static_cast<uint32_t>(tiles - 1) * s.rows <= static_cast<uint32_t>(s.rows / 2); }
  __device__ __forceinline__ int units() const { return tiles * s.copies; }
  __device__ __forceinline__ bool same() const { return L < n || hi < L; }   // all rows end alike: fewer keys than rows, or than the table holds
  __device__ __forceinline__ int seen(int tile) const {   // keys, 1 at least
    if (same()) return max(hi, 1);
    const uint32_t last = min(static_cast<uint32_t>(tile + 1) * s.rows, all) - 1;
    return L - n + static_cast<int>(last / static_cast<uint32_t>(s.heads)) + 1;
  }
  __device__ __forceinline__ int steps(int tile, bool as_half) const { return as_half ? (seen(tile) - 1) / s.half_keys + 1 : (seen(tile) - 1) / s.keys + 1; }
  __device__ __forceinline__ int steps(int tile) const { return steps(tile, tile == half); }
  __device__ __forceinline__ int cost(int tile, bool as_half) const { return steps(tile, as_half) * (as_half ? s.half_cost : s.cost) + s.unit_cost; }
  __device__ __forceinline__ int64_t before_tile(int tile) const {   // of one copy of the tiles before; tile < tiles
    if (tile == 0) return 0;
    if (same()) return static_cast<int64_t>(cost(0, false)) * tile;
    return static_cast<int64_t>(s.floors(tile, s.rows - 1 + static_cast<uint64_t>(L - n) * s.heads)) * s.cost + static_cast<int64_t>(tile) * (s.cost + s.unit_cost);
  }
  __device__ __forceinline__ int64_t before(int unit) const {        // unit < units()
    const int tile = unit / s.copies, copy = unit - tile * s.copies;
    return before_tile(tile) * s.copies + static_cast<int64_t>(copy) * (copy ? cost(tile, tile == half) : 0);
  }
};

// A unit of a CTA, or its part of one.
template <class Shape>
struct Unit {
  int b;                            // request
  int unit;                         // shares: of the request; turns: counted from request `base`'s first
  int64_t left;                     // shares: cost, this unit's included; turns: 1 as long as there are any
  int off, spent, rest;             // shares: cost of the unit that is the shares' before, this one's, those' behind
  int step, count, all_steps;       // the unit's steps: first, how many, of all
  int tile, copy;
  Request<Shape> r;
  __device__ __forceinline__ bool half() const { return tile == r.half; }
  // Shares: the first unit from `unit` of request `b` on that has the begin of a step in this share (which ends inside the last one).
  template <class Args>
  __device__ __forceinline__ void find(const Args& a, bool halves) {
    for (;; left -= spent, ++unit, off = 0) {
      if (left <= 0) return;
      while (unit >= r.units()) {
        if (++b >= a.requests) {
          left = 0;
          return;
        }
        r = a.request(b, halves), unit = 0;
      }
      tile = unit / r.s.copies, copy = unit - tile * r.s.copies;
      all_steps = r.steps(tile);
      rest = all_steps * (half() ? r.s.half_cost : r.s.cost) + r.s.unit_cost - off;
      spent = static_cast<int>(min(static_cast<int64_t>(rest), left)), rest -= spent;
      auto begun = [&](int x) {   // steps that begin before x; what the unit itself takes comes first
        x = max(x - r.s.unit_cost, 0);
        return half() ? (x + r.s.half_cost - 1) / r.s.half_cost : (x + r.s.cost - 1) / r.s.cost;
      };
      step = begun(off), count = begun(off + spent) - step;
      if (count > 0) return;
    }
  }
};

// Halves: in kHalvesCut only where none of them fits a share, so that all of them are cut.
enum Halves { kHalvesCut, kHalvesAlways };
template <class Shape>
struct ShareRoom {   // shared memory
  Unit<Shape> first;
  int per, halves;   // cost of a share; whether halves are told apart
  int64_t sums[2][32];
  int shortest, longest, units, cut;
  __device__ __forceinline__ void clear() { shortest = 0x7fffffff, longest = units = 0; }   // before find_share
};

// By the whole block up to the sums over requests, then by one warp (all of them take turns issuing: 1000 to 2000 cycles more);
// false: whole units by turns take no longer.  They are not cut, which costs about two units' begins and ends,
// one for the other part and one for the joining (35 requests of two units each, of eight steps, on 74 pairs of CTAs: 29 us; 39 in shares).
template <int kThreads, Halves kHalves, class Args>
__device__ __forceinline__ bool find_share(const Args& a, int worker, int workers, int least, ShareRoom<typename Args::Shape>& room) {
  const int tid = threadIdx.x, lane = tid & 31, warp = tid >> 5;
  const int each = (a.requests + kThreads - 1) / kThreads;
  const int b0 = min(tid * each, a.requests), b1 = min(b0 + each, a.requests);
  int shortest = 0x7fffffff, longest = 0, units = 0;   // of the halves; of all units, their number
  auto total = [&](int b, int64_t (&t)[2]) {   // cost without, with halves
    const auto r = a.request(b, false);
    t[0] = t[1] = 0;
    if (r.tiles == 0) return;
    const int64_t before = r.before_tile(r.tiles - 1);
    const int last = r.cost(r.tiles - 1, false);
    t[0] = t[1] = (before + last) * r.s.copies;
    longest = max(longest, last), units += r.units();
    if (!r.may_halve()) return;
    const int half = r.cost(r.tiles - 1, true);
    t[1] = (before + half) * r.s.copies;
    shortest = min(shortest, half);
  };
  int64_t mine[2] = {0, 0};
#pragma unroll 1
  for (int b = b0; b < b1; ++b) {
    int64_t t[2];
    total(b, t);
    mine[0] += t[0], mine[1] += t[1];
  }
  constexpr int kFirst = kHalves == kHalvesAlways ? 1 : 0;
  auto inclusive = [&](int64_t v) {
#pragma unroll
    for (int o = 1; o < 32; o <<= 1) {
      const int64_t x = __shfl_up_sync(0xffffffffu, v, o);
      if (lane >= o) v += x;
    }
    return v;
  };
#pragma unroll
  for (int h = kFirst; h < 2; ++h) {
    const int64_t in = inclusive(mine[h]);
    if (lane == 31) room.sums[h][warp] = in;
  }
  if (kHalves == kHalvesCut) shortest = __reduce_min_sync(0xffffffffu, shortest);
  longest = __reduce_max_sync(0xffffffffu, longest), units = __reduce_add_sync(0xffffffffu, units);
  if (lane == 0 && units > 0) {
    if (kHalves == kHalvesCut) atomicMin(&room.shortest, shortest);
    atomicMax(&room.longest, longest), atomicAdd(&room.units, units);
  }
  __syncthreads();
  if (warp == 0) {
    auto per_of = [&](int64_t cost) {   // (a 64-bit division takes 700 cycles)
      const uint64_t up = static_cast<uint64_t>(cost + workers - 1);
      return max(static_cast<int64_t>(up >> 32 ? up / workers : static_cast<uint32_t>(up) / static_cast<uint32_t>(workers)), static_cast<int64_t>(least));
    };
    int h = 1;
    int64_t of_warp = lane < kThreads / 32 ? room.sums[1][lane] : 0, in = inclusive(of_warp), all = __shfl_sync(0xffffffffu, in, 31), per = per_of(all);
    if (kHalves == kHalvesCut && room.shortest <= per) {
      h = 0, of_warp = lane < kThreads / 32 ? room.sums[0][lane] : 0, in = inclusive(of_warp), all = __shfl_sync(0xffffffffu, in, 31);
      per = per_of(all);
    }
    const bool cut = (room.units + workers - 1) / workers * static_cast<int64_t>(room.longest) > per + 2 * a.shape().unit_cost;
    const int64_t first = per * worker;
    Unit<typename Args::Shape> u;
    u.left = cut ? max(min(per, all - first), static_cast<int64_t>(0)) : 0;
    if (u.left > 0) {
      // whose requests: a warp's, a thread's, one of them; then the last unit of it that begins at or before `first`, 32 at a time
      const int w = __ffs(__ballot_sync(0xffffffffu, first < in)) - 1;
      int64_t at = first - __shfl_sync(0xffffffffu, in - of_warp, w);
      const int r0 = min((w * 32 + lane) * each, a.requests), r1 = min(r0 + each, a.requests);
      int64_t of_lane = h ? mine[1] : mine[0];
      if (w > 0) {
        of_lane = 0;
#pragma unroll 1
        for (int b = r0; b < r1; ++b) {
          int64_t t[2];
          total(b, t);
          of_lane += h ? t[1] : t[0];
        }
      }
      in = inclusive(of_lane);
      const int owner = __ffs(__ballot_sync(0xffffffffu, at < in)) - 1;
      at -= in - of_lane;
      u.b = r0;
      if (lane == owner) {
        for (; u.b < r1 - 1; ++u.b) {
          int64_t t[2];
          total(u.b, t);
          const int64_t x = h ? t[1] : t[0];
          if (at < x) break;
          at -= x;
        }
      }
      u.b = __shfl_sync(0xffffffffu, u.b, owner), at = __shfl_sync(0xffffffffu, at, owner);
      u.r = a.request(u.b, h != 0), u.unit = 0;
      int n = u.r.units();
      while (n > 1) {
        const int stride = (n + 31) / 32, probe = lane * stride;
        const uint32_t yes = __ballot_sync(0xffffffffu, probe < n && u.r.before(u.unit + probe) <= at);   // of lane 0 always
        const int k = 31 - __clz(yes);
        u.unit += k * stride, n = min(stride, n - k * stride);
      }
      u.off = static_cast<int>(at - u.r.before(u.unit));
      u.find(a, h != 0);
    }
    if (lane == 0) room.first = u, room.per = static_cast<int>(min(per, static_cast<int64_t>(0x7fffffff))), room.halves = h, room.cut = cut;
  }
  __syncthreads();
  return room.cut != 0;
}

// Walks the units of one CTA, as every warp of it does for itself; all lanes together.  The first one of a share is found once for
// all warps (each by itself, from code of its own, took up to 5000 cycles).  By turns, a lane keeps one of 32 requests, so that going
// on to the next unit reads no memory (it took 3000 cycles between a unit's end and the next one's begin).
template <class Args>
struct Walk : Unit<typename Args::Shape> {
  using Shape = typename Args::Shape;
  using Base = Unit<Shape>;
  using Base::b, Base::unit, Base::left, Base::off, Base::spent, Base::rest, Base::step, Base::count, Base::all_steps, Base::tile, Base::copy, Base::r, Base::half;
  const Args& a;
  const bool shares, halves;
  int step_there, step_back;        // turns: to the next unit
  Request<Shape> mine;              // turns: the lane's, base + lane
  int base, in;                     // units of the requests from base to the lane's, its own included
  __device__ __forceinline__ Walk(const Args& args, const ShareRoom<Shape>& room, bool by_shares, bool halve, int worker, int of)
      : a(args), shares(by_shares), halves(by_shares ? room.halves != 0 : halve) {
    if (shares) {
      static_cast<Base&>(*this) = room.first;
    } else {
      step_there = 2 * (of - 1 - worker) + 1, step_back = 2 * worker + 1, unit = worker, left = 1, base = 0;
      fetch();
      find();
    }
  }
  __device__ __forceinline__ bool more() const { return left > 0; }
  __device__ __forceinline__ bool whole() const { return count == all_steps; }
  __device__ __forceinline__ void next() {
    if (shares) {
      left -= spent, ++unit, off = 0;
    } else {
      const int x = step_there;
      unit += x, step_there = step_back, step_back = x;
    }
    find();
  }
  // Parts of a unit whose first steps are this share's: every share behind it that has the begin of a step has one.
  __device__ __forceinline__ int parts(int per) const {
    return 1 + (max(rest - ((half() ? r.s.half_cost : r.s.cost) - 1), 0) + per - 1) / per;
  }
  __device__ __forceinline__ void fetch() {
    const int lane = threadIdx.x & 31;
    in = 0;
    if (base + lane < a.requests) mine = a.request(base + lane, halves), in = mine.units();
#pragma unroll
    for (int o = 1; o < 32; o <<= 1) {
      const int x = __shfl_up_sync(0xffffffffu, in, o);
      if (lane >= o) in += x;
    }
  }
  __device__ __forceinline__ void find() {
    if (left <= 0) return;
    if (shares) return Base::find(a, halves);
    for (;;) {
      const uint32_t behind = __ballot_sync(0xffffffffu, in > unit);
      if (behind) {
        const int at = __ffs(behind) - 1;
        const int before = __shfl_sync(0xffffffffu, in, max(at - 1, 0));
        b = base + at;
        r.q0 = __shfl_sync(0xffffffffu, mine.q0, at), r.n = __shfl_sync(0xffffffffu, mine.n, at);
        r.k0 = __shfl_sync(0xffffffffu, mine.k0, at), r.L = __shfl_sync(0xffffffffu, mine.L, at), r.hi = __shfl_sync(0xffffffffu, mine.hi, at);
        r.s = a.shape();
        r.settle(halves);
        const int of_request = unit - (at > 0 ? before : 0);
        tile = of_request / r.s.copies, copy = of_request - tile * r.s.copies;
        tile = r.tiles - 1 - tile;
        step = 0, count = all_steps = r.steps(tile);
        return;
      }
      unit -= __shfl_sync(0xffffffffu, in, 31);
      base += 32;
      if (base >= a.requests) break;
      fetch();
    }
    left = 0;
  }
};

// Joins the parts of a unit that was cut: a thread has 16 values of one row, lanes along the rows.  A part is [values / 4][kRows]
// x 4 sums, then [kRows] x (reference, sum of weights); part(i) is the i-th of `parts`, `first` the thread's first value, `to` where
// its row has them (nullptr: there is no such row).  All of four parts is loaded at once: L2 latency bounds it.
// kGroups > 1: so many threads of a block share a row's parts, in blocks of kGroups x kRows threads.  One request of 52000 tokens
// in 148 parts: 54 us with one group, 40 with four; 64 requests in two or three parts each, where four times the blocks
// come in waves: 123 and 140.
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

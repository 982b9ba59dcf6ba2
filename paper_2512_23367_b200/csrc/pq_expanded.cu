// Latent attention, expanded form: ragged queries over keys and values multiplied out per head, with one rotary key a token
// for all heads, on the tcgen05 tensor cores.  See include/pq.h for the contract.
#include <cuda_fp16.h>

#include <cmath>
#include <type_traits>

#include "pq_attention.h"
#include "pq_attn_mma.cuh"
#include "pq_internal.h"
#include "pq_ptx.cuh"
#include "pq_schedule.cuh"

namespace pq {

namespace {

constexpr int kTile = 128;          // query rows of one accumulator
constexpr int kUnit = 2 * kTile;    // of a unit
constexpr int kKeys = 80;           // keys of one step
constexpr int kNope = 128, kValue = 128, kQuery = kNope + PQ_LATENT_ROPE;
constexpr int kSoft = 512;          // threads of the four softmax warpgroups, two per accumulator
constexpr int kIssuer = 16, kLoadK = 17, kWatcher = 18, kLoadV = 19, kThreads = 640;   // warps
constexpr int kSoftRegs = 104, kRestRegs = 64;   // 512 x 104 + 128 x 64 = 640 x 96, what the launch holds
constexpr int kPanelQ = kTile * 128, kPanelK = kKeys * 128;   // bytes of 64 values of all rows
constexpr int kQueryBytes = 3 * kPanelQ, kKeyBytes = 3 * kPanelK, kValueBytes = 2 * kPanelK;
constexpr int kSmem = 2 * kQueryBytes + 2 * kKeyBytes + 2 * kValueBytes + 1024 /* alignment */;
constexpr int kPartFloats = kUnit * (kValue + 2);   // per query tile [32][128 rows] x 4 sums, then [128 rows] x (reference, sum of weights)
constexpr int kLeastSteps = 4;      // of a CTA, so that its parts are worth joining
// Tensor memory columns: S, P and O of each accumulator.
constexpr uint32_t kColP = 2 * kKeys, kColO = 256;
static_assert(kColP + kKeys <= kColO, "tensor memory");
// Named barriers, as in the paged tile kernel: "P written" (two), "operand tile landed", the two warps that share 32 rows
// (eight pairs), "S read" (two), accumulators' sums.
constexpr uint32_t kBarP = 1, kBarTile = 3, kBarPair = 4, kBarRead = 12, kBarSoft = 14;

// Halves take a key tile by the accumulators in turn, which costs five eighths of a step of both query tiles (1430 of 2330 cycles:
// keys and values come from L2 for half as many products), and a unit about as much as three steps.
struct ExpandedShape {
  static constexpr int rows = kUnit, heads = 1, keys = kKeys, half_keys = kKeys, halves = 1, cost = 8, half_cost = 5, unit_cost = 20;
  int copies;
  // (rows and keys are below 2^31)
  __device__ __forceinline__ static uint64_t floors(uint64_t n, uint64_t b) { return floor_sum_of<kKeys, kUnit>(static_cast<uint32_t>(n), static_cast<uint32_t>(b)); }
};
struct ExpandedArgs {
  using Shape = ExpandedShape;
  const int* q_start;
  const int* kv_start;
  __half* out;
  int64_t tokens;
  int requests, heads;
  float scale_log2;      // > 0
  uint32_t q_and, q_xor; // a scale of 0 or below is folded into the products: (s & q_and) ^ q_xor
  int shares;            // units are handed out in equal runs of steps, with parts to join
  float* partials;       // two parts per CTA
  int4* joins;           // per CTA: first token, tokens, head, parts
  int* status;
  uint32_t wait_limit;

  __device__ __forceinline__ Shape shape() const { return Shape{heads}; }
  __device__ __forceinline__ Request<Shape> request(int b, bool halves) const {
    Request<Shape> r;
    r.s = shape();
    r.q0 = q_start[b];
    r.n = static_cast<int>(min(static_cast<int64_t>(max(q_start[b + 1] - r.q0, 0)), tokens));
    r.k0 = kv_start[b];
    r.L = r.hi = max(kv_start[b + 1] - r.k0, 0);
    r.settle(halves);
    return r;
  }
};

// A CTA's units.
struct ExpandedWalk : Walk<ExpandedArgs> {
  __device__ __forceinline__ ExpandedWalk(const ExpandedArgs& args, const ShareRoom<Shape>& room, bool by_shares) : Walk<ExpandedArgs>(args, room, by_shares, true, blockIdx.x, gridDim.x) {}
};
// The key tiles of a unit, or of the part of one that a CTA has.
struct Part {
  int toks, N, lag;      // tokens; (S, O) steps; steps that an O follows its S by
  bool two;              // more than one accumulator's rows: the accumulators are two query tiles, else the even and the odd key tiles
  __device__ __forceinline__ explicit Part(const ExpandedWalk& w)
      : toks(min(kUnit, w.r.n - w.tile * kUnit)), two(!w.half()) {
    N = two ? 2 * w.count : w.count;
    lag = two ? 2 : 1;
  }
};

// Tensor bound.  A unit is 256 query rows of one head as two accumulators of 128, or up to 128 rows as two accumulators that
// take the even and the odd key tiles and are joined at the end: one's softmax runs while the tensor core works for the
// other, as in the paged tile kernel.  What differs:
//   - the product with the keys goes over 192 values, 128 of the head and 64 that all heads share, so that queries and keys
//     take half as much shared memory again.  With steps of 128 keys one step and a half would fit; with 80 two steps do, loads
//     run a whole step ahead, and tensor memory has room for an S of each accumulator (with 96 keys and one S in turn, the
//     tensor core waited 300 of 1390 cycles for S to be read: a prompt of 4096 took 180 us).  S takes 12 MMAs of N = 80 (51
//     cycles each, bound by shared memory; 40 by arithmetic), O 5 of N = 128 (64): 1864 cycles per 256 x 80 scores where
//     arithmetic alone would take 1600.
//   - a CTA stays on its SM and walks through its units: queries of the next one are on the way, and its first S computed,
//     while the results of the last one go out.
//   - keys and values are rows of one linear's output, read through one tensor map with heads as its second dimension.
// A step of 256 x 80 takes 2150 to 2200 cycles, and a unit's begin and end 7000: the next queries' way in, and the sums' way out, which
// the next unit's first S overlaps.  A prompt of 4096 of 32 heads: 158 us alone, 175 to 180 in a row under the power cap, where the tensor cores at
// cuBLAS's rate take 106; chunks of up to 700 tokens of 16 heads over up to 5000: 98 and 9 for joining the parts, where 53.
__global__ void __launch_bounds__(kThreads, 1)
expanded_kernel(const __grid_constant__ CUtensorMap map_q, const __grid_constant__ CUtensorMap map_kv, const __grid_constant__ CUtensorMap map_rope,
                const ExpandedArgs a) {
  constexpr float kTop = 7.0f;      // a weight at the reference is 2^kTop
  extern __shared__ uint8_t smem_raw[];
  __shared__ __align__(8) uint64_t bars[16];
  __shared__ uint32_t s_tmem;
  __shared__ volatile int s_abort;
  __shared__ ShareRoom<ExpandedShape> s_share;
  __shared__ float s_swap[2 * kTile];
  __shared__ float2 s_ml[kTile];

  const int tid = threadIdx.x, warp = __shfl_sync(0xffffffffu, tid >> 5, 0), lane = tid & 31;
  const uint32_t bar_k = smem_u32(bars), bar_v = bar_k + 16, bar_kfree = bar_v + 16, bar_vfree = bar_kfree + 16;   // two of each
  const uint32_t bar_s = bar_vfree + 16, bar_o = bar_s + 16;                                                       // per accumulator
  const uint32_t bar_q = bar_o + 16, bar_qfree = bar_q + 8, bar_read = bar_qfree + 8, bar_drain = bar_read + 8;
  if (tid == 0) {
    for (int i = 0; i < 12; ++i) mbar_init(bar_k + 8 * i, 1);
    mbar_init(bar_q, 1);
    mbar_init(bar_qfree, 1);
    mbar_init(bar_read, 1);
    mbar_init(bar_drain, 1);
    fence_mbar_init();
    s_abort = 0, s_share.clear();
    tma_prefetch_desc(&map_q), tma_prefetch_desc(&map_kv), tma_prefetch_desc(&map_rope);
  }
  if (warp == kIssuer) {
    tmem_alloc(smem_u32(&s_tmem), 512);
    tmem_relinquish();
  }
  tc_fence_before_sync();
  __syncthreads();
  tc_fence_after_sync();
  grid_dep_wait();
  const bool shares = a.shares != 0 && find_share<kThreads, kHalvesAlways>(a, blockIdx.x, gridDim.x, kLeastSteps * ExpandedShape::cost, s_share);
  grid_dep_launch();   // only now: a later launch's CTA may take this SM's tensor memory when it is given back
  const uint32_t tmem = __shfl_sync(0xffffffffu, s_tmem, 0);
  const uint32_t sq = (smem_u32(smem_raw) + 1023u) & ~1023u, ring_k = sq + 2 * kQueryBytes, ring_v = ring_k + 2 * kKeyBytes;
  const WaitCtx wc{&s_abort, a.wait_limit};
  uint32_t issued = 0, units = 0;   // producers: tiles requested; units

  if (warp >= kSoft / 32) {
    asm volatile("setmaxnreg.dec.sync.aligned.u32 %0;" ::"n"(kRestRegs));
    if (warp == kLoadK) {
      // ------------------------------------------------------------------ queries and keys
      bool ok = true;
      for (ExpandedWalk w(a, s_share, shares); ok && w.more(); w.next()) {
        const Part part(w);
        if (units > 0 && !(ok = warp_wait(bar_qfree, (units - 1) & 1, wc))) break;
        if (lane == 0) mbar_arrive_expect_tx(bar_q, part.two ? 2 * kQueryBytes : kQueryBytes);
        __syncwarp();
        if (lane < (part.two ? 6 : 3)) {
          const int tile = lane / 3, x = lane % 3;
          tma_load_3d(sq + lane * kPanelQ, &map_q, bar_q, x * 64, w.copy, w.r.q0 + w.tile * kUnit + tile * kTile);
        }
        ++units;
        for (int i = 0; i < w.count; ++i) {
          const uint32_t st = issued & 1, dst = ring_k + st * kKeyBytes, bar = bar_k + 8 * st;
          if (issued >= 2 && !(ok = warp_wait(bar_kfree + 8 * st, ((issued >> 1) & 1) ^ 1, wc))) break;
          const int row = w.r.k0 + (w.step + i) * kKeys;
          if (lane == 0) mbar_arrive_expect_tx(bar, kKeyBytes);
          __syncwarp();
          if (lane < 2) tma_load_3d(dst + lane * kPanelK, &map_kv, bar, lane * 64, w.copy, row);
          if (lane == 2) tma_load_3d(dst + 2 * kPanelK, &map_rope, bar, 0, 0, row);
          ++issued;
          __syncwarp();
        }
      }
    } else if (warp == kLoadV) {
      // ------------------------------------------------------------------ values
      bool ok = true;
      for (ExpandedWalk w(a, s_share, shares); ok && w.more(); w.next()) {
        const Part part(w);
        for (int i = 0; i < w.count; ++i) {
          const uint32_t st = issued & 1, dst = ring_v + st * kValueBytes;
          if (issued >= 2 && !(ok = warp_wait(bar_vfree + 8 * st, ((issued >> 1) & 1) ^ 1, wc))) break;
          const uint32_t bar = bar_v + 8 * st;
          if (lane == 0) mbar_arrive_expect_tx(bar, kValueBytes);
          __syncwarp();
          if (lane < 2) tma_load_3d(dst + lane * kPanelK, &map_kv, bar, kNope + lane * 64, w.copy, w.r.k0 + (w.step + i) * kKeys);
          ++issued;
          __syncwarp();
        }
      }
    } else if (warp == kIssuer) {
      // ------------------------------------------------------------------ MMA issuer
      // As in the paged tile kernel: the whole warp walks, one elected thread issues, and after the watcher has given up the
      // steps go on without MMAs, so that the named barriers stay in step.
      constexpr uint32_t id_qk = umma_idesc_f16(kKeys, false), id_pv = umma_idesc_f16(kValue, true);
      const uint32_t leader = elect_one();
      const uint32_t q_lo = desc_k(sq), k_lo0 = desc_k(ring_k), v_lo0 = desc_mn(ring_v, kPanelK);
      bool live = true;
      uint32_t n = 0, seg = 0;   // key tiles, units before
      // S = Q K^T of the accumulator's query tile, O += P V of the step before it.  Which accumulator, and so every operand but the
      // stage, is known at compile time: with operands in other than uniform registers an MMA takes 85 to 100 cycles to issue, and
      // a step took 3300.
      auto scores = [&](auto acc, auto tile, uint32_t stage, bool gives_back, bool last) {
        if (leader && live) {
          const uint32_t ql = q_lo + decltype(tile)::value * (kQueryBytes / 16), kl = k_lo0 + stage * (kKeyBytes / 16);
          const uint32_t d = tmem + decltype(acc)::value * kKeys;
          umma_f16_ss<0>(d, ql, kl, id_qk);
#pragma unroll
          for (int k = 1; k < kQuery / 16; ++k) umma_f16_ss<1>(d, ql + (k / 4) * (kPanelQ / 16) + (k % 4) * 2, kl + (k / 4) * (kPanelK / 16) + (k % 4) * 2, id_qk);
          umma_commit(bar_s + 8 * decltype(acc)::value);
          if (gives_back) umma_commit(bar_kfree + 8 * stage);
          if (last) umma_commit(bar_qfree);
        }
        __syncwarp();
      };
      auto sums = [&](auto acc, uint32_t stage, bool first, bool gives_back) {
        named_bar_sync(kBarP + decltype(acc)::value, 288);
        tc_fence_after_sync();
        if (leader && live) {
          const uint32_t vl = v_lo0 + stage * (kValueBytes / 16), d = tmem + kColO + decltype(acc)::value * kValue, p = tmem + kColP + decltype(acc)::value * (kKeys / 2);
          umma_f16_ts(d, p, vl, id_pv, first ? 0u : 1u);
#pragma unroll
          for (int k = 1; k < kKeys / 16; ++k) umma_f16_ts(d, p + 8 * k, vl + k * 128, id_pv, 1u);
          umma_commit(bar_o + 8 * decltype(acc)::value);
          if (gives_back) umma_commit(bar_vfree + 8 * stage);
        }
        __syncwarp();
      };
      auto landed = [&]() {
        live = tile_landed(kBarTile, true) && live;
        tc_fence_after_sync();
      };
      auto read = [&](auto acc) {   // the accumulator's S is in registers
        named_bar_sync(kBarRead + decltype(acc)::value, 288);
        tc_fence_after_sync();
      };
      constexpr std::integral_constant<int, 0> k0{};
      constexpr std::integral_constant<int, 1> k1{};
      for (ExpandedWalk w(a, s_share, shares); w.more(); w.next()) {
        const Part part(w);
        live = live && warp_wait(bar_q, seg & 1, wc);
        auto sums_free = [&](int t) {   // the sums of the unit before have been read
          if (t == 1 && seg > 0) live = warp_wait(bar_read, (seg - 1) & 1, wc) && live;
        };
        if (part.two) {   // S of both query tiles, then O of both of the key tile before
          for (int t = 0; t <= w.count; ++t) {
            const bool more = t < w.count;
            if (t > 0) read(k0);
            if (more) landed(), scores(k0, k0, n & 1, false, false);
            if (t > 0) landed(), sums_free(t), sums(k0, (n - 1) & 1, t == 1, false);
            if (t > 0) read(k1);
            if (more) scores(k1, k1, n & 1, true, t == w.count - 1);
            if (t > 0) sums(k1, (n - 1) & 1, t == 1, true);
            if (more) ++n;
          }
        } else {     // the accumulators take the even and the odd key tiles of one query tile
          for (int t = 0; t <= w.count; t += 2) {
            if (t < w.count) landed(), scores(k0, k0, n & 1, true, t == w.count - 1);
            if (t > 0) landed(), read(k1), sums(k1, (n - 1) & 1, t == 2, true);
            if (t < w.count) ++n;
            if (t + 1 > w.count) break;
            if (t + 1 < w.count) landed(), scores(k1, k0, n & 1, true, t + 1 == w.count - 1);
            landed(), sums_free(t + 1), read(k0), sums(k0, (n - 1) & 1, t == 0, true);
            if (t + 1 < w.count) ++n;
          }
        }
        ++seg;
      }
    } else if (warp == kWatcher) {
      // ------------------------------------------------------------------ watcher: waits for the operand tiles a step ahead
      bool ok = true;
      uint32_t g = 0;
      for (ExpandedWalk w(a, s_share, shares); w.more(); w.next()) {
        const Part part(w);
        for (int u = 0; u < part.N + part.lag; ++u) {
#pragma unroll
          for (int is_v = 0; is_v < 2; ++is_v) {
            const int x = u - is_v * part.lag;
            if (x < 0 || x >= part.N || (part.two && (x & 1))) continue;
            const uint32_t t = g + (part.two ? x >> 1 : x);
            ok = ok && warp_wait((is_v ? bar_v : bar_k) + 8 * (t & 1), (t >> 1) & 1, wc);
            const int dead = w.r.hi - (w.step + (part.two ? x >> 1 : x)) * kKeys;   // from here on rows are not the request's
            if (is_v && ok && dead < kKeys) {   // their weights are 0, but 0 x NaN is not
              for (int j = lane; j < (kKeys - max(dead, 0)) * 16; j += 32) {
                const int r = max(dead, 0) + (j >> 4), c = j & 15;
                asm volatile("st.shared.v4.u32 [%0], {%1, %1, %1, %1};" ::"r"(ring_v + (t & 1) * kValueBytes + (c >> 3) * kPanelK + r * 128 + (c & 7) * 16), "r"(0) : "memory");
              }
              fence_proxy_async_smem();
              __syncwarp();
            }
            tile_landed(kBarTile, ok);
          }
        }
        g += w.count;
      }
    }
  } else {
    // -------------------------------------------------------------------- softmax, two threads per row
    asm volatile("setmaxnreg.inc.sync.aligned.u32 %0;" ::"n"(kSoftRegs));
    const int acc = warp >> 3;                       // accumulator
    const int half = (warp >> 2) & 1;                // the thread's 40 keys of a tile, and its half of the values
    const int r = tid & 127;                         // row of the tile
    const uint32_t lane_off = static_cast<uint32_t>(warp & 3) << 21;   // 32 lanes per warp, lane in bits 16 and up
    const uint32_t t_s = tmem + acc * kKeys + 40 * half + lane_off, t_p = tmem + kColP + acc * (kKeys / 2) + 20 * half + lane_off;
    const uint32_t t_out = tmem + kColO + acc * kValue + half * (kValue / 2) + lane_off;
    float* swap = s_swap + acc * kTile + r;
    const uint32_t pair = kBarPair + acc * 4 + (warp & 3);
    const float sc = a.scale_log2;
    const uint64_t sc2 = pair_f32(sc, sc);
    uint32_t n = 0;                                  // the accumulator's steps so far
    int4 join = make_int4(0, 0, 0, 0);
    bool ok = true;
    for (ExpandedWalk w(a, s_share, shares); w.more();) {
      const Part part(w);
      const bool two = part.two;
      const int tok = (two ? acc * kTile : 0) + r;   // of the unit
      const int p0 = w.r.L - w.r.n + w.tile * kUnit + (two ? acc * kTile : 0);   // position of the tile's first row
      const int see_to = min(p0 + r, w.r.hi - 1) - 40 * half;                    // last key of the row, from the thread's first
      const int all_to = min(p0 + 1, w.r.hi);                                    // every row sees the keys before
      const int mine = two ? w.count : (w.count - acc + 1) >> 1;
      float m = -INFINITY, l = 0.0f;   // m: the reference that is subtracted, in powers of two; l: the thread's own keys
      for (int i = 0; i < mine; ++i, ++n) {
        const int key0 = (w.step + (two ? i : 2 * i + acc)) * kKeys;
        ok = ok && warp_wait(bar_s + 8 * acc, n & 1, wc);
        tc_fence_after_sync();
        uint32_t s[32], s2[8];
        tmem_ld_32x32(t_s, s);
        tmem_ld_32x8(t_s + 32, s2);
        tmem_ld_wait();
        tc_fence_before_sync();
        hand_over(kBarRead + acc, 288, ok);
        if (a.q_xor != 0u || a.q_and == 0u) {
#pragma unroll
          for (int j = 0; j < 32; ++j) s[j] = (s[j] & a.q_and) ^ a.q_xor;
#pragma unroll
          for (int j = 0; j < 8; ++j) s2[j] = (s2[j] & a.q_and) ^ a.q_xor;
        }
        if (key0 + kKeys > all_to) {   // some row does not see all keys
          const int to = see_to - key0;
#pragma unroll
          for (int j = 0; j < 32; ++j)
            if (j > to) s[j] = 0xff800000u;   // -inf
#pragma unroll
          for (int j = 0; j < 8; ++j)
            if (32 + j > to) s2[j] = 0xff800000u;
        }
        float top[4];   // of the eights at 8 h, and of those left at 32
#pragma unroll
        for (int h = 0; h < 4; ++h) {
          const uint32_t* v = s + 8 * h;
          top[h] = max3(__uint_as_float(v[0]), __uint_as_float(v[1]), __uint_as_float(v[2]));
          top[h] = max3(top[h], __uint_as_float(v[3]), __uint_as_float(v[4]));
          top[h] = max3(top[h], __uint_as_float(v[5]), __uint_as_float(v[6]));
          top[h] = max3(top[h], __uint_as_float(v[7]), __uint_as_float(s2[2 * h]));
          top[h] = fmaxf(top[h], __uint_as_float(s2[2 * h + 1]));
        }
        float t = fmaxf(max3(top[0], top[1], top[2]), top[3]) * sc;
        bool done = i == 0;   // the product with the weights before these has been taken
        if (pair_any(pair, t > m + 8.0f)) {   // rare after the first tiles: some row of the 32
          t = pair_combine<false>(swap, pair, half, t);
          const bool grown = t > m + 8.0f;
          const float f = grown ? (m == -INFINITY ? 0.0f : exp2_approx(m - t)) : 1.0f;
          if (grown) m = t;
          l *= f;
          if (i > 0) {   // O holds the sums up to the tile before
            ok = ok && warp_wait(bar_o + 8 * acc, (n - 1) & 1, wc);
            done = true;
            tc_fence_after_sync();
#pragma unroll 1
            for (int h = 0; h < kValue / 32; ++h) {
              uint32_t o[16];
              tmem_ld_32x16(t_out + 16 * h, o);
              tmem_ld_wait();
#pragma unroll
              for (int j = 0; j < 16; ++j) o[j] = __float_as_uint(__uint_as_float(o[j]) * f);
              tmem_st_32x16(t_out + 16 * h, o);
            }
          }
        }
        const float off = kTop - (m == -INFINITY ? 0.0f : m);
        const uint64_t off2 = pair_f32(off, off);
        uint32_t p[16], p2[4], asked = 0;
        uint64_t sum = 0;
        auto weigh = [&](uint32_t x0, uint32_t x1) {
          float e0, e1;
          unpair_f32(fma_f32x2(pair_f32(__uint_as_float(x0), __uint_as_float(x1)), sc2, off2), e0, e1);
          e0 = exp2_approx(e0);
          e1 = exp2_approx(e1);
          sum = add_f32x2(sum, pair_f32(e0, e1));
          return pack_f16(e0, e1);
        };
#pragma unroll
        for (int j = 0; j < 16; ++j) p[j] = weigh(s[2 * j], s[2 * j + 1]);
        asked = mbar_test2(bar_o + 8 * acc, (n - 1) & 1, bar_o + 8 * acc, (n - 1) & 1);
#pragma unroll
        for (int j = 0; j < 4; ++j) p2[j] = weigh(s2[2 * j], s2[2 * j + 1]);
        float l0, l1;
        unpair_f32(sum, l0, l1);
        l += l0 + l1;
        if (!done && !__all_sync(0xffffffffu, asked)) ok = ok && warp_wait(bar_o + 8 * acc, (n - 1) & 1, wc);
        tc_fence_after_sync();
        tmem_st_32x16(t_p, p);
        tmem_st_32x4(t_p + 16, p2);
        tmem_st_wait();
        tc_fence_before_sync();
        hand_over(kBarP + acc, 288, ok);
      }
      // ------------------------------------------------------------------ the unit's (or part's) end
      const bool both = !two && w.count > 1, writer = two || acc == 0, whole = w.whole(), begins = w.step == 0;
      const int64_t row = static_cast<int64_t>(w.r.q0) + w.tile * kUnit + tok;
      const bool writes = tok < part.toks && row >= 0 && row < a.tokens;
      __half* to = a.out + (row * a.heads + w.copy) * kValue + half * (kValue / 2);
      if (!whole && begins) join = make_int4(w.r.q0 + w.tile * kUnit, part.toks, w.copy, w.parts(s_share.per));
      w.next();   // (the next request's lengths are on the way while the last product is waited for)
      if (mine > 0) ok = ok && warp_wait(bar_o + 8 * acc, (n - 1) & 1, wc);
      tc_fence_after_sync();
      l = pair_combine<true>(swap, pair, half, l);   // the sum of the row's two threads
      // Accumulators of the even and the odd tiles are joined in the first one's threads: both lie in the same lanes.
      float f0 = 1.0f, f1 = 0.0f;
      if (both) {
        if (acc == 1 && half == 0) s_ml[r] = make_float2(m, l);
        tc_fence_before_sync();
        named_bar_sync(kBarSoft, kSoft);
        tc_fence_after_sync();
        if (acc == 0) {
          const float2 ml = s_ml[r];
          const float M = fmaxf(m, ml.x), Ms = M == -INFINITY ? 0.0f : M;
          f0 = exp2_approx(m - Ms), f1 = exp2_approx(ml.x - Ms);
          l = l * f0 + ml.y * f1;
          m = M;
        }
      }
      if (writer) {
        const float inv = l > 0.0f ? 1.0f / l : 0.0f;
        float* pp = a.partials + (2 * static_cast<int64_t>(blockIdx.x) + begins) * kPartFloats + (two ? acc : 0) * (kTile * (kValue + 2));
#pragma unroll 1
        for (int h = 0; h < kValue / 32; ++h) {
          uint32_t o[16];
          tmem_ld_32x16(t_out + 16 * h, o);
          float v[16];
          if (both) {
            uint32_t o1[16];
            tmem_ld_32x16(t_out + kValue + 16 * h, o1);
            tmem_ld_wait();
#pragma unroll
            for (int j = 0; j < 16; ++j) v[j] = fmaf(__uint_as_float(o1[j]), f1, __uint_as_float(o[j]) * f0);
          } else {
            tmem_ld_wait();
#pragma unroll
            for (int j = 0; j < 16; ++j) v[j] = __uint_as_float(o[j]);
          }
          if (!writes) continue;
          if (whole) {
            store_32_bytes(to + 16 * h, pack_f16(v[0] * inv, v[1] * inv), pack_f16(v[2] * inv, v[3] * inv), pack_f16(v[4] * inv, v[5] * inv),
                           pack_f16(v[6] * inv, v[7] * inv), pack_f16(v[8] * inv, v[9] * inv), pack_f16(v[10] * inv, v[11] * inv),
                           pack_f16(v[12] * inv, v[13] * inv), pack_f16(v[14] * inv, v[15] * inv));
          } else {
#pragma unroll
            for (int j = 0; j < 4; ++j)
              reinterpret_cast<float4*>(pp)[(half * 16 + 4 * h + j) * kTile + r] = make_float4(v[4 * j], v[4 * j + 1], v[4 * j + 2], v[4 * j + 3]);
          }
        }
        if (!whole && half == 0) reinterpret_cast<float2*>(pp + kTile * kValue)[r] = make_float2(m, l);
      }
      // All together go to the next unit: the second accumulator's threads may have had nothing to do in this one, and
      // must not run ahead of the sums, and of s_ml, that the first one's threads still read.
      tc_fence_before_sync();
      named_bar_sync(kBarSoft, kSoft);
      if (tid == 0) mbar_arrive(bar_read);
    }
    if (a.shares != 0 && tid == 0) a.joins[blockIdx.x] = join;
  }

  // ---------------------------------------------------------------------- teardown
  tc_fence_before_sync();
  __syncthreads();
  tc_fence_after_sync();
  if (s_abort) {
    // Some role gave up.  What has been handed to the hardware still completes by itself and must have done so before shared
    // and tensor memory go away: the producers' copies and the issuer's MMAs.
    if (warp == kIssuer && elect_one()) {
      umma_commit(bar_drain);
      mbar_drain(bar_drain, 0u);
    }
    if ((warp == kLoadK || warp == kLoadV) && lane == 0) {
      for (uint32_t i = issued > 2 ? issued - 2 : 0; i < issued; ++i) mbar_drain((warp == kLoadK ? bar_k : bar_v) + 8 * (i & 1), (i >> 1) & 1);
      if (warp == kLoadK && units > 0) mbar_drain(bar_q, (units - 1) & 1);
    }
    __syncthreads();
    if (tid == 0) atomicExch(a.status, static_cast<int>(PQ_ERR_TIMEOUT));
  }
  if (warp == kIssuer) tmem_dealloc(tmem, 512);
}

// Joins the parts of units that were cut: blocks per CTA that had a unit's first part, query tile and 32 values with one group of
// threads per row, 16 with four.
template <int kGroups>
__global__ void __launch_bounds__((kGroups > 1 ? kGroups : 2) * kTile) expanded_join_kernel(const ExpandedArgs a) {
  grid_dep_launch();
  grid_dep_wait();
  const int4 join = a.joins[blockIdx.x];   // first token, tokens, head, parts
  const int tile = blockIdx.y, tok = tile * kTile + static_cast<int>(threadIdx.x % kTile);
  const int first = kGroups > 1 ? blockIdx.z * 16 : blockIdx.z * 32 + static_cast<int>(threadIdx.x / kTile) * 16;
  if (join.w == 0 || tile * kTile >= join.y) return;
  const int64_t row = static_cast<int64_t>(join.x) + tok;
  // the unit's first part is the second one of its CTA, the others the first of theirs
  auto part = [&](int i) { return a.partials + (2 * (static_cast<int64_t>(blockIdx.x) + i) + (i == 0)) * kPartFloats + tile * (kTile * (kValue + 2)); };
  const bool there = tok < join.y && row >= 0 && row < a.tokens;
  join_parts<kTile, kValue, kGroups>(part, join.w, first, there ? a.out + (row * a.heads + join.z) * kValue + first : nullptr);
}

}  // namespace

size_t expanded_partial_bytes(int sms) { return static_cast<size_t>(sms) * (2 * kPartFloats * sizeof(float) + sizeof(int4)); }

}  // namespace pq

using namespace pq;

extern "C" {

int pq_expanded_attention(const void* q_f16, int64_t q_stride, int32_t heads, const void* kv_f16, int64_t kv_stride, const void* k_rope_f16,
                          int64_t k_rope_stride, int64_t keys, const int32_t* q_start, const int32_t* kv_start, int64_t requests,
                          int64_t tokens, int64_t max_q, float scale, void* out_f16, void* workspace, size_t workspace_bytes, void* stream) {
  if (heads < 1 || heads > 1024 || requests < 0 || requests > 0x7fffffff || tokens < 0 || tokens > 0x7fffffff / heads) return PQ_ERR_SHAPE;
  if (keys < 0 || keys > 0x7fffffff || max_q < 0 || !std::isfinite(scale)) return PQ_ERR_SHAPE;
  const int64_t limit = int64_t(1) << 38;   // what a tensor map holds
  if (q_stride < static_cast<int64_t>(heads) * kQuery || kv_stride < static_cast<int64_t>(heads) * (kNope + kValue) || k_rope_stride < PQ_LATENT_ROPE) return PQ_ERR_SHAPE;
  if (q_stride % 8 != 0 || kv_stride % 8 != 0 || k_rope_stride % 8 != 0 || q_stride >= limit || kv_stride >= limit || k_rope_stride >= limit) return PQ_ERR_SHAPE;
  if (requests > PQ_MAX_REQUESTS) return PQ_ERR_LIMIT;
  if (requests == 0 || tokens == 0) return PQ_OK;
  if (!q_f16 || !q_start || !kv_start || !out_f16 || (keys > 0 && (!kv_f16 || !k_rope_f16))) return PQ_ERR_NULL;
  if (!aligned16(q_f16) || !aligned16(kv_f16) || !aligned16(k_rope_f16) || !aligned16(out_f16) || !aligned256(workspace)) return PQ_ERR_ALIGN;
  int rc = check_arch();
  if (rc != PQ_OK) return rc;
  cudaStream_t st = static_cast<cudaStream_t>(stream);
  const bool none = keys == 0;
  if (none) {   // nothing is seen, and a tensor map needs a row: one of the queries', masked
    kv_f16 = k_rope_f16 = q_f16;
    keys = 1;
  }
  ExpandedArgs a{q_start, kv_start, static_cast<__half*>(out_f16), tokens, static_cast<int>(requests), heads, scale * 1.44269504f,
                 0xffffffffu, 0u, 0, nullptr, nullptr, device_status_ptr(), wait_limit()};
  if (a.status == nullptr) return PQ_ERR_CUDA;
  if (a.scale_log2 == 0.0f) {
    a.q_and = 0u, a.scale_log2 = 1.0f;
  } else if (a.scale_log2 < 0.0f) {
    a.q_xor = 0x80000000u, a.scale_log2 = -a.scale_log2;
  }
  const int sms = sm_count();
  // Units, at most.  Many of them are handed out whole, in turn; of few, every SM takes an equal share.
  if (max_q > tokens) max_q = tokens;
  const int64_t by_rows = tokens / kUnit + requests, by_request = requests * ((max_q + kUnit - 1) / kUnit);
  const int64_t units = (by_rows < by_request ? by_rows : by_request) * heads;
  const Scratch sc = scratch_from(workspace, workspace_bytes);
  if (sc.partials != nullptr && sc.partial_bytes >= expanded_partial_bytes(sms) && units < 3 * sms && keys > kFewSteps * kKeys) {
    a.shares = 1;
    a.partials = reinterpret_cast<float*>(sc.partials);
    a.joins = reinterpret_cast<int4*>(a.partials + static_cast<size_t>(sms) * 2 * kPartFloats);
  }
  static PerDeviceOnce once;
  if ((rc = set_dynamic_smem_once(once, expanded_kernel, kSmem)) != PQ_OK) return rc;
  // The kernel's register split draws on what the launch holds: a build whose launch holds less must not run.
  static const int regs = [] {
    cudaFuncAttributes f = {};
    return cudaFuncGetAttributes(&f, expanded_kernel) == cudaSuccess ? f.numRegs : 0;
  }();
  if (regs * kThreads < kSoft * kSoftRegs + (kThreads - kSoft) * kRestRegs) return PQ_ERR_CUDA;
  CUtensorMap mq = {}, mkv = {}, mr = {};
  if ((rc = make_tmap_heads(&mq, q_f16, tokens, heads, kQuery, q_stride, kQuery, kTile)) != PQ_OK) return rc;
  if ((rc = make_tmap_heads(&mkv, kv_f16, keys, none ? 1 : heads, none ? kQuery : kNope + kValue, kv_stride, kNope + kValue, kKeys)) != PQ_OK) return rc;
  if ((rc = make_tmap_heads(&mr, k_rope_f16, keys, 1, PQ_LATENT_ROPE, k_rope_stride, PQ_LATENT_ROPE, kKeys)) != PQ_OK) return rc;
  if ((rc = launch_dependent(expanded_kernel, dim3(sms), dim3(kThreads), kSmem, st, mq, mkv, mr, a)) != PQ_OK || !a.shares) return rc;
  return many_parts(units, sms, keys / kKeys, kLeastSteps) ? launch_dependent(expanded_join_kernel<4>, dim3(sms, kUnit / kTile, kValue / 16), dim3(4 * kTile), 0, st, a)
                          : launch_dependent(expanded_join_kernel<1>, dim3(sms, kUnit / kTile, kValue / 32), dim3(2 * kTile), 0, st, a);
}

}  // extern "C"

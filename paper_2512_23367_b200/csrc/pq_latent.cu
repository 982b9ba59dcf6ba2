// Latent attention, absorbed form: queries in the latent space over the paged cache of latent vectors and rotary keys, on
// the tcgen05 tensor cores.  See include/pq.h for the contract.
#include <cuda_fp16.h>

#include <cmath>

#include "pq_attention.h"
#include "pq_attn_mma.cuh"
#include "pq_internal.h"
#include "pq_ptx.cuh"
#include "pq_schedule.cuh"

namespace pq {

namespace {

constexpr int kRows = 64;            // query rows (token x head) of a CTA
constexpr int kKeys = 64;            // cached tokens of one step
constexpr int kPanel = kKeys * 128;  // 64 rows of 64 values
constexpr int kSoft = 256;           // softmax threads: four per row
constexpr int kIssuer = 8, kLoader = 9, kWatcher = 10, kAhead = 11, kThreads = 384;   // warps
constexpr int kDistance = 2;         // steps that tokens are brought into L2 ahead of their use
constexpr int kLeastSteps = 2;       // of a CTA, so that its parts are worth joining

template <int kLatent>
struct LatentCfg {
  static constexpr int kPanels = kLatent / 64 + 1;        // of a row: the last one holds the rotary values
  static constexpr int kValuePanels = kLatent / 64;
  static constexpr int kGroups = kLatent / 256;           // panels are brought in and given back four at a time, the values of one MMA
  // Queries lie in tensor memory, as many panels of them as there is room for, the others in shared memory.
  static constexpr int kHeld = kLatent == 512 ? 7 : 4, kQueryPanels = kPanels - kHeld;
  static constexpr int kStages = kLatent == 512 ? 3 : 6;   // steps whose latent vectors fit at once
  static constexpr int kStage = kValuePanels * kPanel;
  static constexpr int kSmem = kQueryPanels * kPanel + kStages * kStage + 2 * kPanel /* rotary keys, P */ + 1024 /* alignment */;
  static constexpr int kPartFloats = kRows * (kLatent + 2);   // [kLatent / 4][64 rows] x 4 sums, [64 rows] x (reference, sum of weights)
  // Tensor memory columns: O; S; the queries, two FP16 values each.
  static constexpr uint32_t kCols = kLatent / 2, kColS = kCols, kColQ = kColS + kKeys / 2;
  static_assert(kColQ + 32 * kHeld <= 512, "tensor memory");
};

// Halves, of no more than 64 rows where two CTAs serve units: each takes every second one of their steps of 64 tokens, for five
// quarters of the time (3100 of 2450 cycles: no other CTA reads the tokens); a unit takes about as much as four steps.
struct LatentShape {
  static constexpr int keys = kKeys, half_keys = 2 * kKeys, copies = 1, cost = 4, half_cost = 5, unit_cost = 16;
  int rows, heads, halves;
  __device__ __forceinline__ uint64_t floors(uint64_t n, uint64_t b) const { return floor_sum(n, static_cast<uint64_t>(keys) * heads, rows, b); }
};
struct LatentArgs {
  using Shape = LatentShape;
  pq_latent_cache c;
  const int* table;
  int64_t width;
  const int* q_start;
  const int* kv_len;
  __half* out;
  int64_t tokens;
  int requests, heads;
  int paired;            // two CTAs serve the two halves of a unit of 128 rows
  float scale_log2;      // > 0
  uint32_t q_and, q_xor; // a scale of 0 or below is folded into the products: (s & q_and) ^ q_xor
  float* partials;       // two parts per CTA (nullptr: units are handed out whole, in turn)
  int4* joins;           // per CTA: first row (a 64-bit number), rows, parts (negative: of both CTAs each)
  int box;               // tokens of a TMA box: the largest power of two that divides both the page and 64
  int* status;
  uint32_t wait_limit;

  __device__ __forceinline__ Shape shape() const { return Shape{paired ? 2 * kRows : kRows, heads, paired}; }
  __device__ __forceinline__ Request<Shape> request(int b, bool halves) const {
    Request<Shape> r;
    r.s = shape();
    r.q0 = q_start[b];
    r.n = static_cast<int>(min(static_cast<int64_t>(max(q_start[b + 1] - r.q0, 0)), tokens));
    r.k0 = 0;
    r.L = max(kv_len[b], 0);
    r.hi = static_cast<int>(min(static_cast<int64_t>(r.L), width * c.page));
    r.settle(halves);
    return r;
  }
};

// A CTA's units, with the 64 rows of a unit that are its own.
struct LatentWalk : Walk<LatentArgs> {
  __device__ __forceinline__ LatentWalk(const LatentArgs& args, const ShareRoom<Shape>& room, bool by_shares)
      : Walk<LatentArgs>(args, room, by_shares, false, args.paired ? blockIdx.x >> 1 : blockIdx.x, args.paired ? gridDim.x >> 1 : gridDim.x) {}
  __device__ __forceinline__ int second() const { return a.paired ? blockIdx.x & 1 : 0; }
  __device__ __forceinline__ int row0() const { return tile * r.s.rows + (half() ? 0 : second() * kRows); }
  __device__ __forceinline__ int rows() const { return max(min(static_cast<int>(r.all) - row0(), kRows), 0); }
  __device__ __forceinline__ int key0(int i) const { return (half() ? 2 * (step + i) + second() : step + i) * kKeys; }
  __device__ __forceinline__ bool whole() const { return !half() && count == all_steps; }
};

// MMAs with M = 64 in the form that keeps B in place: all 128 lanes of tensor memory take part, lane r and lane 64 + r
// holding the lower and the upper half of row r's columns.  Per 16 of K: 32 cycles with N = 64 and 80 with 256, the time
// that shared memory takes to give the operands; the other form of M = 64 takes 32 and 128, and half of the lanes stay empty.
// Tokens lie in shared memory as [group of four panels][8 tokens][panel][128-byte rows, swizzled]: the swizzle's atoms of 8 rows
// stay whole, panels are 1024 bytes apart and groups of 8 tokens 4096, so that one TMA box brings all four panels of as many
// tokens as a page holds in a row.  (Panel after panel, a page of 16 tokens takes 36 boxes a step, 100 cycles each.)
constexpr uint32_t kAtom = 1024, kTokens8 = 4 * kAtom;
constexpr uint32_t kTokenHi = (kTokens8 >> 4) | (1u << 14) | (2u << 29);
template <int kAccumulate, uint32_t kHi>
__device__ __forceinline__ void umma_ws(uint32_t d, uint32_t a_lo, uint32_t b_lo, uint32_t idesc) {
  asm volatile("{\n\t.reg .pred p;\n\t.reg .b64 a, b;\n\tsetp.ne.b32 p, %4, 0;\n\tmov.b64 a, {%1, %5};\n\tmov.b64 b, {%2, %6};\n\t"
               "tcgen05.mma.ws.cta_group::1.kind::f16 [%0], a, b, %3, p;\n\t}"
               ::"r"(d), "r"(a_lo), "r"(b_lo), "r"(idesc), "n"(kAccumulate), "n"(kDescHi), "n"(kHi) : "memory");
}
__device__ __forceinline__ void umma_ws_first(uint32_t d, uint32_t a_lo, uint32_t b_lo, uint32_t idesc, uint32_t accumulate) {
  asm volatile("{\n\t.reg .pred p;\n\t.reg .b64 a, b;\n\tsetp.ne.b32 p, %4, 0;\n\tmov.b64 a, {%1, %5};\n\tmov.b64 b, {%2, %6};\n\t"
               "tcgen05.mma.ws.cta_group::1.kind::f16 [%0], a, b, %3, p;\n\t}"
               ::"r"(d), "r"(a_lo), "r"(b_lo), "r"(idesc), "r"(accumulate), "n"(kDescHi), "n"(kTokenHi) : "memory");
}
// A in tensor memory, row r in lane r and again in lane 64 + r, which multiplies it with the upper half of the columns.
template <int kAccumulate>
__device__ __forceinline__ void umma_ws_ts(uint32_t d, uint32_t a, uint32_t b_lo, uint32_t idesc) {
  asm volatile("{\n\t.reg .pred p;\n\t.reg .b64 b;\n\tsetp.ne.b32 p, %4, 0;\n\tmov.b64 b, {%2, %5};\n\t"
               "tcgen05.mma.ws.cta_group::1.kind::f16 [%0], [%1], b, %3, p;\n\t}"
               ::"r"(d), "r"(a), "r"(b_lo), "r"(idesc), "n"(kAccumulate), "n"(kTokenHi) : "memory");
}

// The sum, or the largest, of a value of the row's four threads, the same in all: `mine` is the thread's word, the others'
// lie 64 floats apart.
template <bool kSum>
__device__ __forceinline__ float row_combine(float* mine, const float* row, uint32_t id, float v) {
  *mine = v;
  named_bar_sync(id, 128);
  const float a = row[0], b = row[kRows], c = row[2 * kRows], d = row[3 * kRows];
  named_bar_sync(id, 128);
  return kSum ? (a + b) + (c + d) : fmaxf(fmaxf(a, b), fmaxf(c, d));
}

// Named barriers: the four warps that share 32 rows (two of them); "operands landed", between the watcher's and the issuer's
// warp; "S read" and "P written", 256 threads to the issuer's (S of the next step is only there when the issuer has had both).
// They do not pass through shared memory, which the tensor core
// keeps busy: with mbarriers, polled for in whichever order they came, a step took 3200 cycles.
constexpr uint32_t kBarRow = 1, kBarTile = 3, kBarRead = 4, kBarP = 5;

// A CTA serves 64 rows over its share of the steps.  All heads share the cache, so a row is any (token, head) and a step's 64
// tokens are read once for 64 rows; units of 128 rows are served by two CTAs, the second of which finds the tokens in L2.
// Per step, latent 512:
//   S = Q C^T            28 MMAs with A in tensor memory (28 cycles each: without it shared memory, which has to give A and B,
//                        takes 32) and 8 from shared memory; the latent vectors first, then the rotary keys, which have room
//                        for one step and are brought in while the vectors are multiplied
//   softmax              four threads per row: S to registers, running maximum, P = 2^(S - reference + 7) as FP16 to shared memory
//   O += P C             8 MMAs with N = 256 (80 cycles each), C as it lies (values contiguous), O of 64 rows in 256 columns
// in the order S(u + 1), O(u), so that a softmax runs under the next S: 1680 cycles of MMAs.  The reference moves, and O is
// multiplied, only when the maximum has grown by more than 2^8.
//
// Bound by HBM up to 64 rows a request: 72 KB a step take an SM's share of the bandwidth 3150 cycles, and steps come every
// 3300.  Two CTAs that share their tokens have 1580 cycles of bandwidth a step and take 2080 to 2300: the tensor cores wait for S to be
// read and for P.  (64 requests of 128 heads and 1000 to 8200 tokens: 115 us and 10 for joining the parts, where their bytes take 63;
// with latent 256 84 in all, where 35; 7 requests of up to four tokens of 32 heads and 4000 to 30000 tokens: 53 and 11, where 26; 1000 tokens
// of 16 heads: 13 and 5.)  A unit's begin and end take about 9000 cycles: queries, the first tokens, 128 KB of partial sums at 30 bytes
// a cycle.  Taken back for being slower: queries in shared memory and two steps of tokens (236 us for the 131 that it took then), two
// CTAs as a cluster that exchange halves of S (5300 cycles a step), MMAs over a pair of CTAs (2340).
template <int kLatent>
__global__ void __launch_bounds__(kThreads, 1)
latent_kernel(const __grid_constant__ CUtensorMap map_q, const __grid_constant__ CUtensorMap map_c, const __grid_constant__ CUtensorMap map_r, const LatentArgs a) {
  using C = LatentCfg<kLatent>;
  constexpr float kTop = 7.0f;          // a weight at the reference is 2^kTop
  constexpr int kCols = C::kCols;
  extern __shared__ uint8_t smem_raw[];
  __shared__ __align__(8) uint64_t bars[2 * C::kStages * C::kGroups + 8];
  __shared__ uint32_t s_tmem;
  __shared__ volatile int s_abort;
  __shared__ ShareRoom<LatentShape> s_share;
  __shared__ volatile uint32_t s_landed;   // steps
  __shared__ float s_swap[4][kRows];

  const int tid = threadIdx.x, warp = __shfl_sync(0xffffffffu, tid >> 5, 0), lane = tid & 31;
  // Of every stage's groups, of the rotary keys: they are there, they are free.  S is there; O has been summed.
  const uint32_t bar_full = smem_u32(bars), bar_free = bar_full + 8 * C::kStages * C::kGroups, bar_rope = bar_free + 8 * C::kStages * C::kGroups;
  const uint32_t bar_rfree = bar_rope + 8, bar_s = bar_rfree + 8, bar_o = bar_s + 8;
  // A unit's queries are there, are free; its sums have been read.
  const uint32_t bar_q = bar_o + 8, bar_qfree = bar_q + 8, bar_read = bar_qfree + 8, bar_drain = bar_read + 8;
  if (tid == 0) {
    for (int i = 0; i < 2 * C::kStages * C::kGroups + 4; ++i) mbar_init(bar_full + 8 * i, 1);   // up to bar_o
    mbar_init(bar_q, kSoft / 32 + (C::kQueryPanels > 0 ? 1 : 0));
    mbar_init(bar_qfree, 1);
    mbar_init(bar_read, kSoft / 32);
    mbar_init(bar_drain, 1);
    fence_mbar_init();
    s_abort = 0, s_landed = 0, s_share.clear();
    tma_prefetch_desc(&map_q), tma_prefetch_desc(&map_c), tma_prefetch_desc(&map_r);
  }
  if (warp == kIssuer) {
    tmem_alloc(smem_u32(&s_tmem), 512);
    tmem_relinquish();
  }
  tc_fence_before_sync();
  __syncthreads();
  tc_fence_after_sync();
  grid_dep_wait();
  const bool shares = a.partials != nullptr && find_share<kThreads, kHalvesCut>(a, blockIdx.x >> a.paired, gridDim.x >> a.paired, kLeastSteps * LatentShape::cost, s_share);
  grid_dep_launch();   // only now: a later launch's CTA may take this SM's tensor memory when it is given back
  const uint32_t tmem = __shfl_sync(0xffffffffu, s_tmem, 0), tmem_s = tmem + C::kColS;
  const uint32_t sq = (smem_u32(smem_raw) + 1023u) & ~1023u, ring = sq + C::kQueryPanels * kPanel, rope = ring + C::kStages * C::kStage, weights = rope + kPanel;
  const WaitCtx wc{&s_abort, a.wait_limit};
  uint32_t filled = 0, issued = 0, units = 0;   // loader: stages filled, steps (a unit's queries take a stage, too); units

  if (warp == kLoader) {
    // -------------------------------------------------------------------- loader: a lane requests one box
    const int pieces = kKeys / a.box, groups8 = a.box / 8;
    const int rows_all = static_cast<int>(a.c.pages * a.c.page);
    const bool mine = lane < pieces;
    bool ok = true;
    auto wait_free = [&](int g) {
      if (ok && filled >= C::kStages) ok = warp_wait(bar_free + 8 * ((filled % C::kStages) * C::kGroups + g), ((filled / C::kStages) & 1) ^ 1, wc);
    };
    for (LatentWalk w(a, s_share, shares); ok && w.more(); w.next()) {
      if (w.rows() == 0) continue;
      const int* trow = a.table + static_cast<int64_t>(w.b) * a.width;
      int id = -1, off = 0;
      auto look_up = [&](int i) {
        const int key = w.key0(i) + lane * a.box;
        id = -1;
        if (!mine || i >= w.count || key >= w.r.hi) return;
        const int col = key / a.c.page;
        off = key - col * a.c.page;
        id = trow[col];
      };
      look_up(0);
      // The unit's queries: panels for tensor memory by way of a stage, from which the softmax threads take them, the others to stay.
      const int q_row = w.r.q0 * a.heads + w.row0();
#pragma unroll
      for (int g = 0; g < C::kGroups; ++g) {
        const int panels = min(4, C::kHeld - 4 * g);
        const uint32_t full = bar_full + 8 * ((filled % C::kStages) * C::kGroups + g);
        wait_free(g);
        if (ok && lane == 0) mbar_arrive_expect_tx(full, panels * kPanel);
        __syncwarp();
        if (ok && lane < panels) tma_load_2d(ring + (filled % C::kStages) * C::kStage + (4 * g + lane) * kPanel, &map_q, full, (4 * g + lane) * 64, q_row);
      }
      if (ok && units > 0) ok = warp_wait(bar_qfree, (units - 1) & 1, wc);
      if (!ok) break;
      if (lane == 0) mbar_arrive_expect_tx(bar_q, C::kQueryPanels * kPanel);
      __syncwarp();
      if (lane < C::kQueryPanels) tma_load_2d(sq + lane * kPanel, &map_q, bar_q, (C::kHeld + lane) * 64, q_row);
      ++units, ++filled;
      for (int i = 0; i < w.count; ++i) {
        const uint32_t st = filled % C::kStages;
        const int row = (id < 0 || id >= a.c.pages ? rows_all : id * a.c.page + off) / 8;   // beyond the tensor: zeros
        const uint32_t dst = ring + st * C::kStage;
#pragma unroll
        for (int g = 0; g < C::kGroups; ++g) {
          const uint32_t full = bar_full + 8 * (st * C::kGroups + g);
          wait_free(g);
          if (ok && lane == 0) mbar_arrive_expect_tx(full, 4 * kPanel);
          __syncwarp();
          if (ok && mine) tma_load_4d(dst + 4 * g * kPanel + lane * groups8 * kTokens8, &map_c, full, 0, 0, 4 * g, row);
        }
        if (ok && issued > 0) ok = warp_wait(bar_rfree, (issued & 1) ^ 1, wc);
        if (!ok) break;
        if (lane == 0) mbar_arrive_expect_tx(bar_rope, kPanel);
        __syncwarp();
        if (mine) tma_load_4d(rope + lane * groups8 * kAtom, &map_r, bar_rope, 0, 0, C::kValuePanels, row);
        look_up(i + 1);   // used, and so waited for, in the next round
        ++issued, ++filled;
        __syncwarp();
      }
    }
  } else if (warp == kIssuer) {
    // -------------------------------------------------------------------- MMA issuer: the whole warp walks, one thread issues
    // (Descriptors have to stay in uniform registers, or an MMA takes 100 cycles to issue: hence plain loops over steps and
    // groups, and immediate accumulate flags.)  After the watcher has given up the steps go on without MMAs, so that the
    // named barriers stay in step.
    constexpr uint32_t id_s = umma_idesc_f16(kKeys, false, kRows), id_o = umma_idesc_f16(256, true, kRows);
    constexpr uint32_t kStage16 = C::kStage / 16, kPanel16 = kPanel / 16;
    const uint32_t leader = elect_one();
    const uint32_t q_lo = desc_k(sq), k_lo0 = desc_k(ring), v_lo0 = desc_mn(ring, kAtom), r_lo = desc_k(rope), p_lo = desc_k(weights), t_q = tmem + C::kColQ;
    uint32_t n = 0, seg = 0;   // stages, units before
    bool on = true;
    for (LatentWalk w(a, s_share, shares); w.more(); w.next()) {
      if (w.rows() == 0) continue;
      on = on && warp_wait(bar_q, seg & 1, wc);
      if (leader && on) {   // the queries have been taken out of their stage
#pragma unroll
        for (int g = 0; g < C::kGroups; ++g) mbar_arrive(bar_free + 8 * ((n % C::kStages) * C::kGroups + g));
      }
      __syncwarp();
      ++n;
      for (int i = 0; i <= w.count; ++i) {
        if (i > 0) named_bar_sync(kBarRead, kSoft + 32);   // S(u - 1) is in registers
        if (i < w.count) {   // S(u) = Q C^T: the latent vectors, a group as it lands, then the rotary keys, whose room is single
#pragma unroll
          for (int g = 0; g < C::kGroups; ++g) {
            on = tile_landed(kBarTile, true) && on;
            tc_fence_after_sync();
            if (leader && on) {
              const uint32_t kl = k_lo0 + (n % C::kStages) * kStage16 + g * (4 * kPanel16);
              if (g == 0) umma_ws_ts<0>(tmem_s, t_q, kl, id_s);
#pragma unroll
              for (int j = g == 0 ? 1 : 0; j < 16; ++j) {
                const uint32_t b = kl + (j / 4) * (kAtom / 16) + (j % 4) * 2;
                const int panel = 4 * g + j / 4;
                if (panel < C::kHeld) umma_ws_ts<1>(tmem_s, t_q + 8 * (16 * g + j), b, id_s);
                else umma_ws<1, kTokenHi>(tmem_s, q_lo + (panel - C::kHeld) * kPanel16 + (j % 4) * 2, b, id_s);
              }
            }
            __syncwarp();
          }
          on = tile_landed(kBarTile, true) && on;
          tc_fence_after_sync();
          if (leader && on) {
#pragma unroll
            for (int k = 0; k < 4; ++k) umma_ws<1, kDescHi>(tmem_s, q_lo + (C::kQueryPanels - 1) * kPanel16 + 2 * k, r_lo + 2 * k, id_s);
            umma_commit(bar_s);
            umma_commit(bar_rfree);
            if (i == w.count - 1) umma_commit(bar_qfree);
          }
          __syncwarp();
        }
        if (i > 0) {         // O += P C of the step before, while S(u) is read
          const uint32_t st = (n - 1) % C::kStages;
          if (i == 1 && seg > 0) on = warp_wait(bar_read, (seg - 1) & 1, wc) && on;   // O of the unit before has been read
          named_bar_sync(kBarP, kSoft + 32);
          tc_fence_after_sync();
          if (leader && on) {
            const uint32_t vl = v_lo0 + st * kStage16;
#pragma unroll
            for (int h = 0; h < C::kGroups; ++h) {
              umma_ws_first(tmem + 128 * h, p_lo, vl + 4 * h * kPanel16, id_o, i > 1);
#pragma unroll
              for (int k = 1; k < kKeys / 16; ++k) umma_ws<1, kTokenHi>(tmem + 128 * h, p_lo + 2 * k, vl + 4 * h * kPanel16 + k * (2 * kTokens8 / 16), id_o);
              umma_commit(bar_free + 8 * (st * C::kGroups + h));
            }
            umma_commit(bar_o);
          }
          __syncwarp();
        }
        if (i < w.count) ++n;
      }
      ++seg;
    }
  } else if (warp == kWatcher) {
    // -------------------------------------------------------------------- watcher: waits for the operands a step ahead
    bool ok = true;
    uint32_t u = 0, n = 0;
    for (LatentWalk w(a, s_share, shares); w.more(); w.next()) {
      if (w.rows() == 0) continue;
      ++n;   // the queries' stage is the softmax threads'
      for (int i = 0; i < w.count; ++i, ++u, ++n) {
        const int dead = max(w.r.hi - w.key0(i), 0);   // first token of the step that was never written
#pragma unroll
        for (int g = 0; g < C::kGroups; ++g) {
          ok = ok && warp_wait(bar_full + 8 * ((n % C::kStages) * C::kGroups + g), (n / C::kStages) & 1, wc);
          if (ok && dead < kKeys) {   // 0 x NaN is not 0: the weights of such tokens are, their vectors have to be
            for (int j = lane; j < (kKeys - dead) * 32; j += 32) {
              const int r = dead + (j >> 5), c = j & 31;
              const uint32_t at = ring + (n % C::kStages) * C::kStage + g * (4 * kPanel) + (r >> 3) * kTokens8 + (c >> 3) * kAtom + (r & 7) * 128 + (c & 7) * 16;
              asm volatile("st.shared.v4.u32 [%0], {%1, %1, %1, %1};" ::"r"(at), "r"(0) : "memory");
            }
            fence_proxy_async_smem();
            __syncwarp();
          }
          tile_landed(kBarTile, ok);
        }
        if (lane == 0) s_landed = u + 1;
        ok = ok && warp_wait(bar_rope, u & 1, wc);
        tile_landed(kBarTile, ok);
      }
    }
  } else if (warp == kAhead) {
    // -------------------------------------------------------------------- tokens into L2, kDistance steps ahead of their use,
    // where two CTAs share them.  There three steps of room are less than what memory's latency asks for at twice the rate
    // (64 ragged requests: 130 us without, 126 with one or two steps ahead, 130 with six, whose lines come too early; with latent 256
    // 103 without, 88, 84 and 86; 32 requests of 4000 tokens 69, 66, 64 and 70).  One CTA by itself is bound by memory, and gains nothing
    // (148 requests of 2000 tokens of 16 heads: 84.6 us without, 85.6 with).
    const char* data = static_cast<const char*>(a.c.data);
    constexpr int kLines = C::kPanels;   // of 128 bytes, per token
    const int tokens = kKeys / 2, first = static_cast<int>(blockIdx.x & 1) * tokens;
    uint32_t n = 0;
    bool on = a.paired != 0;
    for (LatentWalk w(a, s_share, shares); on && w.more(); w.next()) {
      if (w.rows() == 0) continue;
      const int* trow = a.table + static_cast<int64_t>(w.b) * a.width;
      for (int i = 0; on && i < w.count; ++i, ++n) {
        if (n < static_cast<uint32_t>(C::kStages) || w.half()) continue;   // being loaded; not shared
        for (uint32_t polls = 0; on && (s_landed == 0 || s_landed + kDistance < n); ++polls) {   // (not in the way of the first ones)
          __nanosleep(100);
          on = polls < wc.limit && !s_abort;
        }
        for (int t = lane; t < tokens; t += 32) {
          const int key = w.key0(i) + first + t;
          const int id = key < w.r.hi ? trow[key / a.c.page] : -1;
          if (id < 0 || id >= a.c.pages) continue;
          const char* at = data + (static_cast<int64_t>(id) * a.c.page + key % a.c.page) * (kLines * 128);
#pragma unroll
          for (int j = 0; j < kLines; ++j) asm volatile("prefetch.global.L2 [%0];" ::"l"(at + 128 * j));
        }
      }
    }
  } else {
    // -------------------------------------------------------------------- softmax, four threads per row
    const int r = tid & 63;
    const int half = (warp >> 1) & 1, part = 2 * half + (warp >> 2);   // the lanes' 32 tokens of a step; the thread's 16 of them
    const uint32_t lane_off = static_cast<uint32_t>(warp & 3) << 21;   // 32 lanes per warp, lane in bits 16 and up
    const uint32_t t_s = tmem_s + 16 * (warp >> 2) + lane_off, t_q = tmem + C::kColQ + lane_off, t_o = tmem + (kCols / 2) * (warp >> 2) + lane_off;
    const uint32_t id = kBarRow + (warp & 1);
    float* swap = &s_swap[part][r];
    const float* swap_row = &s_swap[0][r];
    const float sc = a.scale_log2;
    const uint64_t sc2 = pair_f32(sc, sc);
    uint32_t u = 0, n = 0;   // steps, stages
    int4 join = make_int4(0, 0, 0, 0);
    bool ok = true;
    // A unit's queries are taken, and its first S computed, before the sums of the unit before go out.
    LatentWalk w(a, s_share, shares);
    bool begins = false, whole = false, there = false, open = false;   // of the unit before
    float m = 0.0f, l = 0.0f;
    int64_t at = 0;   // row of the output
    for (;;) {
      while (w.more() && w.rows() == 0) w.next();
      const bool more = w.more();
      if (more) {   // the unit's queries out of their stage: the two warps of a lane take half of the row's panels each
        const uint32_t stage = ring + (n % C::kStages) * C::kStage + r * 128;
#pragma unroll
        for (int g = 0; g < C::kGroups; ++g) ok = ok && warp_wait(bar_full + 8 * ((n % C::kStages) * C::kGroups + g), (n / C::kStages) & 1, wc);
        for (int c = warp >> 2; c < 2 * C::kHeld; c += 2) {   // of 32 values
          uint32_t x[16];
#pragma unroll
          for (int j = 0; j < 4; ++j)
            asm volatile("ld.shared.v4.u32 {%0, %1, %2, %3}, [%4];" : "=r"(x[4 * j]), "=r"(x[4 * j + 1]), "=r"(x[4 * j + 2]), "=r"(x[4 * j + 3])
                         : "r"(stage + (c >> 1) * kPanel + ((((c & 1) * 4 + j) ^ (r & 7)) << 4)) : "memory");
          tmem_st_32x16(t_q + 16 * c, x);
        }
        tmem_st_wait();
        tc_fence_before_sync();
        __syncwarp();
        if (lane == 0) mbar_arrive(bar_q);
        n += 1 + w.count;
      }
      if (open) {   // ---------------------------------------------------- the end of the unit (or part) before
        ok = ok && warp_wait(bar_o, (u - 1) & 1, wc);
        tc_fence_after_sync();
        l = row_combine<true>(swap, swap_row, id, l);
        const float inv = l > 0.0f ? 1.0f / l : 0.0f;
        float* pp = a.partials + (2 * static_cast<int64_t>(blockIdx.x) + begins) * C::kPartFloats;
#pragma unroll 1
        for (int c = (kCols / 2) * (warp >> 2), k = 0; k < kCols / 2; k += 32, c += 32) {
          uint32_t o[32];
          tmem_ld_32x32(t_o + k, o);
          tmem_ld_wait();
          const int value = (c >> 7) * 256 + half * 128 + (c & 127);   // columns 128 h .. of tensor memory are the values 256 h + 128 half ..
          if (!there) continue;
          if (whole) {
            __half* to = a.out + at * kLatent + value;
#pragma unroll
            for (int j = 0; j < 2; ++j) {   // whole 32-byte sectors
              uint32_t x[8];
#pragma unroll
              for (int i = 0; i < 8; ++i) x[i] = pack_f16(__uint_as_float(o[16 * j + 2 * i]) * inv, __uint_as_float(o[16 * j + 2 * i + 1]) * inv);
              store_32_bytes(to + 16 * j, x[0], x[1], x[2], x[3], x[4], x[5], x[6], x[7]);
            }
          } else {
            float4* to = reinterpret_cast<float4*>(pp) + (value / 4) * kRows + r;
#pragma unroll
            for (int j = 0; j < 8; ++j)
              to[j * kRows] = make_float4(__uint_as_float(o[4 * j]), __uint_as_float(o[4 * j + 1]), __uint_as_float(o[4 * j + 2]), __uint_as_float(o[4 * j + 3]));
          }
        }
        if (!whole && there && part == 0) reinterpret_cast<float2*>(pp + kRows * kLatent)[r] = make_float2(m, l);
        tc_fence_before_sync();
        __syncwarp();
        if (lane == 0) mbar_arrive(bar_read);
      }
      if (!more) break;
      const int rows = w.rows(), shift = w.r.L - w.r.n;
      const int row0 = w.row0(), row = row0 + r;
      const bool live = r < rows;
      const int p0 = shift + row0 / a.heads;                                     // the first row's position
      const int see_to = live ? min(shift + row / a.heads, w.r.hi - 1) - 16 * part : -1;   // from the thread's first token
      const int all_to = min(p0 + 1, w.r.hi);                                    // every row sees the tokens before
      m = -INFINITY, l = 0.0f;   // m: the reference, in powers of two; l: the thread's own tokens
      for (int i = 0; i < w.count; ++i, ++u) {
        const int key0 = w.key0(i);
        ok = ok && warp_wait(bar_s, u & 1, wc);
        tc_fence_after_sync();
        uint32_t s[16];
        tmem_ld_32x16(t_s, s);
        tmem_ld_wait();
        tc_fence_before_sync();
        hand_over(kBarRead, kSoft + 32, ok);
        if (a.q_xor != 0u || a.q_and == 0u) {
#pragma unroll
          for (int j = 0; j < 16; ++j) s[j] = (s[j] & a.q_and) ^ a.q_xor;
        }
        if (key0 + kKeys > all_to || rows < kRows) {
          const int to = see_to - key0;
#pragma unroll
          for (int j = 0; j < 16; ++j)
            if (j > to) s[j] = 0xff800000u;   // -inf
        }
        float top[2];
#pragma unroll
        for (int h = 0; h < 2; ++h) {
          const uint32_t* v = s + 8 * h;
          top[h] = max3(__uint_as_float(v[0]), __uint_as_float(v[1]), __uint_as_float(v[2]));
          top[h] = max3(top[h], __uint_as_float(v[3]), __uint_as_float(v[4]));
          top[h] = max3(top[h], __uint_as_float(v[5]), __uint_as_float(v[6]));
          top[h] = fmaxf(top[h], __uint_as_float(v[7]));
        }
        float t = fmaxf(top[0], top[1]) * sc;
        bool taken = i == 0;   // the weights of the step before
        if (pair_any<128>(id, t > m + 8.0f)) {   // rare after the first steps: some row of the 32
          t = row_combine<false>(swap, swap_row, id, t);
          const bool grown = t > m + 8.0f;
          const float f = grown ? (m == -INFINITY ? 0.0f : exp2_approx(m - t)) : 1.0f;
          if (grown) m = t;
          l *= f;
          if (i > 0) {   // O holds the sums up to the step before
            ok = ok && warp_wait(bar_o, (u - 1) & 1, wc);
            taken = true;
            tc_fence_after_sync();
#pragma unroll 1
            for (int c = 0; c < kCols / 2; c += 32) {
              uint32_t o[32];
              tmem_ld_32x32(t_o + c, o);
              tmem_ld_wait();
#pragma unroll
              for (int j = 0; j < 32; ++j) o[j] = __float_as_uint(__uint_as_float(o[j]) * f);
              tmem_st_32x32(t_o + c, o);
            }
            tmem_st_wait();
          }
        }
        const float off = kTop - (m == -INFINITY ? 0.0f : m);
        const uint64_t off2 = pair_f32(off, off);
        uint64_t sum = 0;
        uint32_t q[8];
#pragma unroll
        for (int j = 0; j < 8; ++j) {
          float e0, e1;
          unpair_f32(fma_f32x2(pair_f32(__uint_as_float(s[2 * j]), __uint_as_float(s[2 * j + 1])), sc2, off2), e0, e1);
          e0 = exp2_approx(e0);
          e1 = exp2_approx(e1);
          sum = add_f32x2(sum, pair_f32(e0, e1));
          q[j] = pack_f16(e0, e1);
        }
        if (!taken) ok = ok && warp_wait(bar_o, (u - 1) & 1, wc);
        const uint32_t to = weights + r * 128;
#pragma unroll
        for (int c = 0; c < 2; ++c)
          asm volatile("st.shared.v4.u32 [%0], {%1, %2, %3, %4};" ::"r"(to + (((2 * part + c) ^ (r & 7)) << 4)),
                       "r"(q[4 * c]), "r"(q[4 * c + 1]), "r"(q[4 * c + 2]), "r"(q[4 * c + 3]) : "memory");
        fence_proxy_async_smem();
        tc_fence_before_sync();
        hand_over(kBarP, kSoft + 32, ok);
        float l0, l1;
        unpair_f32(sum, l0, l1);
        l += l0 + l1;
      }
      at = static_cast<int64_t>(w.r.q0) * a.heads + row;
      there = live && at >= 0 && at < a.tokens * a.heads, whole = w.whole(), begins = w.step == 0, open = true;
      if (!whole && begins) {
        const int64_t first = at - r;
        join = make_int4(static_cast<int>(first & 0xffffffff), static_cast<int>(first >> 32), rows,
                         w.parts(s_share.per) * (w.half() ? -2 : 1));
      }
      w.next();
    }
    if (a.partials && tid == 0) a.joins[blockIdx.x] = join;
  }

  // ---------------------------------------------------------------------- teardown
  tc_fence_before_sync();
  __syncthreads();
  tc_fence_after_sync();
  if (s_abort) {
    // Some role gave up.  What has been handed to the hardware still completes by itself and must have done so before shared
    // and tensor memory go away: the loader's copies and the issuer's MMAs.
    if (warp == kIssuer && elect_one()) {
      umma_commit(bar_drain);
      mbar_drain(bar_drain, 0u);
    }
    if (warp == kLoader && lane == 0) {
      for (uint32_t i = filled >= C::kStages ? filled + 1 - C::kStages : 0; i <= filled; ++i) {   // the last may be in part on its way
        for (int g = 0; g < C::kGroups; ++g) mbar_drain(bar_full + 8 * ((i % C::kStages) * C::kGroups + g), (i / C::kStages) & 1);
      }
      mbar_drain(bar_rope, (issued & 1) ^ 1), mbar_drain(bar_rope, issued & 1);
      if (units > 0) mbar_drain(bar_q, (units - 1) & 1);
    }
    __syncthreads();
    if (tid == 0) atomicExch(a.status, static_cast<int>(PQ_ERR_TIMEOUT));
  }
  if (warp == kIssuer) tmem_dealloc(tmem, 512);
}

// Joins the parts of units that were cut: blocks per CTA that had a unit's first part, of 16 values with four groups of threads
// per row, of 64 with one.
constexpr int kJoinGroups = 4, kJoinThreads = 4 * kRows;
template <int kLatent, int kGroups>
__global__ void __launch_bounds__(kJoinThreads) latent_join_kernel(const LatentArgs a) {
  grid_dep_launch();
  grid_dep_wait();
  const int4 join = a.joins[blockIdx.x];
  const bool both = join.w < 0;   // the parts of two neighbouring CTAs each; the first one joins them
  if (join.w == 0 || (both && (blockIdx.x & 1))) return;
  const int r = threadIdx.x % kRows, first = kGroups > 1 ? blockIdx.y * 16 : blockIdx.y * 64 + threadIdx.x / kRows * 16;
  const int64_t at = (static_cast<int64_t>(join.y) << 32 | static_cast<uint32_t>(join.x)) + r;
  const int next = a.paired && !both ? 2 : 1, begin = both ? 2 : 1;
  // the unit's first parts are the second ones of their CTAs, the others the first
  auto part = [&](int i) { return a.partials + (2 * (static_cast<int64_t>(blockIdx.x) + i * next) + (i < begin)) * LatentCfg<kLatent>::kPartFloats; };
  const bool there = r < join.z && at >= 0 && at < a.tokens * a.heads;
  join_parts<kRows, kLatent, kGroups>(part, abs(join.w), first, there ? a.out + at * kLatent + first : nullptr);
}

size_t partial_bytes(int latent, int sms) { return static_cast<size_t>(sms) * (2 * kRows * (latent + 2) * sizeof(float) + sizeof(int4)); }

template <int kLatent>
int launch(LatentArgs& a, const void* q, int sms, cudaStream_t stream) {
  using C = LatentCfg<kLatent>;
  auto kern = latent_kernel<kLatent>;
  static PerDeviceOnce once;
  if (const int rc = set_dynamic_smem_once(once, kern, C::kSmem); rc != PQ_OK) return rc;
  CUtensorMap mq = {}, mc = {}, mr = {};
  const uint64_t wide = kLatent + PQ_LATENT_ROPE, rows = static_cast<uint64_t>(a.c.pages) * a.c.page;
  if (const int rc = make_tmap_2d(&mq, q, static_cast<uint64_t>(a.tokens) * a.heads, wide, kRows, 64, 2, 128); rc != PQ_OK) return rc;
  // values of a panel, rows of 8, panels, groups of 8 rows
  const uint64_t dims[4] = {64, 8, static_cast<uint64_t>(C::kPanels), rows / 8}, strides[3] = {wide * 2, 128, wide * 16};
  const uint32_t box[4] = {64, 8, 4, static_cast<uint32_t>(a.box / 8)}, rope_box[4] = {64, 8, 1, static_cast<uint32_t>(a.box / 8)};
  if (const int rc = make_tmap_f16(&mc, a.c.data, 4, dims, strides, box); rc != PQ_OK) return rc;
  if (const int rc = make_tmap_f16(&mr, a.c.data, 4, dims, strides, rope_box); rc != PQ_OK) return rc;
  const unsigned grid = static_cast<unsigned>(a.paired ? sms & ~1 : sms);
  if (const int rc = launch_dependent(kern, dim3(grid), dim3(kThreads), C::kSmem, stream, mq, mc, mr, a); rc != PQ_OK || !a.partials) return rc;
  const int64_t units = a.tokens * a.heads / (a.paired ? 2 * kRows : kRows) + a.requests;
  return many_parts(units, static_cast<int>(grid), a.width * a.c.page / kKeys, kLeastSteps) ? launch_dependent(latent_join_kernel<kLatent, kJoinGroups>, dim3(grid, kLatent / 16), dim3(kJoinThreads), 0, stream, a)
                           : launch_dependent(latent_join_kernel<kLatent, 1>, dim3(grid, kLatent / 64), dim3(kJoinThreads), 0, stream, a);
}

}  // namespace
}  // namespace pq

using namespace pq;

extern "C" {

int pq_latent_attention(const void* q_f16, int32_t heads, const pq_latent_cache* cache, const int32_t* block_table, int64_t width,
                        const int32_t* q_start, const int32_t* kv_len, int64_t requests, int64_t tokens, float scale, void* out_f16,
                        void* workspace, size_t workspace_bytes, void* stream) {
  int rc = check_latent_cache(cache);
  if (rc != PQ_OK) return rc;
  if (heads < 1 || heads > 1024 || requests < 0 || requests > 0x7fffffff || tokens < 0 || tokens > 0x7fffffff / heads) return PQ_ERR_SHAPE;
  if (width < 1 || width > 0x7fffffff || !std::isfinite(scale)) return PQ_ERR_SHAPE;
  if (requests > PQ_MAX_REQUESTS || width > kMostKeys / cache->page) return PQ_ERR_LIMIT;
  if (requests == 0 || tokens == 0) return PQ_OK;
  if (!q_f16 || !block_table || !q_start || !kv_len || !out_f16) return PQ_ERR_NULL;
  if (!aligned16(q_f16) || !aligned16(out_f16) || !aligned256(workspace)) return PQ_ERR_ALIGN;
  if ((rc = check_arch()) != PQ_OK) return rc;
  LatentArgs a{*cache, block_table, width, q_start, kv_len, static_cast<__half*>(out_f16), tokens, static_cast<int>(requests), heads,
               0, scale * 1.44269504f, 0xffffffffu, 0u, nullptr, nullptr, kKeys, device_status_ptr(), wait_limit()};
  if (a.status == nullptr) return PQ_ERR_CUDA;
  while (cache->page % a.box != 0) a.box /= 2;   // the page is a multiple of 16
  if (a.scale_log2 == 0.0f) {
    a.q_and = 0u, a.scale_log2 = 1.0f;
  } else if (a.scale_log2 < 0.0f) {
    a.q_xor = 0x80000000u, a.scale_log2 = -a.scale_log2;
  }
  a.paired = static_cast<int64_t>(tokens) * heads > kRows * requests;   // more than 64 rows a request, on average
  const int sms = sm_count();
  const Scratch sc = scratch_from(workspace, workspace_bytes);
  // (Where the table holds so few tokens, whole units are done sooner than the parts' joining.)
  if (width * cache->page > kFewSteps * kKeys && sc.partials != nullptr && sc.partial_bytes >= partial_bytes(cache->latent, sms)) {
    a.partials = reinterpret_cast<float*>(sc.partials);
    a.joins = reinterpret_cast<int4*>(a.partials + static_cast<size_t>(sms) * 2 * kRows * (cache->latent + 2));
  }
  return cache->latent == 512 ? launch<512>(a, q_f16, sms, static_cast<cudaStream_t>(stream)) : launch<256>(a, q_f16, sms, static_cast<cudaStream_t>(stream));
}

size_t pq_latent_workspace_bytes(int32_t sms) {
  if (sms < 1) return 0;
  const size_t absorbed = partial_bytes(512, sms), expanded = expanded_partial_bytes(sms);
  return kScratchHeaderBytes + (absorbed > expanded ? absorbed : expanded);
}

}  // extern "C"

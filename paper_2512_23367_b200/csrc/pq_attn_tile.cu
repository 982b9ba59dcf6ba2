// Attention of more than 16 query rows per (request, key/value head) over the paged cache, on the tcgen05 tensor
// cores: prompts, chunks of prompts and wide drafts.
#include "pq_attention.h"
#include "pq_attn_mma.cuh"
#include "pq_ptx.cuh"

namespace pq {

namespace {

constexpr int kTile = 128;          // query rows of one accumulator, keys of one step
constexpr int kSoft = 512;          // threads of the four softmax warpgroups, two per accumulator
constexpr int kIssuer = 16, kLoadK = 17, kWatcher = 18, kLoadV = 19;   // warps; from 20 on the INT8 converters

template <bool kInt8, int D>
struct TileCfg {
  static constexpr int kConv = kInt8 ? 256 : 0;                // converter threads
  static constexpr int kThreads = 640 + kConv;
  // Registers: softmax, issuer's warpgroup, converters.  512 x 104 + 128 x 64 = 640 x 96 and
  // 512 x 96 + 128 x 40 + 256 x 40 = 896 x 72, what the launch holds.  With 88 and 56
  // for INT8 six chunks of up to 700 over up to 5000 took 217 us in place of 211.
  static constexpr int kSoftRegs = kInt8 ? 96 : 104, kRestRegs = kInt8 ? 40 : 64, kConvRegs = 40;
  static constexpr int kRegsNeeded = kSoft * kSoftRegs + 128 * kRestRegs + kConv * kConvRegs;
  static constexpr int kTileBytes = kTile * D * 2;            // one operand tile: D / 64 panels of 128 rows x 128 B
  static constexpr int kPanel = kTile * 128;
  static constexpr int kStages = (kInt8 ? 131072 : 163840) / kTileBytes;   // keys and values alternate
  // INT8: scales of a tile (keys'; values' over their units; log2 of the values'; the units, of 32 keys each; the largest of
  // the keys'), and 128 ones.
  static constexpr int kScaleTiles = kInt8 ? kStages / 2 + 1 : 0;
  static constexpr int kScaleFloats = 3 * kTile + 8;
  static constexpr int kBars = 2 * kStages + 7 + kScaleTiles;
  static constexpr int kSmem = (2 + kStages) * kTileBytes + kScaleTiles * kScaleFloats * 4 + (kInt8 ? 4 * kTile : 0) +
                               6 * 16 * kConv /* the converters' slots */ + 1024 /* alignment */;
};

// Named barriers (0 is __syncthreads): the softmax warpgroups among themselves; "P written", one per accumulator
// (256 threads arrive, the issuer's warp waits); "operand tile landed", between the watcher's and the issuer's warp;
// the two warps that share 32 rows, eight pairs; "S read", 256 threads of an accumulator to the issuer, one each;
// "tensor memory read", all softmax threads to the issuer, at the end.
// They do not pass through shared memory, which the tensor core keeps busy: a wait on an mbarrier that has long
// completed takes 200 to 400 cycles here, one on a named barrier about 30.
constexpr uint32_t kBarSoft = 1, kBarP = 2, kBarTile = 4, kBarPair = 5, kBarRead = 13, kBarFree = 15;
// Blocks of 16 keys of one request, a lane each, so that one look-up serves four key tiles: the index of the block's first
// cache vector, or -1 where there is nothing to read.  The page ids of the next 32 blocks are on the way meanwhile.
struct BlockWalk {
  const int* trow;
  int64_t key, pages;
  int hi, lo, page16, col, off, step_col, step_off, heads, hk, id;
  __device__ __forceinline__ BlockWalk(const AttnArgs& a, const AttnRange& rg, int b, int head, int key_base, int lane)
      : trow(a.table + static_cast<int64_t>(b) * a.width), key(key_base + 16 * lane), pages(a.c.pages), hi(rg.hi), lo(rg.lo),
        page16(a.c.page >> 4), heads(a.c.heads), hk(head) {
    const int block = (key_base >> 4) + lane;
    col = block / page16, off = block - col * page16;
    step_col = 32 / page16, step_off = 32 - step_col * page16;
    fetch();
  }
  __device__ __forceinline__ void fetch() { id = key < hi && key + 16 > lo ? trow[col] : -1; }
  __device__ __forceinline__ int next() {
    const int v = id < 0 || id >= pages ? -1 : static_cast<int>(((static_cast<int64_t>(id) * heads + hk) * page16 + off) * 16);
    key += 4 * kTile;
    col += step_col, off += step_off;
    if (off >= page16) off -= page16, ++col;
    fetch();
    return v;
  }
};

struct TileArgs {
  AttnArgs a;
  int* status;
  uint32_t wait_limit;
  int box;               // rows of a TMA box: the largest power of two that divides both the page and 128
  uint32_t group_mul;    // i / group = i * group_mul >> 16 for i up to 256
  int whole, split, parts;   // as planned: CTAs of whole units, then part 0 of the others, part 1, ...
  uint32_t q_and, q_xor; // a scale of 0 or below is folded into the queries: (q & q_and) ^ q_xor
};

// Which request and which of its tiles of `qt` tokens: the slot-th over all requests that this kernel serves (a request's
// last tile, which sees most keys, comes first).  found: request (-1: there are fewer), tile, first row, rows, cached
// tokens.  By the whole block; sums: one word per warp.
template <int kThreads>
__device__ __forceinline__ void find_slot(const AttnArgs& a, int slot, int qt, volatile int* found, volatile int* sums) {
  const int tid = threadIdx.x, warp = tid >> 5, lane = tid & 31;
  if (tid == 0) found[0] = -1;
  int before = 0;
  for (int base = 0; base < a.requests; base += kThreads) {
    const int b = base + tid;
    int cnt = 0, n = 0, q0 = 0, L = 0;
    if (b < a.requests) {
      q0 = a.q_start[b];
      n = a.q_start[b + 1] - q0;
      L = a.kv_len[b];
      if (n > a.row_tokens) cnt = (n - 1) / qt + 1;   // the others are the row kernel's
    }
    const int in = warp_prefix(cnt, lane);
    if (lane == 31) sums[warp] = in;
    __syncthreads();
    const int of_warp = lane < kThreads / 32 ? sums[lane] : 0, to_warp = warp_prefix(of_warp, lane);
    const int off = before + __shfl_sync(0xffffffffu, to_warp - of_warp, warp);
    before += __shfl_sync(0xffffffffu, to_warp, 31);
    const int mine = slot - (off + in - cnt);
    if (mine >= 0 && mine < cnt) found[0] = b, found[1] = cnt - 1 - mine, found[2] = q0, found[3] = n, found[4] = L;
    __syncthreads();
    if (slot < before) break;
  }
}

// The keys that a slot's rows see, and their division.
struct SlotKeys {
  int toks, p_base;        // tokens; position of the first
  int k_lo, tiles;         // first key (a multiple of 128), key tiles
  int per, parts;          // tiles of a part
};
__device__ __forceinline__ SlotKeys slot_keys(const AttnArgs& a, const AttnRange& rg, int tok0, int qt, int most_parts) {
  SlotKeys s;
  s.toks = min(qt, rg.n - tok0);
  s.p_base = rg.L - rg.n + tok0;
  const int k_hi = min(rg.hi, s.p_base + s.toks);
  s.k_lo = first_key(s.p_base, a.window) & ~(kTile - 1);
  s.tiles = k_hi > s.k_lo ? (k_hi - s.k_lo + kTile - 1) / kTile : 0;
  s.per = a.part_keys / kTile;
  s.parts = most_parts == 1 ? 1 : max(1, min(most_parts, (s.tiles + s.per - 1) / s.per));
  return s;
}

// Floats of one part: per query tile [D / 4][128 rows] x 4 sums, then [128 rows] x (reference, sum of weights).
template <int D>
constexpr int kPartFloats = 2 * kTile * (D + 2);

// Joins the parts of the units whose keys were split, in their order: grid (unit, 32 rows, 32 features), a warp per 4
// features, lanes along the rows; L2 latency, so one short chain of
// loads per thread.  (One CTA per unit, the last to arrive, took 30 us for 16 parts of 133 KB.)
constexpr int kJoinThreads = 256;
template <int D>
__global__ void __launch_bounds__(kJoinThreads) attn_join_kernel(const AttnArgs a, int whole, int most_parts) {
  __shared__ int s_assign[5];
  __shared__ int s_warp_sum[kJoinThreads / 32];
  grid_dep_launch();
  grid_dep_wait();
  const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
  const int G = a.heads / a.c.heads, tpt = kTile / G, qt = 2 * tpt;
  const int unit = whole + blockIdx.x, slot = unit / a.c.heads, hk = unit - slot * a.c.heads;
  __syncthreads();
  find_slot<kJoinThreads>(a, slot, qt, s_assign, s_warp_sum);
  if (s_assign[0] < 0) return;
  const int tok0 = s_assign[1] * qt;
  const SlotKeys sk = slot_keys(a, attn_range(a, s_assign[3], s_assign[4]), tok0, qt, most_parts);
  const int tile = blockIdx.y / 4, r = (blockIdx.y % 4) * 32 + lane;
  const int tok = tile * tpt + r / G;
  const int64_t row = static_cast<int64_t>(s_assign[2]) + tok0 + tok;
  if (sk.parts == 1 || (tile == 1 && sk.toks <= tpt)) return;
  const bool live = r < tpt * G && tok < sk.toks && row >= 0 && row < a.tokens;
  if (!live) return;   // no barrier follows
  constexpr int kPart = kPartFloats<D>;
  const float* p0 = a.partials + static_cast<int64_t>(blockIdx.x) * most_parts * kPart + tile * kTile * (D + 2);
  const int f4 = blockIdx.z * (kJoinThreads / 32) + warp;   // of 4 features each
  float M = -INFINITY, L = 0.0f;
  float4 v = make_float4(0.0f, 0.0f, 0.0f, 0.0f);
  constexpr int kBatch = 8;   // parts whose loads are in flight together
  for (int q0 = 0; q0 < sk.parts; q0 += kBatch) {
    float2 ml[kBatch];   // reference, sum of weights
    float4 x[kBatch];
#pragma unroll
    for (int j = 0; j < kBatch; ++j) {
      const float* pq = p0 + static_cast<int64_t>(min(q0 + j, sk.parts - 1)) * kPart;
      ml[j] = __ldcg(reinterpret_cast<const float2*>(pq + kTile * D) + r);
      x[j] = __ldcg(reinterpret_cast<const float4*>(pq) + f4 * kTile + r);
    }
    float top = M;
#pragma unroll
    for (int j = 0; j < kBatch; ++j) top = fmaxf(top, ml[j].x);
    const float ref = top == -INFINITY ? 0.0f : top, f = exp2_approx(M - ref);
    M = top;
    L *= f, v.x *= f, v.y *= f, v.z *= f, v.w *= f;
#pragma unroll
    for (int j = 0; j < kBatch; ++j) {
      const float w = q0 + j < sk.parts ? exp2_approx(ml[j].x - ref) : 0.0f;
      L = fmaf(ml[j].y, w, L);
      v.x = fmaf(x[j].x, w, v.x), v.y = fmaf(x[j].y, w, v.y), v.z = fmaf(x[j].z, w, v.z), v.w = fmaf(x[j].w, w, v.w);
    }
  }
  const float inv = L > 0.0f ? 1.0f / L : 0.0f;
  v.x *= inv, v.y *= inv, v.z *= inv, v.w *= inv;
  *reinterpret_cast<uint2*>(a.out + (row * a.heads + hk * G + r % G) * D + 4 * f4) = make_uint2(pack_f16(v.x, v.y), pack_f16(v.z, v.w));
}

// Tensor bound for long chunks, HBM bound for wide drafts over long caches.
//
// A CTA owns 256 query rows of one key/value head (row = token x query heads of the group) as two accumulators of
// 128, or up to 128 rows as two accumulators that take the even and the odd key tiles and are joined at the end:
// either way one accumulator's softmax runs while the tensor core works for the other.  Per 128 keys and accumulator:
//   S = Q K^T            8 (D / 16) MMAs from shared memory into tensor memory
//   softmax              two threads per row: S to registers, running maximum, P = 2^(S - max + 7) as FP16
//   O += P V             8 MMAs with P from tensor memory, V as it lies in the cache (features contiguous)
// The reference that is subtracted is only moved (and O rescaled, in tensor memory) when the maximum has grown by
// more than 2^8: O is almost never touched, P stays below 2^15, and FP16 keeps its bits down to 2^-21 of the maximum and
// counts it down to 2^-31.
// Tensor memory (512 columns): S, shared by the accumulators in turn, 128; P of each, 64; O of each, 64 or 128.  S is
// free as soon as the softmax threads hold it in registers, so that QK(u + 1) runs under the softmax of u; MMA order
// QK(u), PV(u - 2), u counting the accumulators in turn.  With P over S and one S per accumulator the chain
// QK -> softmax -> PV of an accumulator set the pace: 3240 cycles per 256 x 128 scores; now about 2700, where the MMAs take
// 2048 and so do the exponentials (16 per cycle and SM).  Computing some of them by a polynomial gained nothing: the
// softmax warps' issue slots are the scarcer.
//
// Measured, 32 heads over 8 of 128, FP16: a prompt of 4096 125 us (1.10 PFLOP/s); 2048 tokens over 16384, 545 us in a
// row (1.08 PFLOP/s, SMs at 1.62 GHz under the power cap), 461 in a short burst (1.27).  A unit takes 9 us beyond its
// steps: requests' lengths, page ids, queries and first keys come one after the other out of global memory (8700 cycles up
// to the first S), the results go back (4000), the next CTA starts (1300).
// Keys and values come through TMA boxes of whole page pieces (one lane looks up and requests one box); boxes that
// no visible key needs, or of an unusable page id, are requested beyond the tensor and arrive as zeros.
// Value rows that were never written (beyond the request's length, before its window) are zeroed in shared memory:
// their weight is 0, but 0 x NaN is not.
//
// INT8: two warpgroups of converters take the place of the TMA producers.  A thread keeps six asynchronous copies of
// 16 codes in flight into slots of its own, turns the codes into FP16 (exact) and stores them in the layout that TMA
// would have left.  (Copies into registers cost spills: 4000 cycles per operand tile.)  The
// key's scale (times the softmax scale) multiplies the score.  The value's scale multiplies the weight before it is
// rounded: the power of two above the largest scale of its 32 keys goes into the exponent, the quotient of the two
// multiplies.  The reference is the largest product of weight and value scale, up to 2^8, over the keys that the row
// sees (a key that it does not see moves nothing), and FP16 weights keep their bits down to 2^-21 of that at least.
// Six requests, chunks of up to 700 over up to 5000: 211 us (0.67 PFLOP/s), FP16 158; issue, 70 % of the slots: the
// conversion is done again for every 256 rows, and each score takes two products more.
template <bool kInt8, int D>
__global__ void __launch_bounds__((TileCfg<kInt8, D>::kThreads), 1)
attn_tile_kernel(const __grid_constant__ CUtensorMap map_k, const __grid_constant__ CUtensorMap map_v, const TileArgs ta) {
  using C = TileCfg<kInt8, D>;
  constexpr int kThreads = C::kThreads;
  constexpr int KS = D / 16;        // MMAs of one QK
  constexpr int PS = kTile / 16;    // MMAs of one PV
  constexpr float kTop = 7.0f;      // a weight at the reference is 2^kTop
  extern __shared__ uint8_t smem_raw[];
  __shared__ __align__(8) uint64_t bars[C::kBars];
  __shared__ uint32_t s_tmem;
  __shared__ volatile int s_abort;
  __shared__ int s_assign[5];           // request, tile; its first row, rows and cached tokens
  __shared__ int s_warp_sum[kThreads / 32];
  __shared__ __align__(16) float s_swap[2 * kTile];   // one word between the two threads of a row; a pair per row in the join

  const AttnArgs& a = ta.a;
  const int tid = threadIdx.x, warp = __shfl_sync(0xffffffffu, tid >> 5, 0), lane = tid & 31;
  const int G = a.heads / a.c.heads;
  auto by_group = [&](int i) { return static_cast<int>(static_cast<uint32_t>(i) * ta.group_mul >> 16); };
  const int tpt = by_group(kTile);    // tokens of one accumulator
  const int qt = 2 * tpt;             // tokens of one CTA
  int unit = blockIdx.x, part = 0;
  const int most_parts = unit < ta.whole ? 1 : ta.parts;
  if (unit >= ta.whole) part = (unit - ta.whole) / ta.split, unit -= part * ta.split;
  const int slot = unit / a.c.heads, hk = unit - slot * a.c.heads;

  const uint32_t bar0 = smem_u32(bars);
  const uint32_t bar_full = bar0, bar_free = bar0 + 8 * C::kStages;
  const uint32_t bar_s = bar0 + 16 * C::kStages, bar_o = bar_s + 16;   // two of each
  const uint32_t bar_q = bar_o + 16, bar_fix = bar_q + 8, bar_drain = bar_fix + 8, bar_scale = bar_drain + 8;
  if (kInt8 && tid < kTile) {   // the scales of scores that have been multiplied already
    const uint32_t at = ((smem_u32(smem_raw) + 1023u) & ~1023u) + (2 + C::kStages) * C::kTileBytes + C::kScaleTiles * C::kScaleFloats * 4;
    asm volatile("st.shared.f32 [%0], %1;" ::"r"(at + 4 * tid), "f"(1.0f) : "memory");
  }
  if (tid == 0) {
    for (int i = 0; i < C::kStages; ++i) mbar_init(bar_full + 8 * i, kInt8 ? C::kConv / 32 + (i & 1 ? 0 : 2) : 1), mbar_init(bar_free + 8 * i, 1);
    for (int i = 0; i < 2; ++i) mbar_init(bar_s + 8 * i, 1), mbar_init(bar_o + 8 * i, 1);
    mbar_init(bar_q, kSoft / 32);
    mbar_init(bar_fix, 1);
    mbar_init(bar_drain, 1);
    for (int i = 0; i < C::kScaleTiles; ++i) mbar_init(bar_scale + 8 * i, 1);
    fence_mbar_init();
    s_abort = 0;
    if (!kInt8) tma_prefetch_desc(&map_k), tma_prefetch_desc(&map_v);
  }
  // (All CTAs of the launch before hold their tensor memory by now, or have given it back: they let this one begin.)
  if (warp == kIssuer) {
    tmem_alloc(smem_u32(&s_tmem), 512);
    tmem_relinquish();
  }
  tc_fence_before_sync();
  grid_dep_wait();
  find_slot<kThreads>(a, slot, qt, s_assign, s_warp_sum);   // at least two barriers of the block
  tc_fence_after_sync();
  grid_dep_launch();   // only now: a later launch's CTA may take this SM's tensor memory when it is given back
  const uint32_t tmem = __shfl_sync(0xffffffffu, s_tmem, 0);

  const int b = s_assign[0];
  const int tok0 = s_assign[1] * qt;
  const AttnRange rg = attn_range(a, s_assign[3], s_assign[4]);
  const int64_t row0 = s_assign[2];
  const SlotKeys sk = slot_keys(a, rg, tok0, qt, most_parts);
  const int toks = sk.toks, p_base = sk.p_base, parts = sk.parts;
  const bool two = toks > tpt;
  if (b < 0 || part >= parts) {
    if (warp == kIssuer) tmem_dealloc(tmem, 512);
    return;
  }
  const int t0 = part * sk.per;
  const int n_tiles = part == parts - 1 ? sk.tiles - t0 : sk.per;   // key tiles of this CTA
  const int key_base = sk.k_lo + t0 * kTile;
  const int N = two ? 2 * n_tiles : n_tiles;                      // (QK, PV) steps
  // Steps that a PV follows its QK by: with two query tiles S(u + 1) is computed while the softmax of u runs; with
  // one, where memory is the bound, operand tiles are given back a step earlier instead.
  const int lag = two ? 2 : 1;

  const uint32_t base = (smem_u32(smem_raw) + 1023u) & ~1023u;
  const uint32_t sq = base, ring = base + 2 * C::kTileBytes, scales = ring + C::kStages * C::kTileBytes;
  const WaitCtx wc{&s_abort, ta.wait_limit};
  int issued = 0;           // producers: tiles requested so far
  uint32_t fix_phase = 0;   // the values' producer: tiles that came by bar_fix and have landed

  if (kInt8 && warp >= 20) {
    // -------------------------------------------------------------------- INT8 converters
    asm volatile("setmaxnreg.dec.sync.aligned.u32 %0;" ::"n"(C::kConvRegs));
    if constexpr (kInt8) {
      constexpr int kRow = D / 16;                      // 16-byte pieces of one key
      constexpr int kItems = kTile * kRow / C::kConv;     // of a thread per tile: 4 or 2
      const int c = tid - 20 * 32;
      constexpr int kStep = C::kConv / kRow;
      const int piece = c % kRow, row_in = c / kRow;    // item k: row k * kStep + row_in
      BlockWalk walk(a, rg, b, hk, key_base, lane);
      int vec = walk.next(), vec4 = -1;   // of the four tiles that t is one of, and of the next four
      // Work goes in batches of two items; the batch three further on is copied into the slots that one leaves (the
      // thread's own: no other thread reads them), or zeros.
      constexpr int kBatches = kItems / 2;              // per operand tile
      const uint32_t raw = scales + C::kScaleTiles * C::kScaleFloats * 4 + 4 * kTile + c * 16;
      auto request = [&](int n, int t) {                // batch n of all, while tile t is in work
        const int i = n / kBatches, v = (i >> 3) == (t >> 2) ? vec : vec4;
        if (i < 2 * n_tiles) {
#pragma unroll
          for (int q = 0; q < 2; ++q) {
            const int r = ((n % kBatches) * 2 + q) * kStep + row_in;
            const int first = __shfl_sync(0xffffffffu, v, 8 * ((i >> 1) & 3) + (r >> 4));
            const uint4* src = static_cast<const uint4*>((i & 1) ? a.c.v : a.c.k) + (static_cast<int64_t>(max(first, 0)) + (r & 15)) * kRow + piece;
            asm volatile("cp.async.cg.shared.global [%0], [%1], 16, %2;" ::"r"(raw + ((n % 3) * 2 + q) * (16 * C::kConv)), "l"(src), "r"(first < 0 ? 0 : 16) : "memory");
          }
        }
        asm volatile("cp.async.commit_group;" ::: "memory");
      };
#pragma unroll
      for (int n = 0; n < 3; ++n) request(n, 0);
      bool ok = true, free_next = false;
      for (int i = 0; i < 2 * n_tiles; ++i) {
        const int st = i % C::kStages, t = i >> 1;
        const bool is_v = i & 1;
        if (i >= C::kStages && !free_next) ok = ok && warp_wait(bar_free + 8 * st, ((i / C::kStages) & 1) ^ 1, wc);
        // asked a tile ahead: a wait that succeeds at once takes about 300 cycles
        const int i1 = i + 1, st1 = i1 % C::kStages;
        const uint32_t asked = i1 < C::kStages ? 1u : mbar_test2(bar_free + 8 * st1, ((i1 / C::kStages) & 1) ^ 1, bar_free + 8 * st1, ((i1 / C::kStages) & 1) ^ 1);
        const uint32_t dst = ring + st * C::kTileBytes;
#pragma unroll
        for (int j = 0; j < kBatches; ++j) {
          const int n = i * kBatches + j;
          asm volatile("cp.async.wait_group 2;" ::: "memory");
          uint32_t u[2][4];
#pragma unroll
          for (int q = 0; q < 2; ++q)
            asm volatile("ld.shared.v4.u32 {%0, %1, %2, %3}, [%4];" : "=r"(u[q][0]), "=r"(u[q][1]), "=r"(u[q][2]), "=r"(u[q][3])
                         : "r"(raw + ((n % 3) * 2 + q) * (16 * C::kConv)) : "memory");
#pragma unroll
          for (int q = 0; q < 2; ++q) {
            const int r = (2 * j + q) * kStep + row_in;
            // 16 codes are two 16-byte pieces of the FP16 row; half of the threads store the second one first, so that
            // eight neighbours hit all banks
#pragma unroll
            for (int h = 0; h < 2; ++h) {
              const int second = h ^ ((piece >> 2) & 1);
              const uint32_t w0 = (second ? u[q][2] : u[q][0]) ^ 0x80808080u, w1 = (second ? u[q][3] : u[q][1]) ^ 0x80808080u;
              const int ch = 2 * piece + second;
              asm volatile("st.shared.v4.u32 [%0], {%1, %2, %3, %4};" ::"r"(dst + (ch >> 3) * C::kPanel + r * 128 + (((ch & 7) ^ (r & 7)) << 4)),
                           "r"(codes_f16(w0, 0x4140)), "r"(codes_f16(w0, 0x4342)), "r"(codes_f16(w1, 0x4140)), "r"(codes_f16(w1, 0x4342)) : "memory");
            }
          }
          request(n + 3, t);   // two tiles ahead at most
        }
        if (is_v && (t & 3) == 1) vec4 = walk.next();
        if (is_v && (t & 3) == 3) vec = vec4;
        free_next = __all_sync(0xffffffffu, asked);
        fence_proxy_async_smem();
        __syncwarp();
        if (lane == 0) mbar_arrive(bar_full + 8 * st);
      }
    }
  } else if (warp >= kSoft / 32) {
    asm volatile("setmaxnreg.dec.sync.aligned.u32 %0;" ::"n"(C::kRestRegs));
    if (!kInt8 && (warp == kLoadK || warp == kLoadV)) {
      // ------------------------------------------------------------------ producers, one for keys and one for values
      // A lane requests one box; its page id is looked up a tile ahead.
      const bool is_v = warp == kLoadV;
      const int boxes = kTile / ta.box;
      constexpr int halves = D / 64;
      const int x = lane / boxes, y = lane - x * boxes;
      const bool mine = lane < boxes * halves;
      const int rows_all = static_cast<int>(a.c.pages * a.c.heads * a.c.page);
      const int* trow = a.table + static_cast<int64_t>(b) * a.width;
      int id = -1, off = 0;        // page of the box and the place in it
      auto look_up = [&](int t) {
        const int key = key_base + t * kTile + y * ta.box;
        id = -1;
        if (!mine || t >= n_tiles || key >= rg.hi || key + ta.box <= rg.lo) return;
        const int col = key / a.c.page;
        off = key - col * a.c.page;
        id = trow[col];
      };
      look_up(0);
      for (int t = 0; t < n_tiles; ++t) {
        const int i = 2 * t + is_v, st = i % C::kStages;
        // row of the tensor map; rows_all lies beyond the tensor: zeros
        const int row = id < 0 || id >= a.c.pages ? rows_all : static_cast<int>((static_cast<int64_t>(id) * a.c.heads + hk) * a.c.page) + off;
        if (i >= C::kStages && !warp_wait(bar_free + 8 * st, ((i / C::kStages) & 1) ^ 1, wc)) break;
        const int key0 = key_base + t * kTile;
        // rows of the tile that were never written: before the request's window, beyond its length
        const int dead_lo = min(max(rg.lo - key0, 0), kTile), dead_hi = min(max(rg.L - key0, 0), kTile);
        const bool fix = is_v && (dead_lo > 0 || dead_hi < kTile);
        const uint32_t dst = ring + st * C::kTileBytes, bar = fix ? bar_fix : bar_full + 8 * st;
        if (lane == 0) mbar_arrive_expect_tx(bar, C::kTileBytes);
        __syncwarp();
        if (mine) tma_load_2d(dst + x * C::kPanel + y * ta.box * 128, is_v ? &map_v : &map_k, bar, x * 64, row);
        look_up(t + 1);   // used, and so waited for, in the next round
        issued = t + 1;
        if (fix) {
          if (!warp_wait(bar_fix, fix_phase & 1, wc)) break;
          ++fix_phase;
          const int dead = dead_lo + (kTile - dead_hi);
          for (int j = lane; j < dead * halves * 8; j += 32) {
            const int chunk = j & 7, xx = (j >> 3) % halves, r = (j >> 3) / halves;
            const int rr = r < dead_lo ? r : dead_hi + r - dead_lo;
            asm volatile("st.shared.v4.u32 [%0], {%1, %1, %1, %1};" ::"r"(dst + xx * C::kPanel + rr * 128 + chunk * 16), "r"(0) : "memory");
          }
          fence_proxy_async_smem();
          __syncwarp();
          if (lane == 0) mbar_arrive(bar_full + 8 * st);
        }
        __syncwarp();
      }
    } else if (kInt8 && (warp == kLoadK || warp == kLoadV)) {
      // ------------------------------------------------------------------ INT8: a tile's scales, four keys per lane
      if constexpr (kInt8) {
        const bool is_v = warp == kLoadV;
        const float* from = is_v ? a.c.v_scale : a.c.k_scale;
        BlockWalk walk(a, rg, b, hk, key_base, lane);
        int vec = -1;
        auto load = [&](int t) {
          if ((t & 3) == 0) vec = walk.next();
          const int v = __shfl_sync(0xffffffffu, vec, 8 * (t & 3) + (lane >> 2));
          return v < 0 ? make_float4(0.0f, 0.0f, 0.0f, 0.0f) : __ldg(reinterpret_cast<const float4*>(from + v) + (lane & 3));
        };
        float4 next = load(0);
        bool ok = true;
        for (int t = 0; t < n_tiles; ++t) {
          float4 s = next;
          next = load(t + 1);
          const int key = key_base + t * kTile + 4 * lane;   // 0 where nothing was written
          s.x = key >= rg.lo && key < rg.hi ? s.x : 0.0f, s.y = key + 1 >= rg.lo && key + 1 < rg.hi ? s.y : 0.0f;
          s.z = key + 2 >= rg.lo && key + 2 < rg.hi ? s.z : 0.0f, s.w = key + 3 >= rg.lo && key + 3 < rg.hi ? s.w : 0.0f;
          float factor = a.scale_log2, unit = 0.0f;
          if (is_v) {   // relative to the unit of 32 keys
            float top = fmaxf(fmaxf(s.x, s.y), fmaxf(s.z, s.w));
#pragma unroll
            for (int o = 1; o < 8; o <<= 1) top = fmaxf(top, __shfl_xor_sync(0xffffffffu, top, o));
            unit = scale_unit(top);
            factor = __uint_as_float(0x7f000000u - __float_as_uint(unit));   // 1 / unit, a power of two
          }
          // The keys' stage has to be free as for the converters (an arrival ahead of time would count for the tile that
          // is still being written there), and the product with the weights of the tile that was in the slot taken.
          const int i = 2 * t;
          if (i >= C::kStages) ok = ok && warp_wait(bar_free + 8 * (i % C::kStages), ((i / C::kStages) & 1) ^ 1, wc);
          if (t >= C::kScaleTiles) ok = ok && warp_wait(bar_scale + 8 * (t % C::kScaleTiles), ((t / C::kScaleTiles) & 1) ^ 1, wc);
          const uint32_t s0 = scales + (t % C::kScaleTiles) * (C::kScaleFloats * 4) + (is_v ? 4 * kTile : 0);
          asm volatile("st.shared.v4.f32 [%0], {%1, %2, %3, %4};" ::"r"(s0 + 16 * lane), "f"(s.x * factor), "f"(s.y * factor), "f"(s.z * factor), "f"(s.w * factor) : "memory");
          if (!is_v) {
            float top = fmaxf(fmaxf(s.x, s.y), fmaxf(s.z, s.w)) * factor;
#pragma unroll
            for (int o = 1; o < 32; o <<= 1) top = fmaxf(top, __shfl_xor_sync(0xffffffffu, top, o));
            if (lane == 0) asm volatile("st.shared.f32 [%0], %1;" ::"r"(s0 + 4 * (3 * kTile + 4)), "f"(top) : "memory");
          }
          if (is_v) {   // s0: of the values' scales
            const float4 g = make_float4(scale_log(s.x), scale_log(s.y), scale_log(s.z), scale_log(s.w));
            asm volatile("st.shared.v4.f32 [%0], {%1, %2, %3, %4};" ::"r"(s0 + 4 * kTile + 16 * lane), "f"(g.x), "f"(g.y), "f"(g.z), "f"(g.w) : "memory");
            if ((lane & 7) == 0) asm volatile("st.shared.f32 [%0], %1;" ::"r"(s0 + 8 * kTile + (lane >> 1)), "f"(unit) : "memory");
          }
          __syncwarp();
          if (lane == 0) mbar_arrive(bar_full + 8 * ((2 * t) % C::kStages));
        }
      }
    } else if (warp == kIssuer) {
      // ------------------------------------------------------------------ MMA issuer
      // The whole warp walks the steps, so that every operand is uniform; one elected thread issues.  After the watcher has
      // given up the steps go on, so that the barriers stay in step, without MMAs: a stage must not be given back while
      // its load is still on the way.
      bool live = true;
      constexpr uint32_t id_qk = umma_idesc_f16(kTile, false), id_pv = umma_idesc_f16(D, true);
      constexpr uint32_t kStageUnits = C::kTileBytes / 16;
      const uint32_t leader = elect_one();
      const uint32_t q_lo = desc_k(sq), k_lo0 = desc_k(ring), v_lo0 = desc_mn(ring, C::kPanel);
      const uint32_t q_step = two ? kStageUnits : 0;
      warp_wait(bar_q, 0, wc);
      for (int u = 0; u < N + lag; ++u) {
        if (u > 0 && u <= N) named_bar_sync(kBarRead + ((u - 1) & 1), 288);   // S(u - 1) is in registers
        if (u < N) {   // S(u) = Q K^T
          const int acc = u & 1, st = (2 * (two ? u >> 1 : u)) % C::kStages;
          if (!two || acc == 0) live = tile_landed(kBarTile, true) && live;
          tc_fence_after_sync();
          if (leader && live) {
            const uint32_t ql = q_lo + acc * q_step, kl = k_lo0 + st * kStageUnits;
            umma_f16_ss<0>(tmem, ql, kl, id_qk);
#pragma unroll
            for (int k = 1; k < KS; ++k) umma_f16_ss<1>(tmem, ql + (k / 4) * (C::kPanel / 16) + (k % 4) * 2, kl + (k / 4) * (C::kPanel / 16) + (k % 4) * 2, id_qk);
            umma_commit(bar_s + 8 * acc);
            if (!two || acc == 1) umma_commit(bar_free + 8 * st);
          }
          __syncwarp();
        }
        if (u >= lag) {   // O(u - lag) += P V
          const int v = u - lag, acc = v & 1, st = (2 * (two ? v >> 1 : v) + 1) % C::kStages;
          if (!two || acc == 0) live = tile_landed(kBarTile, true) && live;
          named_bar_sync(kBarP + acc, 288);
          tc_fence_after_sync();
          if (leader && live) {
            const uint32_t vl = v_lo0 + st * kStageUnits, d = tmem + 256 + acc * D, p = tmem + 128 + acc * 64;
            umma_f16_ts(d, p, vl, id_pv, (v >> 1) > 0);
#pragma unroll
            for (int k = 1; k < PS; ++k) umma_f16_ts(d, p + 8 * k, vl + k * 128, id_pv, 1u);
            umma_commit(bar_o + 8 * acc);
            if (!two || acc == 1) {
              umma_commit(bar_free + 8 * st);
              if (kInt8) umma_commit(bar_scale + 8 * ((two ? v >> 1 : v) % (kInt8 ? C::kScaleTiles : 1)));
            }
          }
          __syncwarp();
        }
      }
      // Giving tensor memory back takes 2000 cycles: under the results' way to global memory.  MMAs that the softmax
      // threads have not waited for (only after one of them gave up) have to end first.
      named_bar_sync(kBarFree, kSoft + 32);
      tc_fence_after_sync();
      if (s_abort && leader) {
        umma_commit(bar_drain);
        mbar_drain(bar_drain, 0u);
      }
      __syncwarp();
      tmem_dealloc(tmem, 512);
    } else if (warp == kWatcher) {
      // ------------------------------------------------------------------ watcher: waits for the operand tiles a step ahead
      bool ok = true;
      for (int u = 0; u < N + lag; ++u) {
#pragma unroll
        for (int is_v = 0; is_v < 2; ++is_v) {
          const int w = u - is_v * lag;
          if (w < 0 || w >= N || (two && (w & 1))) continue;
          const int i = 2 * (two ? w >> 1 : w) + is_v;
          ok = ok && warp_wait(bar_full + 8 * (i % C::kStages), (i / C::kStages) & 1, wc);
          tile_landed(kBarTile, ok);
        }
      }
    }
  } else {
    // -------------------------------------------------------------------- softmax, two threads per row
    auto release_tmem = [&]() {   // the warp has read its last
      tc_fence_before_sync();
      named_bar_arrive(kBarFree, kSoft + 32);
    };
    asm volatile("setmaxnreg.inc.sync.aligned.u32 %0;" ::"n"(C::kSoftRegs));
    const int acc = warp >> 3;                       // accumulator
    const int half = (warp >> 2) & 1;                // the thread's 64 keys of a tile, and its half of the features
    const int r = tid & 127;                         // row of the tile
    const uint32_t lane_off = static_cast<uint32_t>(warp & 3) << 21;   // 32 lanes per warp, lane in bits 16 and up
    const uint32_t t_sc = tmem + 64 * half + lane_off, t_p = tmem + 128 + 64 * acc + 32 * half + lane_off, t_out = tmem + 256 + acc * D + half * (D / 2) + lane_off;
    float* swap = s_swap + acc * kTile + r;
    const uint32_t pair = kBarPair + acc * 4 + (warp & 3);
    const int q_tile = two ? acc : 0;
    const int tok = q_tile * tpt + by_group(r);      // token of the row, from tok0
    // Where row i of the query tile begins in a matrix of `stride` elements per token: -1 if there is no such row.
    auto row_at = [&](int64_t stride, int i) -> int64_t {
      const int it = by_group(i), k = q_tile * tpt + it;
      const int64_t row = row0 + tok0 + k;
      return it < tpt && k < toks && row >= 0 && row < a.tokens ? row * stride + (hk * G + i - it * G) * D : -1;
    };
    // Rows go between global and shared memory whole, D / 8 lanes side by side (a thread per row instead took 3000
    // cycles at each end): piece c of row i at its swizzled place.  A warp moves 16 rows; a lane works out where one
    // begins and the others ask it.
    constexpr int kLanes = D / 8, kRowsAtOnce = 32 / kLanes;
    auto place = [&](int i, int c) { return sq + q_tile * C::kTileBytes + (c >> 3) * C::kPanel + i * 128 + (((c & 7) ^ (i & 7)) << 4); };

    if (two || acc == 0) {
      const int64_t begin = row_at(a.q_stride, (warp & 7) * 16 + (lane & 15));
      uint4 x[16 / kRowsAtOnce];
#pragma unroll
      for (int i = 0; i < 16 / kRowsAtOnce; ++i) {
        const int64_t p = __shfl_sync(0xffffffffu, begin, i * kRowsAtOnce + lane / kLanes);
        x[i] = p >= 0 ? __ldg(reinterpret_cast<const uint4*>(a.q + p) + lane % kLanes) : make_uint4(0, 0, 0, 0);
      }
#pragma unroll
      for (int i = 0; i < 16 / kRowsAtOnce; ++i) {
        x[i].x = (x[i].x & ta.q_and) ^ ta.q_xor, x[i].y = (x[i].y & ta.q_and) ^ ta.q_xor;
        x[i].z = (x[i].z & ta.q_and) ^ ta.q_xor, x[i].w = (x[i].w & ta.q_and) ^ ta.q_xor;
        asm volatile("st.shared.v4.u32 [%0], {%1, %2, %3, %4};" ::"r"(place((warp & 7) * 16 + i * kRowsAtOnce + lane / kLanes, lane % kLanes)),
                     "r"(x[i].x), "r"(x[i].y), "r"(x[i].z), "r"(x[i].w) : "memory");
      }
      fence_proxy_async_smem();
    }
    __syncwarp();
    if (lane == 0) mbar_arrive(bar_q);

    const int p = p_base + tok;
    const int see_to = min(p, rg.hi - 1) - 64 * half;                        // last key of the row, from the thread's first
    const int see_from = first_key(p, a.window) - 1 - 64 * half;             // keys above it
    const int all_to = min(p_base + q_tile * tpt + 1, rg.hi);                // every row of the tile sees [all_from, all_to)
    const int all_from = first_key(p_base + toks - 1, a.window);
    const int mine = two ? n_tiles : (n_tiles - acc + 1) >> 1;
    const float sc = kInt8 ? 1.0f : a.scale_log2;   // INT8: in the keys' scales
    const float* ones = reinterpret_cast<const float*>(smem_raw + (scales - smem_u32(smem_raw))) + C::kScaleTiles * C::kScaleFloats;
    float m = -INFINITY, l = 0.0f;   // m: the reference that is subtracted, in powers of two; l: the thread's own keys

    bool ok = true;
    for (int i = 0; i < mine; ++i) {
      const int key0 = key_base + (two ? i : 2 * i + acc) * kTile;
      ok = ok && warp_wait(bar_s + 8 * acc, i & 1, wc);
      tc_fence_after_sync();
      uint32_t s[2][32];
      tmem_ld_32x32(t_sc, s[0]);
      tmem_ld_32x32(t_sc + 32, s[1]);
      tmem_ld_wait();
      tc_fence_before_sync();
      hand_over(kBarRead + acc, 288, ok);
      const float* sct = reinterpret_cast<const float*>(smem_raw + (scales - smem_u32(smem_raw))) +
                         (((key0 - key_base) / kTile) % (kInt8 ? C::kScaleTiles : 1)) * C::kScaleFloats;
      const bool edge = key0 < all_from || key0 + kTile > all_to;   // some row does not see all keys
      const float* ksc = sct + 64 * half;   // INT8: what is still to be multiplied to the scores
      int unit_log[2] = {0, 0};             // of the thread's two runs of 32 keys
      if constexpr (kInt8) {
        const float4 u = *reinterpret_cast<const float4*>(sct + 3 * kTile);
        unit_log[0] = static_cast<int>(__float_as_uint(half ? u.z : u.x) >> 23) - 127;
        unit_log[1] = static_cast<int>(__float_as_uint(half ? u.w : u.y) >> 23) - 127;
      }
      float t;
      bool moves;   // the row's reference
      auto largest = [&]() {
        float top[4];
#pragma unroll
        for (int h = 0; h < 4; ++h) {
          const uint32_t* v = s[h >> 1] + 16 * (h & 1);
          top[h] = max3(__uint_as_float(v[0]), __uint_as_float(v[1]), __uint_as_float(v[2]));
#pragma unroll
          for (int j = 3; j < 15; j += 2) top[h] = max3(top[h], __uint_as_float(v[j]), __uint_as_float(v[j + 1]));
          top[h] = fmaxf(top[h], __uint_as_float(v[15]));
        }
        return fmaxf(max3(top[0], top[1], top[2]), top[3]);
      };
      // INT8: no product of weight and value scale exceeds the largest product of codes times the largest key scale, in
      // powers of two, times the larger unit; as long as that does not move the reference, the keys' scales go into the
      // exponents' FMA below (prompt of 4096: 182 us without, 165 with; 2048 over 18432: 755 and 677).
      bool exact = true;
      if constexpr (kInt8) {
        exact = edge || pair_any(pair, !(fmaf(fmaxf(largest(), 0.0f), sct[3 * kTile + 4], static_cast<float>(max(unit_log[0], unit_log[1]))) <= m + 8.0f));
      }
      if (exact) {
        if constexpr (kInt8) {
#pragma unroll
          for (int j = 0; j < 64; j += 4) {
            const float4 k = *reinterpret_cast<const float4*>(ksc + j);
            uint32_t* v = &s[j >> 5][j & 31];
            float x0, x1, x2, x3;
            unpair_f32(mul_f32x2(pair_f32(__uint_as_float(v[0]), __uint_as_float(v[1])), pair_f32(k.x, k.y)), x0, x1);
            unpair_f32(mul_f32x2(pair_f32(__uint_as_float(v[2]), __uint_as_float(v[3])), pair_f32(k.z, k.w)), x2, x3);
            v[0] = __float_as_uint(x0), v[1] = __float_as_uint(x1), v[2] = __float_as_uint(x2), v[3] = __float_as_uint(x3);
          }
          ksc = ones;
        }
        if (edge) {
          const int to = see_to - key0, from = see_from - key0;
#pragma unroll
          for (int h = 0; h < 2; ++h) {
#pragma unroll
            for (int j = 0; j < 32; ++j)
              if (32 * h + j > to || 32 * h + j <= from) s[h][j] = 0xff800000u;   // -inf
          }
        }
        if constexpr (kInt8) {   // of the products of weight and value scale, over the keys that the row sees
          t = -INFINITY;
#pragma unroll
          for (int j = 0; j < 64; j += 4) {
            const float4 v = *reinterpret_cast<const float4*>(sct + 2 * kTile + 64 * half + j);
            const uint32_t* x = &s[j >> 5][j & 31];
            float x0, x1, x2, x3;
            unpair_f32(add_f32x2(pair_f32(v.x, v.y), pair_f32(__uint_as_float(x[0]), __uint_as_float(x[1]))), x0, x1);
            unpair_f32(add_f32x2(pair_f32(v.z, v.w), pair_f32(__uint_as_float(x[2]), __uint_as_float(x[3]))), x2, x3);
            t = max3(max3(t, x0, x1), x2, x3);
          }
        } else {
          t = largest() * sc;
        }
        moves = pair_any(pair, t > m + 8.0f);   // rare after the first tiles: some row of the 32
      } else {
        moves = false, t = 0.0f;
      }
      bool done = i == 0;   // the product with the weights before these has been taken
      if (moves) {
        t = pair_combine<false>(swap, pair, half, t);
        const bool grown = t > m + 8.0f;
        const float f = grown ? (m == -INFINITY ? 0.0f : exp2_approx(m - t)) : 1.0f;
        if (grown) m = t;
        l *= f;
        if (i > 0) {   // O holds the sums up to the tile before
          ok = ok && warp_wait(bar_o + 8 * acc, (i - 1) & 1, wc);
          done = true;
          tc_fence_after_sync();
#pragma unroll 1
          for (int h = 0; h < D / 32; ++h) {
            uint32_t o[16];
            tmem_ld_32x16(t_out + 16 * h, o);
            tmem_ld_wait();
#pragma unroll
            for (int j = 0; j < 16; ++j) o[j] = __float_as_uint(__uint_as_float(o[j]) * f);
            tmem_st_32x16(t_out + 16 * h, o);
          }
        }
      }
      const float ms = m == -INFINITY ? 0.0f : m;
      const uint64_t sc2 = pair_f32(sc, sc);
      uint32_t w[32], asked = 0;
#pragma unroll
      for (int q = 0; q < 2; ++q) {
        const float off = kInt8 ? static_cast<float>(unit_log[q]) + (kTop - ms) : kTop - ms;
        const uint64_t off2 = pair_f32(off, off);
        uint64_t sum = 0;
        float4 vsc = make_float4(0.0f, 0.0f, 0.0f, 0.0f), kf = vsc;
#pragma unroll
        for (int j = 0; j < 16; ++j) {
          if (kInt8 && j % 2 == 0) kf = *reinterpret_cast<const float4*>(ksc + 32 * q + 2 * j);
          const uint64_t x = fma_f32x2(pair_f32(__uint_as_float(s[q][2 * j]), __uint_as_float(s[q][2 * j + 1])),
                                       kInt8 ? (j % 2 == 0 ? pair_f32(kf.x, kf.y) : pair_f32(kf.z, kf.w)) : sc2, off2);
          float e0, e1;
          unpair_f32(x, e0, e1);
          e0 = exp2_approx(e0);
          e1 = exp2_approx(e1);
          sum = add_f32x2(sum, pair_f32(e0, e1));
          if constexpr (kInt8) {
            if (j % 2 == 0) vsc = *reinterpret_cast<const float4*>(sct + kTile + 64 * half + 32 * q + 2 * j);
            unpair_f32(mul_f32x2(pair_f32(e0, e1), j % 2 == 0 ? pair_f32(vsc.x, vsc.y) : pair_f32(vsc.z, vsc.w)), e0, e1);
          }
          w[16 * q + j] = pack_f16(e0, e1);
        }
        if (q == 0) asked = mbar_test2(bar_o + 8 * acc, (i - 1) & 1, bar_o + 8 * acc, (i - 1) & 1);
        float l0, l1;
        unpair_f32(sum, l0, l1);
        l += kInt8 ? (l0 + l1) * power_of_two(-unit_log[q]) : l0 + l1;
      }
      if (!done && !__all_sync(0xffffffffu, asked)) ok = ok && warp_wait(bar_o + 8 * acc, (i - 1) & 1, wc);
      tc_fence_after_sync();
      tmem_st_32x32(t_p, w);
      tmem_st_wait();
      tc_fence_before_sync();
      hand_over(kBarP + acc, 288, ok);
    }
    if (ok && mine > 0) warp_wait(bar_o + 8 * acc, (mine - 1) & 1, wc);
    tc_fence_after_sync();

    // -------------------------------------------------------------------- epilogue: a thread has half of its row's features
    l = pair_combine<true>(swap, pair, half, l);   // the sum of the row's two threads
    // Accumulators of the even and the odd tiles are joined in the first one's threads.
    float f0 = 1.0f, f1 = 0.0f;
    const bool join = !two && n_tiles > 1;
    float4* room = reinterpret_cast<float4*>(smem_raw + (ring - smem_u32(smem_raw))) + half * (D / 8) * kTile;   // [D / 4][128 rows]
    float2* room_ml = reinterpret_cast<float2*>(s_swap);
    if (join) {
      named_bar_sync(kBarSoft, kSoft);   // every MMA has completed: the operand tiles are free
      if (acc == 1) {
#pragma unroll 1
        for (int h = 0; h < D / 32; ++h) {
          uint32_t o[16];
          tmem_ld_32x16(t_out + 16 * h, o);
          tmem_ld_wait();
#pragma unroll
          for (int j = 0; j < 4; ++j)
            room[(4 * h + j) * kTile + r] = make_float4(__uint_as_float(o[4 * j]), __uint_as_float(o[4 * j + 1]), __uint_as_float(o[4 * j + 2]), __uint_as_float(o[4 * j + 3]));
        }
        if (half == 0) room_ml[r] = make_float2(m, l);
      }
      named_bar_sync(kBarSoft, kSoft);
      if (acc == 0) {
        const float2 ml = room_ml[r];
        const float M = fmaxf(m, ml.x), Ms = M == -INFINITY ? 0.0f : M;
        f0 = exp2_approx(m - Ms), f1 = exp2_approx(ml.x - Ms);
        l = l * f0 + ml.y * f1;
        m = M;
      }
    }
    const bool writes = two || acc == 0;
    constexpr int kPart = kPartFloats<D>;
    float* pu = a.partials + static_cast<int64_t>(unit - ta.whole) * most_parts * kPart;   // of a unit in parts
    const float inv = l > 0.0f ? 1.0f / l : 0.0f;
    if (!writes) release_tmem();
    if (writes) {
      float* pp = pu + part * kPart + q_tile * kTile * (D + 2);
#pragma unroll 1
      for (int h = 0; h < D / 32; ++h) {
        uint32_t o[16];
        if (n_tiles > 0) {
          tmem_ld_32x16(t_out + 16 * h, o);
          tmem_ld_wait();
        }
        float v[16];
#pragma unroll
        for (int j = 0; j < 16; ++j) v[j] = n_tiles > 0 ? __uint_as_float(o[j]) * f0 : 0.0f;
        if (join) {
#pragma unroll
          for (int j = 0; j < 4; ++j) {
            const float4 x = room[(4 * h + j) * kTile + r];
            v[4 * j] = fmaf(x.x, f1, v[4 * j]), v[4 * j + 1] = fmaf(x.y, f1, v[4 * j + 1]);
            v[4 * j + 2] = fmaf(x.z, f1, v[4 * j + 2]), v[4 * j + 3] = fmaf(x.w, f1, v[4 * j + 3]);
          }
        }
        if (parts > 1) {
#pragma unroll
          for (int j = 0; j < 4; ++j)
            reinterpret_cast<float4*>(pp)[(half * (D / 8) + 4 * h + j) * kTile + r] = make_float4(v[4 * j], v[4 * j + 1], v[4 * j + 2], v[4 * j + 3]);
        } else {   // by way of the query tile, which no MMA reads any more
#pragma unroll
          for (int j = 0; j < 2; ++j)
            asm volatile("st.shared.v4.u32 [%0], {%1, %2, %3, %4};" ::"r"(place(r, half * (D / 16) + 2 * h + j)),
                         "r"(pack_f16(v[8 * j] * inv, v[8 * j + 1] * inv)), "r"(pack_f16(v[8 * j + 2] * inv, v[8 * j + 3] * inv)),
                         "r"(pack_f16(v[8 * j + 4] * inv, v[8 * j + 5] * inv)), "r"(pack_f16(v[8 * j + 6] * inv, v[8 * j + 7] * inv)) : "memory");
        }
      }
      release_tmem();
      if (parts == 1) {
        const int row16 = (warp & 3) * 32 + half * 16;   // of the pair's 32 rows
        const int64_t begin = row_at(static_cast<int64_t>(a.heads) * D, row16 + (lane & 15));
        named_bar_sync(pair, 64);   // the row's other half
#pragma unroll
        for (int i = 0; i < 16 / kRowsAtOnce; ++i) {
          uint4 x;
          asm volatile("ld.shared.v4.u32 {%0, %1, %2, %3}, [%4];" : "=r"(x.x), "=r"(x.y), "=r"(x.z), "=r"(x.w)
                       : "r"(place(row16 + i * kRowsAtOnce + lane / kLanes, lane % kLanes)) : "memory");
          const int64_t p = __shfl_sync(0xffffffffu, begin, i * kRowsAtOnce + lane / kLanes);
          if (p >= 0) reinterpret_cast<uint4*>(a.out + p)[lane % kLanes] = x;
        }
      }
      if (parts > 1 && half == 0) reinterpret_cast<float2*>(pp + kTile * D)[r] = make_float2(m, l);
    }
  }

  // ---------------------------------------------------------------------- teardown
  __syncthreads();
  if (s_abort) {
    // Some role gave up.  What has been handed to the hardware still completes by itself and must have done so
    // before shared memory goes away: the producers' loads, and the issuer's MMAs (which it has seen to).
    if (!kInt8 && lane == 0 && (warp == kLoadK || warp == kLoadV)) {
      for (int i = 2 * issued + (warp == kLoadV) - 2; i >= 0 && i >= 2 * issued - C::kStages; i -= 2)
        mbar_drain(bar_full + 8 * (i % C::kStages), (i / C::kStages) & 1u);
      if (warp == kLoadV) mbar_drain(bar_fix, fix_phase & 1u);
    }
    __syncthreads();
    if (tid == 0) atomicExch(ta.status, static_cast<int>(PQ_ERR_TIMEOUT));
  }
}

template <bool kInt8, int D>
int launch(TileArgs& t, const TilePlan& plan, cudaStream_t stream) {
  using C = TileCfg<kInt8, D>;
  auto kern = attn_tile_kernel<kInt8, D>;
  static PerDeviceOnce once;
  if (const int rc = set_dynamic_smem_once(once, kern, C::kSmem); rc != PQ_OK) return rc;
  // The kernel's register split draws on what the launch holds: a build whose launch holds less must not run.
  static const int regs = [] {
    cudaFuncAttributes f = {};
    return cudaFuncGetAttributes(&f, attn_tile_kernel<kInt8, D>) == cudaSuccess ? f.numRegs : 0;
  }();
  if (regs * C::kThreads < C::kRegsNeeded) return PQ_ERR_CUDA;
  CUtensorMap mk = {}, mv = {};
  const pq_kv_cache& c = t.a.c;
  if (!kInt8) {
    const uint64_t rows = static_cast<uint64_t>(c.pages) * c.heads * c.page;
    if (const int rc = make_tmap_2d(&mk, c.k, rows, D, t.box, 64, 2, 128); rc != PQ_OK) return rc;
    if (const int rc = make_tmap_2d(&mv, c.v, rows, D, t.box, 64, 2, 128); rc != PQ_OK) return rc;
  }
  const dim3 grid(static_cast<unsigned>(plan.whole + plan.split * plan.parts));
  if (const int rc = launch_dependent(kern, grid, dim3(C::kThreads), C::kSmem, stream, mk, mv, t); rc != PQ_OK || plan.split == 0) return rc;
  return launch_dependent(attn_join_kernel<D>, dim3(static_cast<unsigned>(plan.split), 8, D / 32), dim3(kJoinThreads), 0, stream, t.a,
                          t.whole, plan.parts);
}

}  // namespace

// Units run on the SMs in waves.  Those of the last, incomplete wave (of the only one, where there are fewer units than
// SMs) have their keys cut into as many parts, of 384 keys or more, as the sum below is least for, counted in steps of 128
// keys: every CTA takes 6 steps more than its keys do, every part 0.04 to be joined, the joining kernel 4.
// (32 heads over 8 of 128, FP16: 1220 tokens over 12176, the last 12 of 160 units in 11 parts, 202 us, 303 with all of
// them whole; 64 tokens over 8064, 8 units in 13 parts, 25 and 105; 512 over 8704, 64 units in 3, 79 and 115.)
TilePlan plan_attn_tile(int64_t requests, int64_t tokens, int64_t max_q, int64_t max_kv, int window, int group, int kv_heads,
                        int dim, int sms, size_t room) {
  TilePlan p;
  const int64_t qt = 2 * (kTile / group);
  const int64_t few = kAttnRows / group + 1;   // tokens that make a request this kernel's, if there are several
  const int64_t served = requests == 1 || tokens / few > requests ? requests : tokens / few;
  const int64_t by_rows = tokens / qt + served, by_request = requests * ((max_q + qt - 1) / qt);
  const int64_t units = (by_rows < by_request ? by_rows : by_request) * kv_heads;
  auto steps_of = [&](int64_t keys) {
    if (window > 0 && keys > window + qt) keys = window + qt;
    return (keys + kTile - 1) / kTile;
  };
  const int64_t all = steps_of(max_kv), waves = units / sms, rest = units - waves * sms;
  p.whole = units;
  p.part_keys = 1 << 30;
  if (rest > 0) {
    // a single request's last units are its first tokens and see fewest keys
    int64_t keys = max_kv;
    if (waves > 0 && requests == 1) keys -= max_q - (max_q < (rest / kv_heads + 1) * qt ? max_q : (rest / kv_heads + 1) * qt);
    const int64_t steps = steps_of(keys);
    int64_t best = 1;
    double least = static_cast<double>(waves * (all + 6) + steps + 6) * 0.95;   // to be worth the other kernel
    // (Units of one query tile are bound by memory: once all SMs have had work, cutting the last of them gains nothing.)
    for (int64_t k = 2; k <= (waves > 0 && 2 * max_q <= qt ? 1 : steps / 3); ++k) {
      const double sum = static_cast<double>(waves * (all + 6)) + static_cast<double>((rest * k + sms - 1) / sms) * (static_cast<double>(steps) / k + 6) +
                         4 + 0.04 * static_cast<double>(rest * k);
      if (sum < least) least = sum, best = k;
      if (rest * k > 8 * sms) break;
    }
    const size_t one = static_cast<size_t>(2 * kTile) * (dim + 2) * 4;
    const int64_t fit = static_cast<int64_t>(room / (static_cast<size_t>(rest) * one));
    if (best > fit) best = fit;
    if (best > 1) {
      p.whole = units - rest;
      p.split = rest;
      p.part_keys = static_cast<int>((steps + best - 1) / best * kTile);
      p.parts = static_cast<int>(((steps + 1) * kTile + p.part_keys - 1) / p.part_keys);   // a window may begin inside a step
      if (p.parts > fit) p.parts = static_cast<int>(fit);   // the last part takes the keys that are left
      p.partial_bytes = static_cast<size_t>(rest) * p.parts * one;
    }
  }
  return p;
}

int launch_attn_tile(const AttnArgs& a, const TilePlan& plan, cudaStream_t stream) {
  if (plan.whole + plan.split < 1) return PQ_OK;
  if (plan.whole + plan.split * plan.parts > 0x7fffffff) return PQ_ERR_SHAPE;
  const uint32_t group = static_cast<uint32_t>(a.heads / a.c.heads);
  TileArgs t{a, device_status_ptr(), wait_limit(), 128, (65535u + group) / group,
             static_cast<int>(plan.whole), static_cast<int>(plan.split), plan.parts, 0xffffffffu, 0u};
  if (t.status == nullptr) return PQ_ERR_CUDA;
  while (a.c.page % t.box != 0) t.box /= 2;   // the page is a multiple of 16
  t.a.part_keys = plan.part_keys;
  if (a.scale_log2 == 0.0f) {
    t.q_and = 0u;
    t.a.scale_log2 = 1.0f;
  } else if (a.scale_log2 < 0.0f) {
    t.q_xor = 0x80008000u;
    t.a.scale_log2 = -a.scale_log2;
  }
  if (a.c.type == PQ_KV_INT8) return a.c.dim == 128 ? launch<true, 128>(t, plan, stream) : launch<true, 64>(t, plan, stream);
  return a.c.dim == 128 ? launch<false, 128>(t, plan, stream) : launch<false, 64>(t, plan, stream);
}

}  // namespace pq

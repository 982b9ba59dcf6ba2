// Attention of up to 16 query rows per (request, key/value head) over the paged cache: decode steps and short drafts.
#include "pq_attention.h"
#include "pq_ptx.cuh"

namespace pq {

namespace {

constexpr int kWarps = 4;
constexpr int kStageBytes = 8192;   // keys and values of one step of one warp

constexpr int rows_ctas(bool int8, int dim) { return int8 || dim == 64 ? 3 : 2; }

// A warp's step: as many keys as fill a stage, in blocks of 16 (a block never leaves its page).
template <bool kInt8, int D>
struct RowCfg {
  // CTAs per SM and stages of a warp's ring.  INT8 and dim 64 have more arithmetic per byte and want the warps:
  // 64 requests of up to 8192 tokens, INT8, dim 128: 127 us with three CTAs of two stages, 140 with two of three; dim
  // 64: 87 and 99; FP16, dim 64 (drafts of 5): 67.4 and 69.5.  FP16, dim 128 is even for one token (206; 3 x 131072: 242
  // and 247) and the other way for drafts of three, whose two tiles do not fit the registers: 173 and 166.
  static constexpr int kCtas = rows_ctas(kInt8, D), kStages = kCtas == 3 ? 2 : 3;
  static constexpr int kRowBytes = kInt8 ? D : 2 * D;
  static constexpr int kKeys = kStageBytes / (2 * kRowBytes);   // 16, 32 or 64
  static constexpr int kBlocks = kKeys / 16;
  static constexpr int kHalf = kKeys * kRowBytes;               // the keys' share of a stage; the values follow
  static constexpr int kScaleBytes = kInt8 ? 2 * kKeys * 4 : 0;
  static constexpr int kStage = kStageBytes + kScaleBytes;
  static constexpr int kSmem = kWarps * kStages * kStage;
  static constexpr int kChunksPerRow = kRowBytes / 16;
};

__device__ __forceinline__ void cp_async16(uint32_t dst, const void* src, bool live) {
  const int n = live ? 16 : 0;   // 0: the 16 bytes are filled with zeros and nothing is read
  asm volatile("cp.async.cg.shared.global [%0], [%1], 16, %2;" ::"r"(dst), "l"(src), "r"(n) : "memory");
}
__device__ __forceinline__ void cp_async4(uint32_t dst, const void* src, bool live) {
  const int n = live ? 4 : 0;
  asm volatile("cp.async.ca.shared.global [%0], [%1], 4, %2;" ::"r"(dst), "l"(src), "r"(n) : "memory");
}
__device__ __forceinline__ void cp_commit() { asm volatile("cp.async.commit_group;" ::: "memory"); }
template <int N>
__device__ __forceinline__ void cp_wait() {
  asm volatile("cp.async.wait_group %0;" ::"n"(N) : "memory");
}
__device__ __forceinline__ void ldsm4(uint32_t addr, uint32_t (&r)[4]) {
  asm volatile("ldmatrix.sync.aligned.m8n8.x4.shared.b16 {%0, %1, %2, %3}, [%4];"
               : "=r"(r[0]), "=r"(r[1]), "=r"(r[2]), "=r"(r[3]) : "r"(addr) : "memory");
}
__device__ __forceinline__ void ldsm4_t(uint32_t addr, uint32_t (&r)[4]) {
  asm volatile("ldmatrix.sync.aligned.m8n8.x4.trans.shared.b16 {%0, %1, %2, %3}, [%4];"
               : "=r"(r[0]), "=r"(r[1]), "=r"(r[2]), "=r"(r[3]) : "r"(addr) : "memory");
}
__device__ __forceinline__ uint4 lds128(uint32_t addr) {
  uint4 v;
  asm volatile("ld.shared.v4.u32 {%0, %1, %2, %3}, [%4];" : "=r"(v.x), "=r"(v.y), "=r"(v.z), "=r"(v.w) : "r"(addr) : "memory");
  return v;
}
__device__ __forceinline__ uint2 lds64(uint32_t addr) {
  uint2 v;
  asm volatile("ld.shared.v2.u32 {%0, %1}, [%2];" : "=r"(v.x), "=r"(v.y) : "r"(addr) : "memory");
  return v;
}
__device__ __forceinline__ float lds_f1(uint32_t addr) {
  float v;
  asm volatile("ld.shared.f32 %0, [%1];" : "=f"(v) : "r"(addr) : "memory");
  return v;
}
// D += A (16 x 16) B (16 x 8), FP16 in, FP32 sums.
__device__ __forceinline__ void mma16816(float (&d)[4], const uint32_t (&a)[4], uint32_t b0, uint32_t b1) {
  asm volatile("mma.sync.aligned.m16n8k16.row.col.f32.f16.f16.f32 {%0, %1, %2, %3}, {%4, %5, %6, %7}, {%8, %9}, {%0, %1, %2, %3};"
               : "+f"(d[0]), "+f"(d[1]), "+f"(d[2]), "+f"(d[3])
               : "r"(a[0]), "r"(a[1]), "r"(a[2]), "r"(a[3]), "r"(b0), "r"(b1));
}
__device__ __forceinline__ uint32_t transposed(uint32_t v) {   // an 8 x 8 tile of 16-bit values over the warp
  uint32_t r;
  asm volatile("movmatrix.sync.aligned.m8n8.trans.b16 %0, %1;" : "=r"(r) : "r"(v));
  return r;
}

// HBM bound: every cached key and value is read once, 2 * dim * (2 | 1 + 4 / dim) bytes per key and head, against
// 16 rows' worth of arithmetic at most, of which the tensor cores do the products.  m16n8k16 with the cache as the
// 16-wide operand: S^T = K Q^T and O^T = V^T P^T, so that up to 8 rows (the query heads of a group times the tokens of
// a draft) take one 8-wide tile, and up to 16 take two (kTiles).
//
// Grid: (part, key/value head, request).  A CTA owns a run of keys; its four warps take steps of 8 KB in turn, each
// with a ring of its own that it fills with 16-byte asynchronous copies a step or two ahead (no barrier between the
// warps until the end) and page ids fetched 32 blocks ahead.  Every warp keeps the running maximum and sum of its
// keys; the four are merged through shared memory, and parts of one unit through the workspace by the CTA that
// arrives last, in the order of the parts.
//
// INT8: the codes go to the tensor cores as FP16 (exact).  The key's scale multiplies the score.  The value's scale is
// split into 2^e and a rest in [1, 2); e is added to the score in powers of two, x, and the running maximum is that of
// x + e over the keys that the row sees: the FP16 weight, 2^(x + e - max + 14) times the rest, then stays below 2^15 and
// keeps its bits down to 2^-28 of the row's largest product of weight and scale, whatever the scales are.  The sum of the
// weights, FP32, takes 2^(x + e - max + 14) times 2^-e.  The feature order of a matrix step is permuted so that a lane's codes
// are 16 consecutive bytes; queries (and the result's rows) are permuted alike.
//
// FP16 holds weights up to 2^15 (kTop), so that they keep their bits down to 2^-29 of the largest and count down to 2^-39:
// 131072 keys of 2^-26 each are 0.2 % of a row, and with weights up to 1 they would be lost.
//
// Measured, 32 heads over 8 of 128, 64 requests of one token over up to 8192: FP16 207 us (6.7 TB/s, what a copy
// reaches); INT8 127 us (5.7 TB/s): issue, 62 % of the slots, for the codes' conversion and the scales.  3 requests over
// 131072: 246 us (6.5 TB/s).  1000 tokens of one request: 6.6 us, INT8 6.2, latency.
template <bool kInt8, int D, int kTiles>
__global__ void __launch_bounds__(kWarps * 32, (RowCfg<kInt8, D>::kCtas)) attn_rows_kernel(const AttnArgs a) {
  using C = RowCfg<kInt8, D>;
  constexpr int KS = D / 16;   // matrix steps over the features
  constexpr int MT = D / 16;   // 16-wide feature tiles of the result
  constexpr float kTop = kInt8 ? 14.0f : 15.0f;   // the largest weight is 2^kTop (INT8: times the rest of its scale, below 2)
  extern __shared__ __align__(128) uint8_t smem[];
  __shared__ bool s_last;

  grid_dep_launch();
  grid_dep_wait();

  const int b = blockIdx.z, hk = blockIdx.y, part = blockIdx.x;
  const int tid = threadIdx.x, lane = tid & 31, warp = tid >> 5;
  const int g = lane >> 2, c = lane & 3;
  const int G = a.heads / a.c.heads;
  const int64_t row0 = a.q_start[b];
  const AttnRange rg = attn_range(a, a.q_start[b + 1] - static_cast<int>(row0), a.kv_len[b]);
  if (rg.n <= 0 || rg.n > a.row_tokens || rg.n > 8 * kTiles / G) return;   // nothing to do, or the tile kernel's
  const int rows = rg.n * G;
  if (row0 < 0 || row0 + rg.n > a.tokens) return;

  const int lo16 = rg.lo & ~15;
  const int span = rg.hi - lo16;
  const int parts = span <= 0 ? 1 : static_cast<int>(min(static_cast<int64_t>(gridDim.x), (static_cast<int64_t>(span) + a.part_keys - 1) / a.part_keys));
  if (part >= parts) return;
  const int k_begin = lo16 + part * a.part_keys;
  const int k_end = part == parts - 1 ? rg.hi : k_begin + a.part_keys;
  const int steps = max(0, (k_end - k_begin + C::kKeys - 1) / C::kKeys);
  const int my_steps = (steps - warp + kWarps - 1) / kWarps;   // steps warp, warp + 4, ...

  const uint32_t ring = smem_u32(smem) + warp * C::kStages * C::kStage;
  const int page16 = a.c.page >> 4;
  const int64_t head_bytes = static_cast<int64_t>(a.c.page) * C::kRowBytes;
  const int* trow = a.table + static_cast<int64_t>(b) * a.width;

  // Page ids of 32 blocks of 16 keys at a time (lane l: block l of the warp's current group of steps).
  constexpr int kGroup = 32 / C::kBlocks;   // steps per group
  auto fetch_ids = [&](int group) {
    const int s = group * kGroup + lane / C::kBlocks;
    const int64_t key = static_cast<int64_t>(k_begin) + static_cast<int64_t>(s * kWarps + warp) * C::kKeys + (lane % C::kBlocks) * 16;
    int id = -1;
    if (s < my_steps && key < k_end) {
      id = trow[static_cast<int>(key >> 4) / page16];
      if (id < 0 || id >= a.c.pages) id = -1;
    }
    return id;
  };
  int ids_next = fetch_ids(0), ids = -1;

  // Requests the copies of the warp's step s into stage s % C::kStages (an empty group beyond the end).
  auto load_step = [&](int s) {
    if (s < my_steps) {
      if (s % kGroup == 0) {
        ids = ids_next;
        ids_next = fetch_ids(s / kGroup + 1);
      }
      const uint32_t st = ring + (s % C::kStages) * C::kStage;
      const int key0 = k_begin + (s * kWarps + warp) * C::kKeys;
#pragma unroll
      for (int blk = 0; blk < C::kBlocks; ++blk) {
        const int id = __shfl_sync(0xffffffffu, ids, (s % kGroup) * C::kBlocks + blk);
        const int kb = key0 + blk * 16;
        const bool there = id >= 0;
        const int off = kb - (kb >> 4) / page16 * a.c.page;   // first key of the block inside its page
        const int64_t vec = (static_cast<int64_t>(there ? id : 0) * a.c.heads + hk) * a.c.page + (there ? off : 0);
        const uint8_t* kp = static_cast<const uint8_t*>(a.c.k) + vec * C::kRowBytes;
        const uint8_t* vp = static_cast<const uint8_t*>(a.c.v) + vec * C::kRowBytes;
        constexpr int kPer = 16 * C::kChunksPerRow / 32;   // chunks of one lane per block
        if (there && kb >= rg.lo && kb + 16 <= k_end) {
#pragma unroll
          for (int i = 0; i < kPer; ++i) {
            const int idx = i * 32 + lane, r = idx / C::kChunksPerRow, ch = idx % C::kChunksPerRow;
            const int R = blk * 16 + r;
            const int kx = kInt8 ? (D == 128 ? ch ^ ((R & 1) << 2) : ch) : ch ^ (R & 7);
            const int vx = kInt8 ? (D == 128 ? ch ^ (((R >> 1) & 3) << 1) : ch ^ (((R >> 2) & 1) << 1)) : ch ^ (R & 7);
            cp_async16(st + R * C::kRowBytes + kx * 16, kp + idx * 16, true);
            cp_async16(st + C::kHalf + R * C::kRowBytes + vx * 16, vp + idx * 16, true);
          }
        } else {
#pragma unroll
          for (int i = 0; i < kPer; ++i) {
            const int idx = i * 32 + lane, r = idx / C::kChunksPerRow, ch = idx % C::kChunksPerRow;
            const int R = blk * 16 + r;
            const int kx = kInt8 ? (D == 128 ? ch ^ ((R & 1) << 2) : ch) : ch ^ (R & 7);
            const int vx = kInt8 ? (D == 128 ? ch ^ (((R >> 1) & 3) << 1) : ch ^ (((R >> 2) & 1) << 1)) : ch ^ (R & 7);
            const bool live = there && kb + r >= rg.lo && kb + r < k_end;
            cp_async16(st + R * C::kRowBytes + kx * 16, live ? kp + idx * 16 : kp, live);
            cp_async16(st + C::kHalf + R * C::kRowBytes + vx * 16, live ? vp + idx * 16 : vp, live);
          }
        }
        if constexpr (kInt8) {
          const int r = lane & 15;
          const bool live = there && kb + r >= rg.lo && kb + r < k_end;
          const float* sp = (lane < 16 ? a.c.k_scale : a.c.v_scale) + vec;
          cp_async4(st + kStageBytes + (lane < 16 ? 0 : C::kKeys * 4) + (blk * 16 + r) * 4, live ? sp + r : sp, live);
        }
      }
    }
    cp_commit();
  };

#pragma unroll
  for (int s = 0; s < C::kStages - 1; ++s) load_step(s);

  // The rows' queries as B fragments: row 8 q + g; row r is token r / G, query head hk * G + r % G.
  uint32_t qb[kTiles][KS][2];
#pragma unroll
  for (int q = 0; q < kTiles; ++q) {
    const int r = 8 * q + g;
    const __half* p = r < rows ? a.q + (row0 + r / G) * a.q_stride + (hk * G + r % G) * D : nullptr;
#pragma unroll
    for (int s = 0; s < KS; ++s) {
#pragma unroll
      for (int i = 0; i < 2; ++i) {
        const int d = kInt8 ? 16 * (c + 4 * (s / 4)) + 4 * (s % 4) + 2 * i : 16 * s + 2 * c + 8 * i;
        qb[q][s][i] = p != nullptr ? __ldg(reinterpret_cast<const uint32_t*>(p + d)) : 0u;
      }
    }
  }
  // The thread's scores are those of rows 8 q + 2 c + i: the last key that each sees, and the first (window).
  int p_row[kTiles][2], w_row[kTiles][2];
#pragma unroll
  for (int q = 0; q < kTiles; ++q) {
#pragma unroll
    for (int i = 0; i < 2; ++i) {
      const int r = 8 * q + 2 * c + i;
      const int p = rg.L - rg.n + r / G;
      p_row[q][i] = r < rows ? min(p, rg.hi - 1) : -1;
      w_row[q][i] = first_key(p, a.window) - 1;   // keys above it
    }
  }
  const int all_from = first_key(rg.L - 1, a.window);           // keys that every row sees: [all_from, all_to)
  const int all_to = min(rg.L - rg.n + 1, rg.hi);

  float o[kTiles][MT][4];
#pragma unroll
  for (int q = 0; q < kTiles; ++q) {
#pragma unroll
    for (int i = 0; i < MT; ++i) o[q][i][0] = o[q][i][1] = o[q][i][2] = o[q][i][3] = 0.0f;
  }
  float m[kTiles][2], l[kTiles][2];
#pragma unroll
  for (int q = 0; q < kTiles; ++q) m[q][0] = m[q][1] = -INFINITY, l[q][0] = l[q][1] = 0.0f;

  for (int s = 0; s < my_steps; ++s) {
    cp_wait<C::kStages - 2>();
    __syncwarp();
    load_step(s + C::kStages - 1);
    const uint32_t st = ring + (s % C::kStages) * C::kStage;
    const int key0 = k_begin + (s * kWarps + warp) * C::kKeys;

    // S^T: rows of a tile are keys g (first two values, rows 2 c and 2 c + 1 of the queries) and g + 8.
    float sc[C::kBlocks][kTiles][4];
#pragma unroll
    for (int blk = 0; blk < C::kBlocks; ++blk) {
#pragma unroll
      for (int q = 0; q < kTiles; ++q) sc[blk][q][0] = sc[blk][q][1] = sc[blk][q][2] = sc[blk][q][3] = 0.0f;
      if constexpr (!kInt8) {
        const int R = blk * 16 + (lane & 15);
#pragma unroll
        for (int k = 0; k < KS; ++k) {
          uint32_t r[4];
          ldsm4(st + R * C::kRowBytes + (((k * 2 + (lane >> 4)) ^ (R & 7)) * 16), r);
#pragma unroll
          for (int q = 0; q < kTiles; ++q) mma16816(sc[blk][q], r, qb[q][k][0], qb[q][k][1]);
        }
      } else {
        const int R0 = blk * 16 + g, R1 = R0 + 8;
#pragma unroll
        for (int q4 = 0; q4 < KS / 4; ++q4) {
          const int ch = c + 4 * q4;
          const uint4 w0 = lds128(st + R0 * C::kRowBytes + (D == 128 ? ch ^ ((R0 & 1) << 2) : ch) * 16);
          const uint4 w1 = lds128(st + R1 * C::kRowBytes + (D == 128 ? ch ^ ((R1 & 1) << 2) : ch) * 16);
          const uint32_t u0[4] = {w0.x ^ 0x80808080u, w0.y ^ 0x80808080u, w0.z ^ 0x80808080u, w0.w ^ 0x80808080u};
          const uint32_t u1[4] = {w1.x ^ 0x80808080u, w1.y ^ 0x80808080u, w1.z ^ 0x80808080u, w1.w ^ 0x80808080u};
#pragma unroll
          for (int i = 0; i < 4; ++i) {
            const uint32_t r[4] = {codes_f16(u0[i], 0x4140), codes_f16(u1[i], 0x4140), codes_f16(u0[i], 0x4342), codes_f16(u1[i], 0x4342)};
#pragma unroll
            for (int q = 0; q < kTiles; ++q) mma16816(sc[blk][q], r, qb[q][q4 * 4 + i][0], qb[q][q4 * 4 + i][1]);
          }
        }
      }
    }

    // Scores in powers of two, masked; the step's maxima.
    const bool all = key0 >= all_from && key0 + C::kKeys <= all_to;
    float vs[C::kBlocks][2], vinv[C::kBlocks][2], top[kTiles][2];
#pragma unroll
    for (int q = 0; q < kTiles; ++q) top[q][0] = top[q][1] = -INFINITY;
#pragma unroll
    for (int blk = 0; blk < C::kBlocks; ++blk) {
#pragma unroll
      for (int h = 0; h < 2; ++h) {   // keys g and g + 8
        const int j = blk * 16 + 8 * h + g;
        float ks = a.scale_log2, vlog = 0.0f;
        if constexpr (kInt8) {
          ks *= lds_f1(st + kStageBytes + j * 4);
          const float v = lds_f1(st + kStageBytes + (C::kKeys + j) * 4);
          const int e = scale_exponent(v);
          vlog = static_cast<float>(e);
          vinv[blk][h] = power_of_two(-e);
          vs[blk][h] = v * vinv[blk][h];
        }
        const int key = key0 + j;
#pragma unroll
        for (int q = 0; q < kTiles; ++q) {
#pragma unroll
          for (int i = 0; i < 2; ++i) {
            float& x = sc[blk][q][2 * h + i];
            x = kInt8 ? fmaf(x, ks, vlog) : x * ks;
            if (!all && (key > p_row[q][i] || key <= w_row[q][i])) x = -INFINITY;
            top[q][i] = fmaxf(top[q][i], x);
          }
        }
      }
    }
    bool grown = false;
#pragma unroll
    for (int d = 4; d < 32; d <<= 1) {
#pragma unroll
      for (int q = 0; q < kTiles; ++q) {
        top[q][0] = fmaxf(top[q][0], __shfl_xor_sync(0xffffffffu, top[q][0], d));
        top[q][1] = fmaxf(top[q][1], __shfl_xor_sync(0xffffffffu, top[q][1], d));
      }
    }
#pragma unroll
    for (int q = 0; q < kTiles; ++q) grown = grown || top[q][0] > m[q][0] || top[q][1] > m[q][1];
    if (__any_sync(0xffffffffu, grown)) {
#pragma unroll
      for (int q = 0; q < kTiles; ++q) {
        float f[2];
#pragma unroll
        for (int i = 0; i < 2; ++i) {
          const float mn = fmaxf(m[q][i], top[q][i]);
          f[i] = m[q][i] == -INFINITY ? 0.0f : exp2_approx(m[q][i] - mn);
          m[q][i] = mn;
          l[q][i] *= f[i];
        }
#pragma unroll
        for (int t = 0; t < MT; ++t) o[q][t][0] *= f[0], o[q][t][1] *= f[1], o[q][t][2] *= f[0], o[q][t][3] *= f[1];
      }
    }

    // Weights as B fragments (transposed: a lane has keys 2 c, 2 c + 1 of row g), then the product with the values.
#pragma unroll
    for (int blk = 0; blk < C::kBlocks; ++blk) {
      uint32_t pb[kTiles][2];
#pragma unroll
      for (int q = 0; q < kTiles; ++q) {
        const float m0 = (m[q][0] == -INFINITY ? 0.0f : m[q][0]) - kTop, m1 = (m[q][1] == -INFINITY ? 0.0f : m[q][1]) - kTop;
#pragma unroll
        for (int h = 0; h < 2; ++h) {
          const float e0 = exp2_approx(sc[blk][q][2 * h] - m0), e1 = exp2_approx(sc[blk][q][2 * h + 1] - m1);
          l[q][0] = kInt8 ? fmaf(e0, vinv[blk][h], l[q][0]) : l[q][0] + e0;
          l[q][1] = kInt8 ? fmaf(e1, vinv[blk][h], l[q][1]) : l[q][1] + e1;
          pb[q][h] = transposed(kInt8 ? pack_f16(e0 * vs[blk][h], e1 * vs[blk][h]) : pack_f16(e0, e1));
        }
      }
      const uint32_t sv = st + C::kHalf;
      if constexpr (!kInt8) {
        const int R = blk * 16 + (lane & 7) + ((lane >> 4) << 3);
#pragma unroll
        for (int t = 0; t < MT; ++t) {
          uint32_t r[4];
          ldsm4_t(sv + R * C::kRowBytes + (((t * 2 + ((lane >> 3) & 1)) ^ (R & 7)) * 16), r);
#pragma unroll
          for (int q = 0; q < kTiles; ++q) mma16816(o[q][t], r, pb[q][0], pb[q][1]);
        }
      } else {
        uint32_t w[4][D / 32];   // four keys (2c, 2c + 1, 2c + 8, 2c + 9), D / 8 consecutive features from D / 8 * g
#pragma unroll
        for (int i = 0; i < 4; ++i) {
          const int R = blk * 16 + 2 * c + (i & 1) + 8 * (i >> 1);
          if constexpr (D == 128) {
            const uint4 x = lds128(sv + R * C::kRowBytes + (g ^ (((R >> 1) & 3) << 1)) * 16);
            w[i][0] = x.x, w[i][1] = x.y, w[i][2] = x.z, w[i][3] = x.w;
          } else {
            const uint2 x = lds64(sv + R * C::kRowBytes + ((g >> 1) ^ (((R >> 2) & 1) << 1)) * 16 + (g & 1) * 8);
            w[i][0] = x.x, w[i][1] = x.y;
          }
        }
#pragma unroll
        for (int i = 0; i < D / 32; ++i) {
          const uint32_t x0 = __byte_perm(w[0][i], w[1][i], 0x5140) ^ 0x80808080u, x1 = __byte_perm(w[0][i], w[1][i], 0x7362) ^ 0x80808080u;
          const uint32_t y0 = __byte_perm(w[2][i], w[3][i], 0x5140) ^ 0x80808080u, y1 = __byte_perm(w[2][i], w[3][i], 0x7362) ^ 0x80808080u;
          const uint32_t r0[4] = {codes_f16(x0, 0x4140), codes_f16(x0, 0x4342), codes_f16(y0, 0x4140), codes_f16(y0, 0x4342)};
          const uint32_t r1[4] = {codes_f16(x1, 0x4140), codes_f16(x1, 0x4342), codes_f16(y1, 0x4140), codes_f16(y1, 0x4342)};
#pragma unroll
          for (int q = 0; q < kTiles; ++q) {
            mma16816(o[q][2 * i], r0, pb[q][0], pb[q][1]);
            mma16816(o[q][2 * i + 1], r1, pb[q][0], pb[q][1]);
          }
        }
      }
    }
    __syncwarp();   // the stage is free
  }
  cp_wait<0>();
  __syncthreads();   // the rings become the merging room

  // Merge of the four warps: [warp][row][dim] sums, then [warp][row] (maximum, sum).
  float* so = reinterpret_cast<float*>(smem);
  float2* sml = reinterpret_cast<float2*>(so + kWarps * kAttnRows * D);
#pragma unroll
  for (int q = 0; q < kTiles; ++q) {
#pragma unroll
    for (int i = 0; i < 2; ++i) {
#pragma unroll
      for (int d = 4; d < 32; d <<= 1) l[q][i] += __shfl_xor_sync(0xffffffffu, l[q][i], d);
      const int r = 8 * q + 2 * c + i;
      if (r < rows) {
        if (g == 0) sml[warp * kAttnRows + r] = make_float2(m[q][i], l[q][i]);
        float* dst = so + (warp * kAttnRows + r) * D;
#pragma unroll
        for (int t = 0; t < MT; ++t) {   // INT8: features D / 8 g + 2 t and the next; FP16: 16 t + g and 8 further
          if constexpr (kInt8) {
            *reinterpret_cast<float2*>(dst + D / 8 * g + 2 * t) = make_float2(o[q][t][i], o[q][t][2 + i]);
          } else {
            dst[16 * t + g] = o[q][t][i];
            dst[16 * t + g + 8] = o[q][t][2 + i];
          }
        }
      }
    }
  }
  __syncthreads();

  const int64_t unit = static_cast<int64_t>(b) * a.c.heads + hk;
  constexpr int kPart = kAttnRows * (D + 2);   // floats of one part
  float* pu = a.partials + unit * gridDim.x * kPart;
  auto store_out = [&](int r, int d4, float4 v) {
    uint2 h = make_uint2(pack_f16(v.x, v.y), pack_f16(v.z, v.w));
    *reinterpret_cast<uint2*>(a.out + ((row0 + r / G) * a.heads + hk * G + r % G) * D + 4 * d4) = h;
  };
  for (int idx = tid; idx < rows * (D / 4); idx += kWarps * 32) {
    const int r = idx / (D / 4), d4 = idx % (D / 4);
    float M = -INFINITY;
#pragma unroll
    for (int w = 0; w < kWarps; ++w) M = fmaxf(M, sml[w * kAttnRows + r].x);
    const float Ms = M == -INFINITY ? 0.0f : M;
    float sum = 0.0f;
    float4 v = make_float4(0.0f, 0.0f, 0.0f, 0.0f);
#pragma unroll
    for (int w = 0; w < kWarps; ++w) {
      const float2 ml = sml[w * kAttnRows + r];
      const float f = exp2_approx(ml.x - Ms);
      const float4 x = *reinterpret_cast<const float4*>(so + (w * kAttnRows + r) * D + 4 * d4);
      sum = fmaf(ml.y, f, sum);
      v.x = fmaf(x.x, f, v.x), v.y = fmaf(x.y, f, v.y), v.z = fmaf(x.z, f, v.z), v.w = fmaf(x.w, f, v.w);
    }
    if (parts == 1) {
      const float inv = sum > 0.0f ? 1.0f / sum : 0.0f;
      store_out(r, d4, make_float4(v.x * inv, v.y * inv, v.z * inv, v.w * inv));
    } else {
      *reinterpret_cast<float4*>(pu + part * kPart + r * D + 4 * d4) = v;
      if (d4 == 0) *reinterpret_cast<float2*>(pu + part * kPart + kAttnRows * D + 2 * r) = make_float2(M, sum);
    }
  }
  if (parts == 1) return;

  // The CTA that arrives last joins the parts, in their order.
  __threadfence();
  __syncthreads();
  if (tid == 0) {
    const unsigned int before = atomicAdd(a.counters + unit, 1u);
    s_last = before == static_cast<unsigned int>(parts) - 1u;
    if (s_last) a.counters[unit] = 0u;
  }
  __syncthreads();
  if (!s_last) return;
  __threadfence();
  for (int idx = tid; idx < rows * (D / 4); idx += kWarps * 32) {
    const int r = idx / (D / 4), d4 = idx % (D / 4);
    float M = -INFINITY, sum = 0.0f;
    float4 v = make_float4(0.0f, 0.0f, 0.0f, 0.0f);
#pragma unroll 4
    for (int p = 0; p < parts; ++p) {
      const float2 ml = __ldcg(reinterpret_cast<const float2*>(pu + p * kPart + kAttnRows * D + 2 * r));
      const float4 x = __ldcg(reinterpret_cast<const float4*>(pu + p * kPart + r * D + 4 * d4));
      const float mn = fmaxf(M, ml.x), ms = mn == -INFINITY ? 0.0f : mn;
      const float f = exp2_approx(M - ms), e = exp2_approx(ml.x - ms);
      M = mn;
      sum = fmaf(sum, f, ml.y * e);
      v.x = fmaf(v.x, f, x.x * e), v.y = fmaf(v.y, f, x.y * e), v.z = fmaf(v.z, f, x.z * e), v.w = fmaf(v.w, f, x.w * e);
    }
    const float inv = sum > 0.0f ? 1.0f / sum : 0.0f;
    store_out(r, d4, make_float4(v.x * inv, v.y * inv, v.z * inv, v.w * inv));
  }
}

template <bool kInt8, int D, int kTiles>
int launch_tiles(const AttnArgs& a, const AttnPlan& plan, cudaStream_t stream) {
  using C = RowCfg<kInt8, D>;
  static_assert(C::kSmem >= kWarps * kAttnRows * (D + 2) * 4, "the merge has to fit the rings");
  static PerDeviceOnce once;
  if (const int rc = set_dynamic_smem_once(once, attn_rows_kernel<kInt8, D, kTiles>, C::kSmem); rc != PQ_OK) return rc;
  const dim3 grid(static_cast<unsigned>(plan.parts), static_cast<unsigned>(a.c.heads), static_cast<unsigned>(a.requests));
  return launch_dependent(attn_rows_kernel<kInt8, D, kTiles>, grid, dim3(kWarps * 32), C::kSmem, stream, a);
}

template <bool kInt8, int D>
int launch(const AttnArgs& a, const AttnPlan& plan, int64_t max_q, cudaStream_t stream) {
  return max_q * (a.heads / a.c.heads) <= 8 ? launch_tiles<kInt8, D, 1>(a, plan, stream) : launch_tiles<kInt8, D, 2>(a, plan, stream);
}

}  // namespace

// How many keys a part gets.  `one`: what fills the resident CTAs exactly once.  Up to 1024 keys that is the choice
// (the fewest dependent steps; 1000 tokens, 8 heads: 6.6 us with parts of 128, 9.1 with 512, 11.4 without a split).
// Beyond, several waves of smaller parts even out: three where the units are few and long (3 x 131072 tokens, INT8:
// 141 us with the parts of 2432 that the rule gives, 163 with 1024, 151 with 4096, 175 with one wave; FP16: 246 with 3584,
// 258 with 1024 and 8192, but 237 with 4096 and 241 with one wave), six where there are many, of different lengths
// (64 requests of up to 8192, FP16: 209 us with the 2816 that the rule gives and with 2048, 216 with 4096, 215 with 512,
// 231 with one wave; INT8: 127 with the rule's 2176 and with 2048, 138 with 4096, 141 with 512, 155 with one wave).
AttnPlan plan_attn_rows(int64_t requests, int64_t max_q, int64_t max_kv, int window, int kv_heads, int dim, bool int8, int sms, size_t room) {
  AttnPlan p;
  p.units = requests * kv_heads;
  if (max_q > kAttnRows) max_q = kAttnRows;   // longer chunks are the tile kernel's
  if (window > 0 && max_kv > window + max_q) max_kv = window + max_q;
  const int64_t slots = static_cast<int64_t>(rows_ctas(int8, dim)) * sms;
  const int64_t one = p.units * max_kv / slots;
  int64_t keys = one;
  if (one > 1024 && p.units < slots) {
    const int64_t some = one * 5 / 8 < 2048 ? one * 5 / 8 : 2048;
    keys = one / 3 > some ? one / 3 : some;
  } else if (one > 1024) {
    keys = one / 6 > 2048 ? one / 6 : 2048;
  }
  if (keys > 4096) keys = 4096;
  if (keys < 128) keys = 128;
  const int64_t n = (max_kv + keys / 2) / keys;   // no part much smaller than the others
  if (n > 0) keys = (max_kv + 15 + n - 1) / n;
  keys = (keys + 127) / 128 * 128;
  p.part_keys = static_cast<int>(keys);
  int64_t parts = (max_kv + 15 + keys - 1) / keys;   // the first part begins at a multiple of 16
  if (p.units > kScratchCounters || parts < 1) parts = 1;
  if (parts > 65535) parts = 65535;
  const size_t bytes = static_cast<size_t>(kAttnRows) * (dim + 2) * 4;
  if (parts > 1 && static_cast<size_t>(p.units) * parts * bytes > room) {
    const int64_t fit = static_cast<int64_t>(room / (static_cast<size_t>(p.units) * bytes));
    parts = fit < 2 ? 1 : fit;   // the last part takes the keys that are left: fewer parts have to be longer
    p.part_keys = static_cast<int>(((max_kv + parts - 1) / parts + 127) / 128 * 128);
  }
  p.parts = static_cast<int>(parts);
  p.partial_bytes = parts > 1 ? static_cast<size_t>(p.units) * parts * bytes : 0;
  return p;
}

int launch_attn_rows(const AttnArgs& a, const AttnPlan& plan, int64_t max_q, cudaStream_t stream) {
  if (a.c.type == PQ_KV_INT8) return a.c.dim == 128 ? launch<true, 128>(a, plan, max_q, stream) : launch<true, 64>(a, plan, max_q, stream);
  return a.c.dim == 128 ? launch<false, 128>(a, plan, max_q, stream) : launch<false, 64>(a, plan, max_q, stream);
}

}  // namespace pq

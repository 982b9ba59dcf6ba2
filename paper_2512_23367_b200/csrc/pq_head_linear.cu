// One matrix per head: the products that take queries into the latent space and results out of it, on the tcgen05 tensor
// cores.  See include/pq.h for the contract.
#include <cuda_fp16.h>

#include "pq_attn_mma.cuh"
#include "pq_internal.h"
#include "pq_ptx.cuh"

namespace pq {

namespace {

constexpr int kOut = 128;       // outputs of a CTA: the MMA's 128 rows
constexpr int kThreads = 192;   // four warps for the results, one for the copies, one for the MMAs
constexpr int kLoader = 4, kIssuer = 5;
constexpr int kPanelK = 64;     // K of one panel
constexpr int kMostPanels = 8;

struct HeadArgs {
  const __half* w;
  __half* y;
  int64_t y_stride, y_head_stride, tokens;
  int N, panels, batch;         // outputs of a head, K / 64, tokens of a CTA (a multiple of 16)
  uint32_t cols;                // tensor memory columns: a power of two >= batch
  int* status;
  uint32_t wait_limit;
};

// Y^T = W X^T: a CTA takes 128 outputs of one head as the MMA's rows and up to 128 tokens as its columns, so that one to
// sixteen tokens cost no more tensor time than the weights' way in takes.  Bound by that way for the token counts that the
// absorbed form serves: all of a CTA's panels are requested at once, behind the wait on the kernel before, and multiplied as they
// land; before it the weights are only brought into L2, which is right whoever writes them.  (The three launches of a decode step of
// 32 tokens and 128 heads over 1000 cached ones, weights in no cache: 43.8 us; 45.0 without bringing them into L2; 42.3 with the weights
// requested before the wait, which takes another operation between their writing and the call.)
// 128 heads of 128 x 512 and 64 tokens 11.7 us alone, 5.2 in a row with the weights in L2, where the bytes take 4.2; 32 heads of
// 512 x 128 and one token 5.7 and 2.5.  Results pass through shared memory to leave as whole rows of 256 bytes.
__global__ void __launch_bounds__(kThreads) head_linear_kernel(const __grid_constant__ CUtensorMap map_w, const __grid_constant__ CUtensorMap map_x,
                                                              const HeadArgs a) {
  extern __shared__ uint8_t smem_raw[];
  __shared__ __align__(8) uint64_t bars[kMostPanels + 1];
  __shared__ uint32_t s_tmem;
  __shared__ volatile int s_abort;
  const int tid = threadIdx.x, warp = __shfl_sync(0xffffffffu, tid >> 5, 0), lane = tid & 31;
  const uint32_t bar_full = smem_u32(bars), bar_done = bar_full + 8 * kMostPanels;
  const int n0 = blockIdx.z * kOut, head = blockIdx.y;
  const int64_t t0 = static_cast<int64_t>(blockIdx.x) * a.batch;   // only the grid's first dimension has room for any number of tokens
  if (tid == 0) {
    for (int i = 0; i < a.panels; ++i) mbar_init(bar_full + 8 * i, 1);
    mbar_init(bar_done, 1);
    fence_mbar_init();
    s_abort = 0;
    tma_prefetch_desc(&map_w), tma_prefetch_desc(&map_x);
  }
  if (warp == kIssuer) {
    tmem_alloc(smem_u32(&s_tmem), a.cols);
    tmem_relinquish();
  }
  tc_fence_before_sync();
  __syncthreads();
  tc_fence_after_sync();
  grid_dep_launch();   // only now: a later launch's CTA may take this SM's tensor memory when it is given back
  const uint32_t tmem = s_tmem;
  const uint32_t sw = (smem_u32(smem_raw) + 1023u) & ~1023u, panel_x = a.batch * 128u, sx = sw + a.panels * (kOut * 128u);
  const WaitCtx wc{&s_abort, a.wait_limit};

  if (warp == kLoader) {
    // The weights come from operations like any others, so that they are read behind the wait; into L2 they go before it.
    const int row = head * a.N + n0;
    if (t0 == 0 && lane < a.panels) l2_prefetch(a.w + static_cast<int64_t>(row) * (a.panels * kPanelK) + lane * (kOut * kPanelK), kOut * kPanelK * 2);
    grid_dep_wait();
    if (lane < a.panels) {
      mbar_arrive_expect_tx(bar_full + 8 * lane, kOut * 128u + panel_x);
      tma_load_2d(sw + lane * (kOut * 128u), &map_w, bar_full + 8 * lane, lane * kPanelK, row);
      tma_load_3d(sx + lane * panel_x, &map_x, bar_full + 8 * lane, lane * kPanelK, head, static_cast<int>(t0));
    }
  } else if (warp == kIssuer) {
    const uint32_t leader = elect_one(), idesc = umma_idesc_f16(a.batch, false);
    const uint32_t w_lo = desc_k(sw), x_lo = desc_k(sx);
    bool ok = true;
    for (int i = 0; ok && i < a.panels; ++i) {
      if (!(ok = __all_sync(0xffffffffu, mbar_wait(bar_full + 8 * i, 0, wc)))) break;
      tc_fence_after_sync();
      if (leader) {
        const uint32_t wl = w_lo + i * (kOut * 128 / 16), xl = x_lo + i * (panel_x / 16);
        if (i == 0) umma_f16_ss<0>(tmem, wl, xl, idesc); else umma_f16_ss<1>(tmem, wl, xl, idesc);
#pragma unroll
        for (int k = 1; k < 4; ++k) umma_f16_ss<1>(tmem, wl + 2 * k, xl + 2 * k, idesc);
      }
      __syncwarp();
    }
    if (leader) umma_commit(bar_done);
    __syncwarp();
  } else {
    grid_dep_wait();
    const bool done = __all_sync(0xffffffffu, mbar_wait(bar_done, 0, wc));
    tc_fence_after_sync();
    // 16 tokens at a time: a thread has one output of each; rows of 128 outputs in shared memory, where the weights were
    uint16_t* room = reinterpret_cast<uint16_t*>(smem_raw + (sw - smem_u32(smem_raw)));
    const int live = static_cast<int>(min(static_cast<int64_t>(a.batch), a.tokens - t0));
    for (int c = 0; done && c < live; c += 16) {
      uint32_t v[16];
      tmem_ld_32x16(tmem + c + (static_cast<uint32_t>(warp) << 21), v);
      tmem_ld_wait();
#pragma unroll
      for (int j = 0; j < 16; ++j) room[(c + j) * kOut + tid] = __half_as_ushort(__float2half_rn(__uint_as_float(v[j])));
    }
    // The four warps meet whatever their own waits came to (one may run out of polls where the next one's last poll succeeds), and
    // store only if all have their outputs there.
    if (!pair_any<128>(1, !done)) {
      for (int i = tid; i < live * (kOut / 8); i += 128) {
        const int t = i / (kOut / 8), c = i % (kOut / 8);
        reinterpret_cast<uint4*>(a.y + (t0 + t) * a.y_stride + head * a.y_head_stride + n0)[c] = reinterpret_cast<const uint4*>(room + t * kOut)[c];
      }
    }
  }
  tc_fence_before_sync();
  __syncthreads();
  tc_fence_after_sync();
  if (s_abort) {   // what is on the way ends by itself, and must have before the memory goes away
    if (tid == 0) {
      for (int i = 0; i < a.panels; ++i) mbar_drain(bar_full + 8 * i, 0);
      mbar_drain(bar_done, 0);
      atomicExch(a.status, static_cast<int>(PQ_ERR_TIMEOUT));
    }
    __syncthreads();
  }
  if (warp == kIssuer) tmem_dealloc(tmem, a.cols);
}

}  // namespace
}  // namespace pq

using namespace pq;

extern "C" {

int pq_head_linear(const void* x_f16, int64_t x_stride, int64_t x_head_stride, const void* w_f16, int32_t heads, int64_t N, int64_t K,
                   int64_t tokens, void* y_f16, int64_t y_stride, int64_t y_head_stride, void* stream) {
  if (heads < 1 || heads > 1024 || N < kOut || N > 1024 || N % kOut != 0 || K < kPanelK || K > kMostPanels * kPanelK || K % kPanelK != 0) return PQ_ERR_SHAPE;
  if (tokens < 0 || tokens > 0x7fffffff) return PQ_ERR_SHAPE;
  if (heads == 1) x_head_stride = K, y_head_stride = N;
  if (tokens <= 1) x_stride = x_head_stride * heads, y_stride = y_head_stride * heads;
  if (x_stride % 8 != 0 || x_head_stride % 8 != 0 || y_stride % 8 != 0 || y_head_stride % 8 != 0) return PQ_ERR_SHAPE;
  if (x_stride < K || x_head_stride < K || y_stride < N || y_head_stride < N) return PQ_ERR_SHAPE;
  if (x_stride >= int64_t(1) << 38 || x_head_stride >= int64_t(1) << 38) return PQ_ERR_SHAPE;   // what a tensor map holds
  if (tokens == 0) return PQ_OK;
  if (!x_f16 || !w_f16 || !y_f16) return PQ_ERR_NULL;
  if (!aligned16(x_f16) || !aligned16(w_f16) || !aligned16(y_f16)) return PQ_ERR_ALIGN;
  int rc = check_arch();
  if (rc != PQ_OK) return rc;
  // tokens of a CTA: as many as there are, up to 128, or 64 where the weights' panels leave no more room
  const int64_t most = K > 256 ? 64 : 128, up = (tokens + 15) / 16 * 16;
  HeadArgs a{static_cast<const __half*>(w_f16), static_cast<__half*>(y_f16), y_stride, y_head_stride, tokens, static_cast<int>(N), static_cast<int>(K / kPanelK),
             static_cast<int>(up < most ? up : most), 32, device_status_ptr(), wait_limit()};
  if (a.status == nullptr) return PQ_ERR_CUDA;
  while (a.cols < static_cast<uint32_t>(a.batch)) a.cols *= 2;
  const int64_t batches = (tokens + a.batch - 1) / a.batch;
  CUtensorMap mw = {}, mx = {};
  if ((rc = make_tmap_2d(&mw, w_f16, static_cast<uint64_t>(heads) * N, K, kOut, kPanelK, 2, 128)) != PQ_OK) return rc;
  if ((rc = make_tmap_heads(&mx, x_f16, tokens, heads, K, x_stride, x_head_stride, a.batch)) != PQ_OK) return rc;
  static PerDeviceOnce once;
  constexpr int kMostSmem = kMostPanels * (kOut + 64) * 128 + 1024;   // K = 512 with 64 tokens; 256 with 128 is less
  if ((rc = set_dynamic_smem_once(once, head_linear_kernel, kMostSmem)) != PQ_OK) return rc;
  const size_t smem = static_cast<size_t>(a.panels) * (kOut + a.batch) * 128 + 1024;
  return launch_dependent(head_linear_kernel, dim3(static_cast<unsigned>(batches), heads, static_cast<unsigned>(N / kOut)), dim3(kThreads), smem,
                          static_cast<cudaStream_t>(stream), mw, mx, a);
}

}  // extern "C"

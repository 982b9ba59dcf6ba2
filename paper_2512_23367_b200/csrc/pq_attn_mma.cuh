// Pieces that the attention kernels on the tcgen05 tensor cores share: FP16 MMAs and their descriptors, stores to
// tensor memory, the exchange between the two threads of a row, paired FP32 arithmetic.
#pragma once
#include <cstdint>

#include "pq_ptx.cuh"

namespace pq {

// ---- tcgen05 with 16-bit floating-point operands
// kind::f16, FP16 A and B, FP32 accumulator, M = 128 unless said otherwise; b_mn: B is stored with its N dimension contiguous.
__host__ __device__ constexpr uint32_t umma_idesc_f16(uint32_t N, bool b_mn, uint32_t M = 128u) {
  return (1u << 4) | (b_mn ? (1u << 16) : 0u) | ((N >> 3) << 17) | ((M >> 4) << 24);
}
// Shared-memory operand descriptors, low word: start address in 16-byte units and the leading byte offset.  The high
// word is the same for both kinds: groups of 8 rows of 128 bytes lie 1024 bytes apart, 128-byte swizzle.
//   K-major (Q, K):   64 features per 128-byte row; a k step of 16 is 32 bytes further.
//   MN-major (V):     panels of 64 columns, `panel` bytes apart; a k step of 16 keys is 2048 bytes further.
constexpr uint32_t kDescHi = (1024u >> 4) | (1u << 14) | (2u << 29);
__device__ __forceinline__ uint32_t desc_k(uint32_t saddr) { return ((saddr & 0x3FFFFu) >> 4) | (1u << 16); }
__device__ __forceinline__ uint32_t desc_mn(uint32_t saddr, uint32_t panel) { return ((saddr & 0x3FFFFu) >> 4) | ((panel >> 4) << 16); }
// One MMA of 128 x N x 16.  Operands stay in uniform registers (the whole warp computes them, one elected thread
// issues): with per-thread operands an issue took 93 to 120 cycles against the 64 that the tensor core needs.
template <int kAccumulate>
__device__ __forceinline__ void umma_f16_ss(uint32_t d, uint32_t a_lo, uint32_t b_lo, uint32_t idesc) {
  asm volatile("{\n\t.reg .pred p;\n\t.reg .b64 a, b;\n\tsetp.ne.b32 p, %4, 0;\n\tmov.b64 a, {%1, %5};\n\tmov.b64 b, {%2, %5};\n\t"
               "tcgen05.mma.cta_group::1.kind::f16 [%0], a, b, %3, p;\n\t}"
               ::"r"(d), "r"(a_lo), "r"(b_lo), "r"(idesc), "n"(kAccumulate), "n"(kDescHi) : "memory");
}
// A in tensor memory: lane = row, a 32-bit column holds two neighbouring k.
__device__ __forceinline__ void umma_f16_ts(uint32_t d, uint32_t a, uint32_t b_lo, uint32_t idesc, uint32_t accumulate) {
  asm volatile("{\n\t.reg .pred p;\n\t.reg .b64 b;\n\tsetp.ne.b32 p, %4, 0;\n\tmov.b64 b, {%2, %5};\n\t"
               "tcgen05.mma.cta_group::1.kind::f16 [%0], [%1], b, %3, p;\n\t}"
               ::"r"(d), "r"(a), "r"(b_lo), "r"(idesc), "r"(accumulate), "n"(kDescHi) : "memory");
}
__device__ __forceinline__ void tmem_st_32x32(uint32_t taddr, const uint32_t (&r)[32]) {
  asm volatile(
      "tcgen05.st.sync.aligned.32x32b.x32.b32 [%0], "
      "{%1, %2, %3, %4, %5, %6, %7, %8, %9, %10, %11, %12, %13, %14, %15, %16, "
      "%17, %18, %19, %20, %21, %22, %23, %24, %25, %26, %27, %28, %29, %30, %31, %32};" ::"r"(taddr),
      "r"(r[0]), "r"(r[1]), "r"(r[2]), "r"(r[3]), "r"(r[4]), "r"(r[5]), "r"(r[6]), "r"(r[7]), "r"(r[8]), "r"(r[9]),
      "r"(r[10]), "r"(r[11]), "r"(r[12]), "r"(r[13]), "r"(r[14]), "r"(r[15]), "r"(r[16]), "r"(r[17]), "r"(r[18]),
      "r"(r[19]), "r"(r[20]), "r"(r[21]), "r"(r[22]), "r"(r[23]), "r"(r[24]), "r"(r[25]), "r"(r[26]), "r"(r[27]),
      "r"(r[28]), "r"(r[29]), "r"(r[30]), "r"(r[31])
      : "memory");
}
__device__ __forceinline__ void tmem_st_32x16(uint32_t taddr, const uint32_t (&r)[16]) {
  asm volatile(
      "tcgen05.st.sync.aligned.32x32b.x16.b32 [%0], {%1, %2, %3, %4, %5, %6, %7, %8, %9, %10, %11, %12, %13, %14, %15, %16};" ::"r"(taddr),
      "r"(r[0]), "r"(r[1]), "r"(r[2]), "r"(r[3]), "r"(r[4]), "r"(r[5]), "r"(r[6]), "r"(r[7]), "r"(r[8]), "r"(r[9]),
      "r"(r[10]), "r"(r[11]), "r"(r[12]), "r"(r[13]), "r"(r[14]), "r"(r[15])
      : "memory");
}
__device__ __forceinline__ void tmem_st_32x4(uint32_t taddr, const uint32_t (&r)[4]) {
  asm volatile("tcgen05.st.sync.aligned.32x32b.x4.b32 [%0], {%1, %2, %3, %4};" ::"r"(taddr), "r"(r[0]), "r"(r[1]), "r"(r[2]), "r"(r[3]) : "memory");
}
__device__ __forceinline__ void tmem_ld_32x8(uint32_t taddr, uint32_t (&r)[8]) {
  asm volatile("tcgen05.ld.sync.aligned.32x32b.x8.b32 {%0, %1, %2, %3, %4, %5, %6, %7}, [%8];"
               : "=r"(r[0]), "=r"(r[1]), "=r"(r[2]), "=r"(r[3]), "=r"(r[4]), "=r"(r[5]), "=r"(r[6]), "=r"(r[7]) : "r"(taddr) : "memory");
}
__device__ __forceinline__ void tmem_st_wait() { asm volatile("tcgen05.wait::st.sync.aligned;" ::: "memory"); }

// 32 bytes by one thread: what a lane per row leaves of a warp's store.  The wide store writes a whole sector, but faults unless its
// address is a multiple of 32, and a caller's output is one of 16 only: there two stores of 16 bytes.  The rows of a call's output
// are multiples of 32 bytes apart, so that all of its stores go the same way.
__device__ __forceinline__ void store_32_bytes(void* to, uint32_t a, uint32_t b, uint32_t c, uint32_t d, uint32_t e, uint32_t f, uint32_t g, uint32_t h) {
  if ((reinterpret_cast<uintptr_t>(to) & 16u) == 0) {
    asm volatile("st.global.v8.b32 [%0], {%1, %2, %3, %4, %5, %6, %7, %8};" ::"l"(to), "r"(a), "r"(b), "r"(c), "r"(d), "r"(e), "r"(f), "r"(g), "r"(h) : "memory");
  } else {
    static_cast<uint4*>(to)[0] = make_uint4(a, b, c, d);
    static_cast<uint4*>(to)[1] = make_uint4(e, f, g, h);
  }
}
__device__ __forceinline__ void named_bar_arrive(uint32_t id, uint32_t nthreads) {
  asm volatile("bar.arrive %0, %1;" ::"r"(id), "r"(nthreads) : "memory");
}
// Meets the other warps that share the barrier (of a pair: 64 threads); whether any of their threads says yes.
template <int kThreads = 64>
__device__ __forceinline__ bool pair_any(uint32_t id, bool yes) {
  uint32_t r;
  asm volatile("{\n\t.reg .pred p, q;\n\tsetp.ne.b32 p, %2, 0;\n\tbar.red.or.pred q, %1, %3, p;\n\tselp.u32 %0, 1, 0, q;\n\t}"
               : "=r"(r) : "r"(id), "r"(static_cast<uint32_t>(yes)), "n"(kThreads) : "memory");
  return r != 0;
}

// Watcher and issuer meet; whether the operand tile has landed (the watcher's word; the issuer says yes).
__device__ __forceinline__ bool tile_landed(uint32_t id, bool yes) {
  uint32_t r;
  asm volatile("{\n\t.reg .pred p, q;\n\tsetp.ne.b32 p, %2, 0;\n\tbar.red.and.pred q, %1, 64, p;\n\tselp.u32 %0, 1, 0, q;\n\t}"
               : "=r"(r) : "r"(id), "r"(static_cast<uint32_t>(yes)) : "memory");
  return r != 0;
}
// "Done" to the issuer.  A warp that has given up waiting for S is no longer paced by it: it meets the issuer instead, so
// that it cannot arrive twice for one of the issuer's waits (which would leave the issuer waiting for good).
__device__ __forceinline__ void hand_over(uint32_t id, uint32_t nthreads, bool ok) {
  if (ok) named_bar_arrive(id, nthreads); else named_bar_sync(id, nthreads);
}
// The sum, or the larger, of a value of the row's two threads, the same in both: the second half's goes to the first
// and the result back.
template <bool kSum>
__device__ __forceinline__ float pair_combine(float* word, uint32_t id, int half, float v) {
  if (half == 1) *word = v;
  named_bar_sync(id, 64);
  if (half == 0) {
    v = kSum ? v + *word : fmaxf(v, *word);
    *word = v;
  }
  named_bar_sync(id, 64);
  if (half == 1) v = *word;
  return v;
}

// Two FP32 operations in one instruction.
__device__ __forceinline__ uint64_t pair_f32(float a, float b) {
  uint64_t r;
  asm("mov.b64 %0, {%1, %2};" : "=l"(r) : "f"(a), "f"(b));
  return r;
}
__device__ __forceinline__ void unpair_f32(uint64_t v, float& a, float& b) { asm("mov.b64 {%0, %1}, %2;" : "=f"(a), "=f"(b) : "l"(v)); }
__device__ __forceinline__ uint64_t fma_f32x2(uint64_t a, uint64_t b, uint64_t c) {
  uint64_t d;
  asm("fma.rn.f32x2 %0, %1, %2, %3;" : "=l"(d) : "l"(a), "l"(b), "l"(c));
  return d;
}
__device__ __forceinline__ uint64_t add_f32x2(uint64_t a, uint64_t b) {
  uint64_t d;
  asm("add.rn.f32x2 %0, %1, %2;" : "=l"(d) : "l"(a), "l"(b));
  return d;
}
__device__ __forceinline__ uint64_t mul_f32x2(uint64_t a, uint64_t b) {
  uint64_t d;
  asm("mul.rn.f32x2 %0, %1, %2;" : "=l"(d) : "l"(a), "l"(b));
  return d;
}
__device__ __forceinline__ float max3(float a, float b, float c) {
  float d;
  asm("max.f32 %0, %1, %2, %3;" : "=f"(d) : "f"(a), "f"(b), "f"(c));
  return d;
}
// A wait of a whole warp whose lanes go on, or give up, together.
__device__ __forceinline__ bool warp_wait(uint32_t bar, uint32_t parity, const WaitCtx& wc) {
  return __all_sync(0xffffffffu, mbar_wait(bar, parity, wc));
}
__device__ __forceinline__ int warp_prefix(int v, int lane) {   // inclusive sums
#pragma unroll
  for (int o = 1; o < 32; o <<= 1) {
    const int x = __shfl_up_sync(0xffffffffu, v, o);
    if (lane >= o) v += x;
  }
  return v;
}

}  // namespace pq

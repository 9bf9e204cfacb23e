// What the warp-specialised tcgen05 kernels share (tree_attn.cu,
// key_weights.cu): bounded waits of a warp in step, ring positions, one
// arrival or one block of TMA boxes by an elected lane.
#pragma once

#include "tcgen05.cuh"

namespace mcpu {

constexpr int kBlockKeys = 128;  // keys of one K or V block
constexpr int kBlockPages = kBlockKeys / kPage;
constexpr int kBlockBytes = kBlockKeys * kRowBytes;  // 16 KiB

// A bounded wait of a warp in step: few instructions, and one outcome for the
// warp, so that its branches are uniform. A test returns when the phase
// completes or after about 1.4 us, so 2^17 of them take 0.2 s; then the role
// ends and raises the abort flag, and the other roles' waits run out likewise.
__device__ __forceinline__ bool wait_warp(uint32_t bar, uint32_t parity) {
  uint32_t left;
  asm volatile(
      "{\n\t.reg .pred p;\n\tmov.b32 %0, 0x20000;\n"
      "again:\n\tmbarrier.try_wait.parity.shared::cta.b64 p, [%1], %2;\n\t"
      "vote.sync.all.pred p, p, 0xffffffff;\n\t@p bra.uni done;\n\t"
      "sub.u32 %0, %0, 1;\n\tsetp.ne.u32 p, %0, 0;\n\t@p bra.uni again;\n"
      "done:\n\t}"
      : "=&r"(left)
      : "r"(bar), "r"(parity)
      : "memory");
  return left != 0;
}

// Whether the phase has completed, asked ahead of the time it matters.
__device__ __forceinline__ bool peek(uint32_t bar, uint32_t parity) {
  uint32_t ok;
  asm volatile(
      "{\n\t.reg .pred p;\n\tmbarrier.test_wait.parity.shared::cta.b64 p, [%1], %2;\n\tselp.u32 %0, 1, 0, p;\n\t}"
      : "=r"(ok)
      : "r"(bar), "r"(parity)
      : "memory");
  return ok != 0;
}

// A block's eight pages by TMA, issued by one elected lane of a warp in step.
// One election for all of it, and operands that differ by constants: from a
// lone lane, or with an election per operation, the operands' way to the
// uniform datapath takes longer than the work that is issued. (The same holds
// for a block's MMAs.)
__device__ __forceinline__ void load_block_e(uint32_t dst, const CUtensorMap* map, const int (&y)[kBlockPages],
                                             uint32_t bar, uint64_t policy) {
  static_assert(kBlockPages == 8 && kTileBytes == 2048, "eight boxes of 2 KiB");
  asm volatile(
      "{\n\t.reg .pred e;\n\t.reg .b32 z;\n\tmov.b32 z, 0;\n\telect.sync _|e, 0xffffffff;\n\t"
      "@e mbarrier.arrive.expect_tx.shared::cta.b64 _, [%2], %4;\n\t"
      "@e cp.async.bulk.tensor.2d.shared::cluster.global.mbarrier::complete_tx::bytes.L2::cache_hint"
      " [%0 + 0], [%1, {z, %5}], [%2], %3;\n\t"
      "@e cp.async.bulk.tensor.2d.shared::cluster.global.mbarrier::complete_tx::bytes.L2::cache_hint"
      " [%0 + 2048], [%1, {z, %6}], [%2], %3;\n\t"
      "@e cp.async.bulk.tensor.2d.shared::cluster.global.mbarrier::complete_tx::bytes.L2::cache_hint"
      " [%0 + 4096], [%1, {z, %7}], [%2], %3;\n\t"
      "@e cp.async.bulk.tensor.2d.shared::cluster.global.mbarrier::complete_tx::bytes.L2::cache_hint"
      " [%0 + 6144], [%1, {z, %8}], [%2], %3;\n\t"
      "@e cp.async.bulk.tensor.2d.shared::cluster.global.mbarrier::complete_tx::bytes.L2::cache_hint"
      " [%0 + 8192], [%1, {z, %9}], [%2], %3;\n\t"
      "@e cp.async.bulk.tensor.2d.shared::cluster.global.mbarrier::complete_tx::bytes.L2::cache_hint"
      " [%0 + 10240], [%1, {z, %10}], [%2], %3;\n\t"
      "@e cp.async.bulk.tensor.2d.shared::cluster.global.mbarrier::complete_tx::bytes.L2::cache_hint"
      " [%0 + 12288], [%1, {z, %11}], [%2], %3;\n\t"
      "@e cp.async.bulk.tensor.2d.shared::cluster.global.mbarrier::complete_tx::bytes.L2::cache_hint"
      " [%0 + 14336], [%1, {z, %12}], [%2], %3;\n\t"
      "}" ::"r"(dst),
      "l"(reinterpret_cast<uint64_t>(map)), "r"(bar), "l"(policy), "n"(kBlockBytes), "r"(y[0]), "r"(y[1]), "r"(y[2]),
      "r"(y[3]), "r"(y[4]), "r"(y[5]), "r"(y[6]), "r"(y[7])
      : "memory");
}

// A ring's position: stage and the parity of its turn, without a division.
template <uint32_t kStages>
struct RingAt {
  uint32_t s = 0, parity = 0;
  __device__ __forceinline__ void next() {
    if (++s == kStages) s = 0, parity ^= 1;
  }
};

// One arrival of a warp in step.
__device__ __forceinline__ void mbar_arrive_e(uint32_t bar) {
  asm volatile(
      "{\n\t.reg .pred e;\n\telect.sync _|e, 0xffffffff;\n\t"
      "@e mbarrier.arrive.shared::cta.b64 _, [%0];\n\t}" ::"r"(bar)
      : "memory");
}

}  // namespace mcpu

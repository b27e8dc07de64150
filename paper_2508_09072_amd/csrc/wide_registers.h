// Accumulation registers managed by hand, for kernels of four wavefronts that carry 64 query rows each
// (tree_attn_wide.hip, prompt_attn.hip).
#pragma once

#include "tree_attn_common.h"

namespace reader {

namespace {

// The accumulation registers (a0..a255 of every lane) are managed by hand in these kernels: the compiler is
// told never to use them (-amdgpu-spill-vgpr-to-agpr=0 and no operand of that class anywhere), the
// instructions below name them by number, and what they hold is invisible to the register allocator, which
// is left with the ~200 vector registers of scores, weights and operand fragments.  Layout per lane:
//   output accumulators O^T of row block r, output block db:  16 registers from o(r, db)
//   query fragment of row block r, k-step kk (B operand of the first product):  4 registers from q(r, kk)
template <int D>
struct AccMap {
    static constexpr int kOB = D / 32, kK = D / 16;
    static constexpr int o(int r, int db) { return (r * kOB + db) * 16; }
    static constexpr int q(int r, int kk) { return 2 * kOB * 16 + (r * kK + kk) * 4; }
    static constexpr int kCount = 2 * kOB * 16 + 2 * kK * 4;   // 192 (D = 128), 96 (D = 64)
    // ... and per-lane values that are needed once per tile or per segment, kept out of the vector
    // registers the pipelined tile code needs for itself (one instruction brings one back):
    static constexpr int kParked = kCount;
    static constexpr int node(int r) { return kParked + r; }            // tree node of the lane's row in row block r
    static constexpr int group(int r) { return kParked + 2 + r; }       // ... and its query head within the kv head
    static constexpr int m_ref(int r) { return kParked + 4 + r; }       // the row's softmax reference (a score, not yet scaled)
    static constexpr int k_off(int i) { return kParked + 6 + i; }       // byte offsets of the lane's part of copy i of a whole prefix tile (K, V)
    static constexpr int v_off(int i) { return kParked + 6 + D / 32 + i; }
    static constexpr int kEnd = kParked + 6 + 2 * (D / 32);
};
// Nothing here is known to the compiler as a matrix instruction, so the waits the hardware leaves to software
// are the caller's business: a result is read by the vector ALU (v_accvgpr_read, or any instruction on a
// score register) no sooner than 11 instructions after the matrix instruction that wrote it; a dependent
// matrix instruction on exactly the same accumulator needs none.
template <int LO> __device__ __forceinline__ void mfma_o(const bf16x8 &a, const bf16x8 &b) {   // a[LO..LO+15] += a . b
    asm volatile("v_mfma_f32_32x32x16_bf16 a[%c0:%c1], %2, %3, a[%c0:%c1]" :: "n"(LO), "n"(LO + 15), "v"(a), "v"(b));
}
template <int Q> __device__ __forceinline__ void mfma_s0(f32x16 &acc, const bf16x8 &k) {       // acc = k . a[Q..Q+3]
    asm volatile("v_mfma_f32_32x32x16_bf16 %0, %1, a[%c2:%c3], 0" : "=&v"(acc) : "v"(k), "n"(Q), "n"(Q + 3));
}
template <int Q> __device__ __forceinline__ void mfma_s(f32x16 &acc, const bf16x8 &k) {        // acc += k . a[Q..Q+3]
    asm volatile("v_mfma_f32_32x32x16_bf16 %0, %1, a[%c2:%c3], %0" : "+v"(acc) : "v"(k), "n"(Q), "n"(Q + 3));
}
template <int I> __device__ __forceinline__ void acc_write(uint32_t v) { asm volatile("v_accvgpr_write_b32 a%c0, %1" :: "n"(I), "v"(v)); }
template <int I> __device__ __forceinline__ void acc_zero() { asm volatile("v_accvgpr_write_b32 a%c0, 0" :: "n"(I)); }
template <int I> __device__ __forceinline__ float acc_read() {
    float x;
    asm volatile("v_accvgpr_read_b32 %0, a%c1" : "=v"(x) : "n"(I));
    return x;
}
template <int I> __device__ __forceinline__ uint32_t acc_read_u32() {
    uint32_t x;
    asm volatile("v_accvgpr_read_b32 %0, a%c1" : "=v"(x) : "n"(I));
    return x;
}
#define READER_RESULT_WAIT() asm volatile("s_nop 15")   /* 16 wait states: matrix result -> vector ALU */

}  // namespace

}  // namespace reader

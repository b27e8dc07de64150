// One query row of the prompts' attention over a range of its keys, by one wavefront, the plain way: scores of 64 keys,
// one per lane, the running maximum and sum of a softmax, then the values, D / 64 of the output per lane.  The whole of
// dims.variant = 1, and what the matrix kernels fall back on for rows that their fixed reference cannot hold.
#pragma once

#include "prompt_common.h"
#include "tree_attn_common.h"

namespace reader {

template <int D>
struct ScalarRow {
    float m = -INFINITY, l = 0.f, o[D / 64] = {};      // maximum (exponent of two), sum, sum of weighted values
};

// Keys [j0, j1) of the sequence whose row of the page table is `table`; a key behind a bad page id is left out.
template <int D>
__device__ inline ScalarRow<D> prompt_row_scalar(const PromptParams &p, const uint16_t *__restrict__ q, const int32_t *__restrict__ table,
                                                 int hkv, int j0, int j1, int lane, int &bad) {
    constexpr int kPer = D / 64;
    ScalarRow<D> s;
    for (int base = j0; base < j1; base += 64) {
        const int j = base + lane;
        const int page = j < j1 ? table[j >> 4] : -1;
        const bool ok = page >= 0 && page < p.num_pages;
        if (j < j1 && !ok) bad |= READER_STATUS_BAD_PAGE;
        const size_t at = (((size_t)(ok ? page : 0) * p.Hkv + hkv) * READER_PAGE_SIZE + (j & 15)) * D;
        float x = -INFINITY;
        if (ok) {
            float dot = 0.f;
            for (int c = 0; c < D; c += 8) {
                const u32x4 k = ld16(p.k_cache + at + c), w = ld16(q + c);
#pragma unroll
                for (int i = 0; i < 4; ++i) {
                    dot += __uint_as_float(k[i] << 16) * __uint_as_float(w[i] << 16);
                    dot += __uint_as_float(k[i] & 0xffff0000u) * __uint_as_float(w[i] & 0xffff0000u);
                }
            }
            x = dot * p.scale_log2;
        }
        float m = x;
#pragma unroll
        for (int off = 32; off >= 1; off >>= 1) m = fmaxf(m, __shfl_xor(m, off));
        m = fmaxf(m, s.m);
        // (nothing seen so far: no weight; the sum of a NaN shows)
        const float keep = s.m == -INFINITY ? 0.f : __builtin_amdgcn_exp2f(s.m - m);
        const float w = ok ? (x == -INFINITY ? 0.f : __builtin_amdgcn_exp2f(x - m)) : 0.f;
        float l = w;
#pragma unroll
        for (int off = 32; off >= 1; off >>= 1) l += __shfl_xor(l, off);
        s.l = s.l * keep + l;
        s.m = m;
#pragma unroll
        for (int e = 0; e < kPer; ++e) s.o[e] *= keep;
        for (unsigned long long todo = __ballot(ok); todo; todo &= todo - 1) {
            const int k = (int)__builtin_ctzll(todo);
            const float wk = __shfl(w, k);
            const size_t v_at = __shfl((unsigned long long)at, k) + lane * kPer;
#pragma unroll
            for (int e = 0; e < kPer; ++e) s.o[e] += wk * __uint_as_float((uint32_t)p.v_cache[v_at + e] << 16);
        }
    }
    return s;
}

}  // namespace reader

// Causal attention of packed prompts over the paged cache, the plain way: one wavefront per (token, query head).
// dims.variant = 1, for cross-checks.
#include "prompt_attn_scalar.h"

namespace reader {

namespace {

template <int D>
__global__ __launch_bounds__(256) void prompt_attn_scalar_kernel(PromptParams p) {
    const int lane = threadIdx.x & 63;
    const long long unit = (long long)blockIdx.x * 4 + __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    const int t = (int)(unit / p.Hq), hq = (int)(unit - (long long)t * p.Hq);
    int bad = 0;
    if (blockIdx.x == 0) report_bad_sequences(p, 256);
    if (t >= p.N) return;
    int first = 0;
    const int b = sequence_of_row(p.cu_tokens, p.B, t, lane, first);
    if (b >= p.B) return;
    const int row = t - first, L = p.seq_lens[b];
    const long long last = (long long)max(L, 0) + row + 1;
    const int keys = (int)(last < p.max_seq_len ? last : p.max_seq_len);
    const ScalarRow<D> s = prompt_row_scalar<D>(p, p.q + ((size_t)t * p.Hq + hq) * D, p.page_table + (size_t)b * p.max_pages,
                                                hq / p.G, 0, keys, lane, bad);
    const float inv = s.l == 0.f ? 0.f : 1.f / s.l;             // (a row that sees no key: zeros)
#pragma unroll
    for (int e = 0; e < D / 64; ++e)
        p.out[((size_t)t * p.Hq + hq) * D + lane * (D / 64) + e] = (uint16_t)pack_bf16x2(s.o[e] * inv, 0.f);
    if (p.lse && lane == 0) p.lse[(size_t)t * p.Hq + hq] = s.l == 0.f ? -INFINITY : (s.m + __builtin_amdgcn_logf(s.l)) * kLn2;
    if (bad && p.status) atomicOr(p.status, bad);
}

}  // namespace

hipError_t launch_prompt_attn_scalar(const PromptParams &p, hipStream_t stream) {
    const unsigned blocks = (unsigned)(((long long)p.N * p.Hq + 3) / 4);
    if (p.D == 64) hipLaunchKernelGGL(prompt_attn_scalar_kernel<64>, dim3(blocks), dim3(256), 0, stream, p);
    else hipLaunchKernelGGL(prompt_attn_scalar_kernel<128>, dim3(blocks), dim3(256), 0, stream, p);
    return note_hip_error("launch prompt_attn_scalar_kernel", hipGetLastError());
}

}  // namespace reader

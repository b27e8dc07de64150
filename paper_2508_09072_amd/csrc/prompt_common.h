// What the operators around the verification step share: where a packed token belongs, and the parameters of their launches.
#pragma once

#include "internal.h"

namespace reader {

// Rows of a packed batch: sequence b owns rows cu_tokens[b] .. cu_tokens[b + 1] - 1 of N.  Bounds outside [0, N] count as the
// nearest one inside, so nothing in a table leads an access out of the tensors.
// `check`, which is zero, or no number once a or b is none.
__device__ __forceinline__ float no_number(float check, float a, float b) { return fmaf(b, 0.f, fmaf(a, 0.f, check)); }

__device__ inline int clamp_row(int row, int N) { return row < 0 ? 0 : (row > N ? N : row); }

// Sequence that owns row t, found by a whole wavefront together: 64 bounds are compared at a time.  first: its first row.  B: nobody's.
// (Several, where bounds go back: the first of them.)
__device__ inline int sequence_of_row(const int32_t *__restrict__ cu_tokens, int B, int t, int lane, int &first) {
    int lo = 0, len = B;
    while (len > 64) {
        const int step = (len + 63) >> 6, at = lo + (lane + 1) * step - 1;
        const bool behind = at < lo + len && cu_tokens[at + 1] <= t;
        const int n = __popcll(__ballot(behind));
        lo += n * step;
        len = min(step, len - n * step);
        if (len <= 0) return B;
    }
    const int at = lo + min(lane, len - 1), from = cu_tokens[at], to = cu_tokens[at + 1];
    const unsigned long long owners = __ballot(lane < len && from <= t && t < to);
    if (owners == 0) return B;
    const int owner = (int)__builtin_ctzll(owners);
    first = max(__builtin_amdgcn_readlane(from, owner), 0);
    return __builtin_amdgcn_readfirstlane(lo + owner);
}

// What is wrong with sequence b's own bounds or its length: READER_STATUS_BAD_LENGTH or 0.
__device__ inline int bad_sequence(const int32_t *__restrict__ cu_tokens, const int32_t *__restrict__ seq_lens, int N, int b) {
    const int lo = cu_tokens[b], hi = cu_tokens[b + 1];
    return seq_lens[b] < 0 || lo < 0 || hi < lo || hi > N ? READER_STATUS_BAD_LENGTH : 0;
}

struct QkvParams {
    const uint16_t *qkv, *q_norm, *k_norm;
    const float *cos_sin;
    const int32_t *cu_tokens;      // packed prompts, or null: trees
    const int32_t *parents, *seq_lens, *positions, *page_table;
    uint16_t *q, *k_tree, *v_tree, *k_cache, *v_cache;
    int32_t *status;
    int32_t B, T, N, Hq, Hkv, D, max_pages, max_positions, rot, interleaved;
    float eps;
    int64_t num_pages;
};
hipError_t launch_qkv(const QkvParams &p, hipStream_t stream);

struct PromptParams {
    const uint16_t *q, *k_cache, *v_cache;
    const int32_t *page_table, *cu_tokens, *seq_lens;
    uint16_t *out;
    float *lse;
    void *workspace;
    int32_t *status;
    int32_t B, N, Hq, Hkv, G, D, max_pages, max_seq_len;
    int64_t num_pages;
    float scale_log2;              // softmax scale * log2(e)
    float g_rcp;                   // 1 / G
    int32_t tokens_per_block;      // (matrix kernels) tokens whose heads fill a block of query rows
    int32_t n_ranges;              // ... and workgroups of the launch
    int32_t nodes;                 // > 0: rows are draft trees of as many nodes, lse is [B, Hq, nodes]
};
// What the attention finds wrong with sequence b, whichever kernel runs: its bounds, its length, or keys beyond the bound on them.
__device__ inline int bad_sequence(const PromptParams &p, int b) {
    const long long tokens = (long long)p.cu_tokens[b + 1] - p.cu_tokens[b];
    return p.seq_lens[b] + tokens > p.max_seq_len ? READER_STATUS_BAD_LENGTH : bad_sequence(p.cu_tokens, p.seq_lens, p.N, b);
}
// ... and with any of them, for kernels whose workgroups do not look at them all: one of them does, threads side by side.
__device__ inline void report_bad_sequences(const PromptParams &p, int threads) {
    int bad = 0;
#pragma unroll 4
    for (int b = threadIdx.x; b < p.B; b += threads) bad |= bad_sequence(p, b);
    if (bad && p.status) atomicOr(p.status, bad);
}
// 256 rows a workgroup (prompt_attn.hip), 32, 64 or 128 and blocks that are never cut (prompt_attn_mid.hip), 16 or 32
// (prompt_attn_few.hip); what the first and the last leave of cut blocks is folded by a second launch (prompt_merge.hip)
size_t prompt_wide_workspace_bytes(int D);
hipError_t launch_prompt_wide(const PromptParams &p, hipStream_t stream);
constexpr int kUncut32 = READER_PROMPT_ROWS_32_UNCUT;
hipError_t launch_prompt_mid(const PromptParams &p, int rows, hipStream_t stream);
size_t prompt_few_workspace_bytes(int D);
hipError_t launch_prompt_few(const PromptParams &p, int rows, hipStream_t stream);
hipError_t launch_prompt_merge(const PromptParams &p, int record_rows, hipStream_t stream);
hipError_t launch_prompt_attn_scalar(const PromptParams &p, hipStream_t stream);

struct KeyWeightsParams {
    const uint16_t *q, *k_cache;
    const float *lse;
    const int32_t *path, *accept_len;              // a step's accepted path, or null: the last rows of packed prompts
    const int32_t *cu_tokens;
    const int32_t *page_table, *seq_lens;
    float *weights;
    int32_t *status;
    int32_t B, T, N, Hq, Hkv, G, D, max_pages, max_path, max_seq_len, max_positions, window;
    int64_t num_pages;
    float scale_log2, decay, g_rcp;
};
hipError_t launch_key_weights(const KeyWeightsParams &p, hipStream_t stream);

struct EvictParams {
    uint16_t *k_cache, *v_cache;   // [NL, num_pages, Hkv, page_size, D]
    const int32_t *page_table;
    int32_t *seq_lens, *status;
    float *weights;                // [NL, B, Hkv, max_positions]
    int32_t *source;               // workspace: [NL * B * Hkv][keep] where each kept row comes from
    int32_t *old_len;              // ... and [NL * B * Hkv] the length before the call (0: nothing to do)
    int32_t NL, B, Hkv, D, max_pages, max_positions, keep, recent;
    int64_t num_pages;
};
hipError_t launch_kv_evict(const EvictParams &p, hipStream_t stream);

}  // namespace reader

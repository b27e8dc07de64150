// Causal attention of packed prompts over the paged cache, blocks of 32, 64 or 128 query rows that are never cut: short prompts,
// batches of them.  One launch and no records: where the blocks of a call are about as many as the chip runs at a time, cutting them evenly
// costs more than it gains (what is written and read again for a row is as much as 2 tiles of keys, and a second launch).
//
// A workgroup is 4 wavefronts of 32 rows (prompt_rows.h) that share the keys, 32 at a time, in a ring of four stages in LDS; two
// workgroups run on a compute unit and fill each other's waits.  Each wavefront copies one of the four pages of a step.
// (64 rows: of 16 each; 32: two of them take the even steps and two the odd ones, half as many one after the other.)  Bound by the
// longest block's steps, 0.75 us each with 64 rows and 1 for two with 32: one prompt of 400 tokens, 32 query and 8 kv heads of 128, 14.7
// us with 64 rows, 12 with 32, 256 tokens on 1000 positions 35 and 25; by all blocks' steps in batches: 16 prompts of 300 43 us with
// 128 rows.  (64 rows, of 32 each, the steps shared out like that: 1500 tokens 41.5 instead of 47, one shape in fourteen that the
// other three do not do better.)
#include "prompt_rows.h"

namespace reader {

namespace {

constexpr int kMidThreads = 256, kMidStages = 4;

// kBlocks: blocks of 16 query rows that a wavefront carries.  kSplit: 1, every wavefront has rows of its own and takes all steps, or
// 2, wavefronts 2 and 3 have the rows of 0 and 1 and take the other half of the steps.
template <int D, int kBlocks, int kSplit>
__device__ __forceinline__ void prompt_mid_block(const PromptParams &p) {
    using Rows = PromptRows<D, kBlocks>;
    using Page = PageLayout<D>;
    constexpr int kStageBytes = 2 * kStepPages * Page::kPageBytes;
    __shared__ __attribute__((aligned(1024))) char s_stage[kMidStages][kStageBytes];   // pages of K, then of V
    __shared__ int s_ids[4][2][64];
    const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    const int i16 = lane & 15, quad = lane >> 4, tb = p.tokens_per_block;
    int bad = 0;

    // Block number j of a kv head, the last ones first (they are the longest).  Sequence b's are numbers cu[b] / tb + b and on: no two
    // the same, some nobody's.  With two workgroups a compute unit at once, the second round runs the other way, so that a long
    // block meets a short one; heads change fastest, so that those of one run on one XCD and share its L2.
    const int n_ids = p.n_ranges;
    int j = (int)blockIdx.x / p.Hkv;
    const int head = (int)blockIdx.x - j * p.Hkv;
    {
        const int half = (kNumCU + p.Hkv - 1) / p.Hkv;
        if (n_ids > half && n_ids <= 2 * half && j >= half) j = half + (n_ids - 1 - j);
    }
    const int id = n_ids - 1 - j;
    // the last sequence whose blocks start at or in front of it
    auto first_id = [&](int b) { return clamp_row(p.cu_tokens[b], p.N) / tb + b; };
    int b = 0, len = p.B;                                // the one is among b .. b + len - 1
    while (len > 1) {
        const int step = (len + 63) >> 6, at = b + min((lane + 1) * step, len);
        const int n = (int)__popcll(__ballot((lane + 1) * step < len && first_id(min(at, p.B - 1)) <= id));
        b += n * step;
        len = min(step, len - n * step);
    }
    b = __builtin_amdgcn_readfirstlane(b);
    const int c0 = clamp_row(p.cu_tokens[b], p.N), n = max(clamp_row(p.cu_tokens[b + 1], p.N) - c0, 0), L = min(max(p.seq_lens[b], 0), p.max_seq_len);
    const int k = id - (c0 / tb + b);
    if (k < 0 || (long long)k * tb >= n) return;
    const int nt = min(tb, n - k * tb), row0 = c0 + k * tb;
    const long long p0 = (long long)L + k * tb;
    const int keys = (int)min(p0 + nt, (long long)p.max_seq_len), steps = max(1, (keys + kStep - 1) / kStep);

    const Page page(lane);
    const unsigned stage_lds = (unsigned)(size_t)(lds_char *)&s_stage[0][0];
    PageIds ids(p.page_table + (size_t)b * p.max_pages, 0, p.max_pages, &s_ids[wave][0][0]);
    // this wavefront's page of step i: page wave % 2, of K or of V
    const char *cache = reinterpret_cast<const char *>(wave < 2 ? p.k_cache : p.v_cache);
    auto issue = [&](int i, int now) {
        const int at = i * kStepPages + (wave & 1), pid = ids.get(at, now, keys, p.num_pages);
        const int rows = pid < 0 ? 0 : keys - at * READER_PAGE_SIZE;
        const char *src = cache + ((size_t)max(pid, 0) * p.Hkv + head) * Page::kPageBytes;
        const unsigned dst = stage_lds + (i & (kMidStages - 1)) * kStageBytes + wave * Page::kPageBytes;
        if (wave < 2) page.copy(src, page.k_off, rows, dst, lane);
        else page.copy(src, page.v_off, rows, dst, lane);
    };
    ids.load(0, lane);
    Rows rows;
    constexpr int kGroups = 4 / kSplit;
    const int first = wave % kGroups * 16 * kBlocks, turn = wave / kGroups;
    rows.load(p, head, row0, p0, nt, first, i16, quad);
    const int first_tok = (int)(((float)first + 0.5f) * p.g_rcp);
    const bool active = first_tok < nt;
    wait_vmcnt<0>();                                     // the first page ids are there
    asm volatile("" ::: "memory");
    ids.begin(lane);
    constexpr int kAhead = kSplit == 1 ? kMidStages - 1 : 2;             // steps asked for in front of the first
    for (int i = 0; i < min(kAhead, steps); ++i) issue(i, 0);
    const int all_see = (int)min(p0 + first_tok + 1, (long long)p.max_seq_len);   // keys that every row of this wavefront sees
    for (int i0 = 0; i0 < steps; i0 += kSplit) {
        ids.advance<kSplit>(i0, steps, lane);
        // this wavefront's pages of the steps have landed once at most those of the next two steps are on their way
        if (kSplit == 1 && i0 + 2 < steps) wait_vmcnt<2 * Page::kCopies>();
        else wait_vmcnt<0>();
        __syncthreads();                                 // ... and everybody's; nobody reads the steps in front any more
#pragma unroll
        for (int c = 0; c < kSplit; ++c)
            if (i0 + kAhead + c < steps) issue(i0 + kAhead + c, i0);
        const int i = i0 + turn, j0 = i * kStep;
        if (kSplit > 1 && i >= steps) break;
        const bool hole0 = j0 < keys && ids.get(i * kStepPages, i0, keys, p.num_pages) < 0;
        const bool hole1 = j0 + READER_PAGE_SIZE < keys && ids.get(i * kStepPages + 1, i0, keys, p.num_pages) < 0;
        if (hole0 || hole1) bad |= READER_STATUS_BAD_PAGE;
        const char *stage = s_stage[i & (kMidStages - 1)];
        rows.scores(stage, i16, quad);
        rows.weights(j0, i == turn, j0 + kStep > all_see || hole0 || hole1, hole0, hole1, p.scale_log2, quad);
        rows.template products<false>(stage + kStepPages * Page::kPageBytes, i16, quad, [] {});
    }
    if constexpr (kSplit > 1) {
        // the second half's rows come to the first through the stages, lane by lane
        f32x4 *theirs = reinterpret_cast<f32x4 *>(&s_stage[0][0]) + (size_t)(wave % kGroups) * (kBlocks * Rows::kOut + 1) * 64 + lane;
        static_assert(kGroups * (kBlocks * Rows::kOut + 1) * 64 * 16 <= kMidStages * kStageBytes && kBlocks <= 2, "they fit");
        __syncthreads();                                 // everybody is done with the keys
        if (turn > 0) {
#pragma unroll
            for (int r = 0; r < kBlocks; ++r)
#pragma unroll
                for (int db = 0; db < Rows::kOut; ++db) theirs[(r * Rows::kOut + db) * 64] = rows.acc[r][db];
            theirs[kBlocks * Rows::kOut * 64] = f32x4{rows.m[0], rows.l[0], rows.m[kBlocks - 1], rows.l[kBlocks - 1]};
        }
        __syncthreads();
        if (turn > 0) {
            if (p.status && bad) atomicOr(p.status, bad);
            return;
        }
        const f32x4 sums = theirs[kBlocks * Rows::kOut * 64];
#pragma unroll
        for (int r = 0; r < kBlocks; ++r) {
            // (a half that has seen nothing has a reference below all others and a sum of zero)
            const float m2 = sums[2 * r], l2 = sums[2 * r + 1], top = fmaxf(rows.m[r], m2);
            const float f1 = __builtin_amdgcn_exp2f(rows.m[r] - top), f2 = __builtin_amdgcn_exp2f(m2 - top);
            rows.l[r] = fmaxf(rows.l[r], l2) < kTooLarge ? rows.l[r] * f1 + l2 * f2 : __builtin_nanf("");   // (NaN: computed again)
            rows.m[r] = top;
#pragma unroll
            for (int db = 0; db < Rows::kOut; ++db) rows.acc[r][db] = rows.acc[r][db] * f1 + theirs[(r * Rows::kOut + db) * 64] * f2;
        }
    }
    if (active) {
        rows.finish_sums();
        if (rows.write(p, head, row0, nt, first, i16, quad))
            rows_the_plain_way<D>(p, ids.table, head, row0, p0, first, min(first + 16 * kBlocks, nt * p.G), 0, keys, nullptr, 0, lane, bad);
    }
    if (p.status && bad) atomicOr(p.status, bad);
}

template <int D, int kBlocks, int kSplit>
__global__ __launch_bounds__(kMidThreads, 2) void prompt_mid_kernel(PromptParams p) {
    prompt_mid_block<D, kBlocks, kSplit>(p);
    // (the last workgroup: it has one of the shortest blocks, or none)
    if (blockIdx.x == gridDim.x - 1) report_bad_sequences(p, kMidThreads);
}

template <int D, int kBlocks, int kSplit>
hipError_t launch_mid(PromptParams p, hipStream_t stream) {
    p.tokens_per_block = 64 * kBlocks / kSplit / p.G;
    p.n_ranges = p.N / p.tokens_per_block + p.B;         // (block numbers of a kv head)
    hipLaunchKernelGGL((prompt_mid_kernel<D, kBlocks, kSplit>), dim3((unsigned)p.n_ranges * p.Hkv), dim3(kMidThreads), 0, stream, p);
    return note_hip_error("launch prompt_mid_kernel", hipGetLastError());
}

}  // namespace

hipError_t launch_prompt_mid(const PromptParams &p, int rows, hipStream_t stream) {
    if (rows == kUncut32) return p.D == 64 ? launch_mid<64, 1, 2>(p, stream) : launch_mid<128, 1, 2>(p, stream);
    if (rows == 64) return p.D == 64 ? launch_mid<64, 1, 1>(p, stream) : launch_mid<128, 1, 1>(p, stream);
    return p.D == 64 ? launch_mid<64, 2, 1>(p, stream) : launch_mid<128, 2, 1>(p, stream);
}

}  // namespace reader

// Folds the parts of the blocks that the prompts' attention has cut: the ranges that hold a part of one follow one another, the
// first has noted it as open, the last as ended, and each has left a record (outputs normalised by their own sum, reference, sum).
#include "prompt_ranges.h"
#include "tree_attn_common.h"

namespace reader {

namespace {

constexpr int kMergeRows = 16, kMergeWaves = 4;

// A workgroup takes 16 rows of the block that its range left open; its four wavefronts share out the parts.  A lane holds a
// quarter of a row.
template <int D>
__global__ __launch_bounds__(64 * kMergeWaves) void prompt_merge_kernel(PromptParams p, int record_rows) {
    constexpr int kChunks = D / 16;                      // of four values, a lane's
    const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), i16 = lane & 15, quad = lane >> 4;
    const int range = blockIdx.x, row = blockIdx.y * kMergeRows + i16;
    const RangeNote *notes = reinterpret_cast<const RangeNote *>(p.workspace);
    // (this range's note and the 64 behind it are asked for together)
    const RangeNote mine = notes[range];
    auto note_at = [&](int w) { return *reinterpret_cast<const int2 *>(&notes[min(w, p.n_ranges - 1)].tiles); };   // tiles, ends
    int2 note = note_at(range + 1 + lane);
    if (!mine.open || blockIdx.y * kMergeRows >= mine.nt * p.G) return;
    const size_t record_floats = (size_t)record_rows * (D + 2);
    const float *records = reinterpret_cast<const float *>(reinterpret_cast<const char *>(p.workspace) + kNotesBytes);
    float m = -INFINITY, l = 0.f;
    float4 acc[kChunks] = {};                            // weighted by l
    auto fold = [&](float m2, float l2, const float4 (&v)[kChunks]) {
        // (a part that the row sees nothing of has a sum of zero; a sum that is not a number shows)
        if (l2 == 0.f) return;
        const float top = fmaxf(m, m2);
        const float a = l == 0.f ? 0.f : __builtin_amdgcn_exp2f(m - top), b = l2 * __builtin_amdgcn_exp2f(m2 - top);
#pragma unroll
        for (int c = 0; c < kChunks; ++c) {
            acc[c].x = acc[c].x * a + v[c].x * b; acc[c].y = acc[c].y * a + v[c].y * b;
            acc[c].z = acc[c].z * a + v[c].z * b; acc[c].w = acc[c].w * a + v[c].w * b;
        }
        l = l * a + b;
        m = top;
    };
    struct Part {
        float m, l;
        float4 v[kChunks];
    };
    auto load = [&](int w, Part &o) {
        const float *rec = records + (size_t)(2 * w + (w == range ? 1 : 0)) * record_floats;
        o.m = rec[(size_t)record_rows * D + row];
        o.l = rec[(size_t)record_rows * (D + 1) + row];
        const float4 *from = reinterpret_cast<const float4 *>(rec) + (size_t)quad * kChunks * record_rows + row;
#pragma unroll
        for (int c = 0; c < kChunks; ++c) o.v[c] = from[(size_t)c * record_rows];
    };
    // (a part is asked for before the one in front of it is folded)
    Part held, next;
    bool any = wave == 0;
    if (any) load(range, held);
    auto part = [&](int w) {
        load(w, next);
        if (any) fold(held.m, held.l, held.v);
        held = next;
        any = true;
    };
    // the ranges behind it, 64 notes at a time, up to the one that ends the block
    for (int base = range + 1, turn = 1; base < p.n_ranges; base += 64) {
        const bool there = base + lane < p.n_ranges && note.x > 0;
        unsigned long long parts = __ballot(there), ends = __ballot(there && note.y != 0);
        if (ends) parts &= (2ull << __builtin_ctzll(ends)) - 1ull;   // (nothing behind the first that ends)
        for (; parts; parts &= parts - 1, ++turn)
            if (turn % kMergeWaves == wave) part(base + (int)__builtin_ctzll(parts));
        if (ends) break;
        note = note_at(base + 64 + lane);
    }
    if (any) fold(held.m, held.l, held.v);
    // the four wavefronts' sums, in their order
    __shared__ float s_part[kMergeWaves - 1][4 * kChunks + 2][64];
    if (wave > 0) {
        float *o = &s_part[wave - 1][0][lane];
        o[0] = m;
        o[64] = l;
#pragma unroll
        for (int c = 0; c < kChunks; ++c) {
            o[(4 * c + 2) * 64] = acc[c].x; o[(4 * c + 3) * 64] = acc[c].y;
            o[(4 * c + 4) * 64] = acc[c].z; o[(4 * c + 5) * 64] = acc[c].w;
        }
    }
    __syncthreads();
    if (wave > 0) return;
#pragma unroll
    for (int g = 0; g < kMergeWaves - 1; ++g) {
        const float *o = &s_part[g][0][lane];
        const float m2 = o[0], l2 = o[64];
        if (l2 == 0.f) continue;
        const float top = fmaxf(m, m2);
        const float a = l == 0.f ? 0.f : __builtin_amdgcn_exp2f(m - top), b = __builtin_amdgcn_exp2f(m2 - top);
#pragma unroll
        for (int c = 0; c < kChunks; ++c) {
            acc[c].x = acc[c].x * a + o[(4 * c + 2) * 64] * b; acc[c].y = acc[c].y * a + o[(4 * c + 3) * 64] * b;
            acc[c].z = acc[c].z * a + o[(4 * c + 4) * 64] * b; acc[c].w = acc[c].w * a + o[(4 * c + 5) * 64] * b;
        }
        l = l * a + l2 * b;
        m = top;
    }
    const int tok = (int)(((float)row + 0.5f) * p.g_rcp), g = row - tok * p.G;
    if (tok >= mine.nt) return;
    const float inv = l == 0.f ? 0.f : 1.f / l;
    const size_t out_row = ((size_t)mine.row0 + tok) * p.Hq + (size_t)mine.head * p.G + g;
    uint16_t *out = p.out + out_row * D + quad * kChunks * 4;
#pragma unroll
    for (int c = 0; c < kChunks; c += 2)
        *reinterpret_cast<uint4 *>(out + c * 4) =
            make_uint4(pack_bf16x2(acc[c].x * inv, acc[c].y * inv), pack_bf16x2(acc[c].z * inv, acc[c].w * inv),
                       pack_bf16x2(acc[c + 1].x * inv, acc[c + 1].y * inv), pack_bf16x2(acc[c + 1].z * inv, acc[c + 1].w * inv));
    if (quad == 0 && p.lse) p.lse[out_row] = l == 0.f ? -INFINITY : (m + __builtin_amdgcn_logf(l)) * kLn2;
}

}  // namespace

hipError_t launch_prompt_merge(const PromptParams &p, int record_rows, hipStream_t stream) {
    const dim3 grid(p.n_ranges, record_rows / kMergeRows);
    if (p.D == 64) hipLaunchKernelGGL(prompt_merge_kernel<64>, grid, dim3(64 * kMergeWaves), 0, stream, p, record_rows);
    else hipLaunchKernelGGL(prompt_merge_kernel<128>, grid, dim3(64 * kMergeWaves), 0, stream, p, record_rows);
    return note_hip_error("launch prompt_merge_kernel", hipGetLastError());
}

}  // namespace reader

// Causal attention of packed prompts over the paged cache for few query rows a kv head: single tokens, short chunks.
//
// Bound by memory: every key and value feeds a handful of rows.  A workgroup takes a range of the (head, sequence, block, key) axis
// (prompt_ranges.h; a block is 16 or 32 rows here) and its four wavefronts take the steps of 32 keys in turn, each through two stages
// of its own in LDS, waiting for nobody; at the end of a segment they add up their rows.  (Wavefronts with ranges of their own
// cut the blocks into four times as many parts: one token on 32 K positions 53 us instead of 37, 16 on 1 to 16 K 104 instead of
// 99.)  Blocks that are cut leave fp32 records for a second launch.  16 single tokens on 1 to 16 K positions, 32 query and 8 kv
// heads of 128: 97 us, 5.9 TB/s, 87 of them this launch.
#include "prompt_rows.h"

namespace reader {

namespace {

using Block = PromptBlock<kStep, 2 * kStep, 4 * kStep>;
constexpr int kWaves = 4;
// Workgroups of the launch, a range each: as many as run at once, by their stages in the LDS.
constexpr int few_ranges(int D) { return kNumCU * (D == 128 ? 1 : 2); }
static_assert(few_ranges(64) <= kMaxRanges && few_ranges(128) <= kMaxRanges, "the workspace has a note for each");

// kBlocks: blocks of 16 query rows
template <int D, int kBlocks>
__global__ __launch_bounds__(64 * kWaves) void prompt_few_kernel(PromptParams p) {
    using Rows = PromptRows<D, kBlocks>;
    using Page = PageLayout<D>;
    constexpr int kStageBytes = 2 * kStepPages * Page::kPageBytes, kStageCopies = 2 * kStepPages * Page::kCopies, kRows = kBlocks * 16;
    constexpr int kMinRange = 2 * kStep * kWaves;        // two steps a wavefront (one or four: the same within 4 %)
    __shared__ __attribute__((aligned(1024))) char s_stage[kWaves][2][kStageBytes];   // pages of K, then of V
    __shared__ int s_ids[kWaves][2][64];
    __shared__ float s_sum[kWaves][2][kRows];            // the rows' references and sums
    __shared__ int s_odd;
    const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    const int i16 = lane & 15, quad = lane >> 4, tb = p.tokens_per_block;
    RangeNote *const notes = reinterpret_cast<RangeNote *>(p.workspace);
    const Sequences seqs{p.seq_lens, p.cu_tokens, p.N, p.max_seq_len};
    int bad = 0;

    // ---- this workgroup's range of the axis (every wavefront finds it for itself)
    long long per_head = 0;
    auto cost_up_to = [&](int base) {                    // of sequences `base` .. base + lane, and what they have wrong
        const int b = base + lane;
        long long c = 0;
        if (b < p.B) {
            c = Block::sequence_cost(seqs.length(b), seqs.tokens(b), tb);
            bad |= bad_sequence(p, b);
        }
        return scan64(c);
    };
    const long long upto0 = cost_up_to(0);
    per_head = lane64(upto0, 63);
    for (int base = 64; base < p.B; base += 64) per_head += lane64(cost_up_to(base), 63);
    if (bad && blockIdx.x == 0 && p.status) atomicOr(p.status, bad);
    bad = 0;
    const long long total = per_head * p.Hkv;
    long long n_ranges = total / kMinRange;
    n_ranges = n_ranges > (long long)gridDim.x ? gridDim.x : (n_ranges < 1 ? 1 : n_ranges);
    const int range = blockIdx.x;
    if (range >= n_ranges || total == 0) {
        if (threadIdx.x == 0) notes[range] = RangeNote{};
        return;
    }
    const PromptAxis axis(per_head, p.Hkv, (int)n_ranges);
    // the places where the range begins and, in lanes 32..63, where the next one does: head, sequence, then the tile
    Block place = {p.Hkv, 0, 0, 0, 0, 0};
    int t_place = 0;
    {
        const long long x = axis.begin(range + (lane >> 5));
        long long r = 0;
        if (x < total) place.head = axis.head(x, r);
        long long before = 0;
#pragma unroll
        for (int half = 0; half < 2; ++half) {
            const long long r_half = lane64(r, 32 * half);
            long long carry = 0, upto = upto0;
            for (int base = 0;; base += 64) {
                if (base > 0) upto = cost_up_to(base);
                const long long all = carry + lane64(upto, 63);
                if (r_half < all) {                      // (the last of these 64 at the latest: r is below per_head)
                    const int i = (int)__popcll(__ballot(carry + upto <= r_half));
                    if (i > 0) carry += lane64(upto, i - 1);
                    if ((lane >> 5) == half) place.b = base + i, before = carry;
                    break;
                }
                carry = all;
            }
        }
        if (x < total) {
            place.load(seqs);
            t_place = place.locate(r - before, seqs, p.B, tb);
        } else place.b = 0;
    }
    const PromptRange<Block> rg(place, t_place, p.Hkv);
    const RangeNote note = rg.note(seqs, p.B, tb, lane);
    if (threadIdx.x == 0) notes[range] = note;

    const Page page(lane);
    const unsigned stage_lds = (unsigned)(size_t)(lds_char *)&s_stage[wave][0][0];

    Block o = rg.at;
    for (bool first_block = true; !rg.behind(o); first_block = false) {
        int t0, t1;
        rg.share(o, first_block, tb, p.max_seq_len, t0, t1);
        const int keys = o.keys(tb, p.max_seq_len), nt = o.tokens(tb), row0 = o.c0 + o.k * tb, all = o.tiles(tb, p.max_seq_len);
        const long long p0 = (long long)o.L + o.k * tb;
        const bool last_block = rg.is_stop(o);
        if (t1 > t0) {
            // steps wave, wave + kWaves, ... of the segment are this wavefront's
            const int steps = (t1 - t0 - wave + kWaves - 1) / kWaves;
            PageIds ids(p.page_table + (size_t)o.b * p.max_pages, t0 * kStepPages, p.max_pages, &s_ids[wave][0][0]);
            auto issue = [&](int j, int now) {           // (at step `now`) kStageCopies copy instructions, whatever the pages are
                const int i = wave + j * kWaves;
                const unsigned stage = stage_lds + (j & 1) * kStageBytes;
#pragma unroll
                for (int pg = 0; pg < kStepPages; ++pg) {
                    const int at = i * kStepPages + pg, id = ids.get(at, now, keys, p.num_pages);
                    const int rows = id < 0 ? 0 : keys - (ids.page0 + at) * READER_PAGE_SIZE;
                    const size_t off = ((size_t)max(id, 0) * p.Hkv + o.head) * Page::kPageBytes;
                    page.copy(reinterpret_cast<const char *>(p.k_cache) + off, page.k_off, rows, stage + pg * Page::kPageBytes, lane);
                    page.copy(reinterpret_cast<const char *>(p.v_cache) + off, page.v_off, rows, stage + (kStepPages + pg) * Page::kPageBytes, lane);
                }
            };
            ids.load(0, lane);
            Rows rows;
            rows.load(p, o.head, row0, p0, nt, 0, i16, quad);
            wait_vmcnt<0>();                             // the first page ids are there (and the last segment's copies)
            asm volatile("" ::: "memory");
            ids.begin(lane);
            if (steps > 0) issue(0, 0);
            if (steps > 1) issue(1, 0);
            for (int j = 0; j < steps; ++j) {
                const int i = wave + j * kWaves;
                ids.advance<kWaves>(i, t1 - t0, lane);
                if (j + 1 < steps) wait_vmcnt<kStageCopies>();
                else wait_vmcnt<0>();
                asm volatile("" ::: "memory");
                const int j0 = (t0 + i) * kStep;
                const bool hole0 = j0 < keys && ids.get(i * kStepPages, i, keys, p.num_pages) < 0;
                const bool hole1 = j0 + READER_PAGE_SIZE < keys && ids.get(i * kStepPages + 1, i, keys, p.num_pages) < 0;
                if (hole0 || hole1) bad |= READER_STATUS_BAD_PAGE;
                const bool masked = j0 + kStep > p0 + 1 || j0 + kStep > p.max_seq_len || hole0 || hole1;
                const char *stage = s_stage[wave][j & 1];
                rows.scores(stage, i16, quad);
                rows.weights(j0, j == 0, masked, hole0, hole1, p.scale_log2, quad);
                rows.template products<true>(stage + kStepPages * Page::kPageBytes, i16, quad, [&] { if (j + 2 < steps) issue(j + 2, i); });
            }
            rows.finish_sums();
            // ---- end of the segment: the whole block is normalised and written out, a part of one leaves a record
            const bool whole = t0 == 0 && t1 == all;
            float *rec = reinterpret_cast<float *>(reinterpret_cast<char *>(p.workspace) + kNotesBytes) +
                         (size_t)(2 * range + (t0 == 0 ? 1 : 0)) * ((size_t)kRows * (D + 2));
            bool odd = false;
            // the wavefronts' rows meet where their keys were: [D / 4 chunks][rows][4 values]
            f32x4 *mine = reinterpret_cast<f32x4 *>(&s_stage[wave][0][0]);
            static_assert(kRows * D * 4 <= 2 * kStageBytes, "a wavefront's rows fit its stages");
            if (threadIdx.x == 0) s_odd = 0;
#pragma unroll
            for (int r = 0; r < kBlocks; ++r) {
#pragma unroll
                for (int db = 0; db < Rows::kOut; ++db) mine[(db * 4 + quad) * kRows + r * 16 + i16] = rows.acc[r][db];
                if (quad == 0) { s_sum[wave][0][r * 16 + i16] = rows.m[r]; s_sum[wave][1][r * 16 + i16] = rows.l[r]; }
            }
            __syncthreads();
#pragma unroll
            for (int r = 0; r < kBlocks; ++r) {
                const int row = r * 16 + i16;
                const size_t at = Rows::out_row(p, o.head, row0, nt, 0, r, i16);
                float top = kNoReference, sum = 0.f, f[kWaves], check = 0.f;   // (check: not a number once any value is none)
#pragma unroll
                for (int w = 0; w < kWaves; ++w) top = fmaxf(top, s_sum[w][0][row]);
#pragma unroll
                for (int w = 0; w < kWaves; ++w) {
                    // (a wavefront whose rows saw nothing has no say, whatever its reference; a sum that is not a number shows)
                    const float lw = s_sum[w][1][row];
                    check = lw < kTooLarge ? check : __builtin_nanf("");
                    f[w] = lw == 0.f ? 0.f : __builtin_amdgcn_exp2f(s_sum[w][0][row] - top);
                    sum += lw * f[w];
                }
                const float inv = sum == 0.f ? 0.f : 1.f / sum;
                // a wavefront takes D / 4 / kWaves chunks of the columns, a lane those of its quarter of them
                constexpr int kMine = D / 16 / kWaves;
                f32x4 v[kMine];
#pragma unroll
                for (int c = 0; c < kMine; ++c) {
                    const int chunk = (wave * 4 + quad) * kMine + c;
                    v[c] = f32x4{0.f, 0.f, 0.f, 0.f};
#pragma unroll
                    for (int w = 0; w < kWaves; ++w) v[c] += reinterpret_cast<const f32x4 *>(&s_stage[w][0][0])[chunk * kRows + row] * f[w];
                    v[c] *= inv;
                    check = check + v[c][0] * 0.f + v[c][1] * 0.f + v[c][2] * 0.f + v[c][3] * 0.f;
                    if (!whole) reinterpret_cast<f32x4 *>(rec)[chunk * kRows + row] = v[c];
                    else if (rows.real[r])
                        *reinterpret_cast<uint2 *>(p.out + at * D + chunk * 4) = make_uint2(pack_bf16x2(v[c][0], v[c][1]), pack_bf16x2(v[c][2], v[c][3]));
                }
                if (wave == 0 && quad == 0) {
                    if (!whole) {
                        rec[(size_t)kRows * D + row] = sum == 0.f ? -INFINITY : top;
                        rec[(size_t)kRows * (D + 1) + row] = sum;
                    } else if (rows.real[r] && p.lse) {
                        p.lse[at] = sum == 0.f ? -INFINITY : (top + __builtin_amdgcn_logf(sum)) * kLn2;
                    }
                }
                odd = odd || (rows.real[r] && !(check == 0.f));
            }
            if (odd) s_odd = 1;
            wait_vmcnt<0>();                         // (should wavefront 0 write the rows again, it writes behind the others)
            __syncthreads();                         // everybody is done with the others' rows: the stages are free
            odd = wave == 0 && s_odd != 0;
            if (odd) rows_the_plain_way<D>(p, ids.table, o.head, row0, p0, 0, nt * p.G, t0 * kStep, t1 * kStep, whole ? nullptr : rec, kRows, lane, bad);
        }
        if (last_block) break;
        o.next(seqs, p.B, tb);
        o = o.of_lane(0);
    }
    if (p.status && bad) atomicOr(p.status, bad);
}

template <int D, int kBlocks>
hipError_t launch_few(PromptParams p, hipStream_t stream) {
    p.n_ranges = few_ranges(D);
    hipLaunchKernelGGL((prompt_few_kernel<D, kBlocks>), dim3(p.n_ranges), dim3(64 * kWaves), 0, stream, p);
    const hipError_t e = hipGetLastError();
    if (e != hipSuccess) return note_hip_error("launch prompt_few_kernel", e);
    return launch_prompt_merge(p, kBlocks * 16, stream);
}

}  // namespace

hipError_t launch_prompt_few(const PromptParams &params, int rows, hipStream_t stream) {
    PromptParams p = params;
    p.tokens_per_block = rows / p.G;
    if (rows == 16) return p.D == 64 ? launch_few<64, 1>(p, stream) : launch_few<128, 1>(p, stream);
    return p.D == 64 ? launch_few<64, 2>(p, stream) : launch_few<128, 2>(p, stream);
}

size_t prompt_few_workspace_bytes(int D) { return ranges_workspace_bytes(few_ranges(D), 32, D); }

}  // namespace reader

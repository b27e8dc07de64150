// Attention over a cache in 4 bits for many query rows a kv head: trees of many nodes, chunks of prompts.
//
// Bound by the matrix units.  A workgroup takes a range of the (head, sequence, block of rows, key) axis with 4 wavefronts, one per
// SIMD, of 16 kBlocks rows each.  They share the keys: bytes come into a ring in LDS by asynchronous copies, every wavefront
// makes a quarter of each step's operands of them (32 keys; two codes an instruction, exact in bf16) and leaves them in LDS as the
// matrix instructions read them, 1 KB an operand, conflict-free.  The scores of step s + 1 are computed beside the weights of
// step s, the operands of step s + 2 made beside the second product of step s; one barrier a step.
#include "kvq_attn.h"

namespace reader {

namespace {

using WideBlock = PromptBlock<kStep, 2 * kStep, 8 * kStep>;
constexpr int kWaves = 4, kThreadsWide = 64 * kWaves;

template <int D>
struct WideLayout {
    static constexpr int kFrag = 1024;                                            // an operand: 16 bytes a lane
    static constexpr int kKSteps = D / 32, kKFrags = kStepPages * kKSteps, kVFrags = D / 16;
    static constexpr int kStepBytes = (kKFrags + kVFrags) * kFrag, kBuffers = 3;
    static constexpr int kCodes = kStepPages * 16 * D, kRaw = kCodes + 256;       // codes of two pages, their scales (D bytes each)
    static constexpr int kSlots = 8, kDepth = 5;                                  // raw steps in the ring; asked for as many steps before they are used
};

template <int D, int kBlocks>
struct WideRows {
    static constexpr int kKSteps = D / 32, kOut = D / 16;
    bf16x8 q[kBlocks][kKSteps];
    f32x4 acc[kBlocks][kOut];
    float m[kBlocks], l[kBlocks];
    u32x4 pk[kBlocks];
    using Scores = f32x4[kBlocks][kStepPages];

    __device__ static __forceinline__ int token(const PromptParams &p, int row) { return (int)(((float)row + 0.5f) * p.g_rcp); }   // row / G
    __device__ static __forceinline__ size_t out_row(const PromptParams &p, int head, int row0, int nt, int row) {
        const int tok = token(p, row);
        return ((size_t)row0 + min(tok, nt - 1)) * p.Hq + (size_t)head * p.G + (row - tok * p.G);
    }
    __device__ __forceinline__ void load(const PromptParams &p, int head, int row0, int nt, int first, int i16, int quad) {
#pragma unroll
        for (int r = 0; r < kBlocks; ++r) {
            const int row = first + r * 16 + i16;
            const bool real = token(p, row) < nt;
            const size_t at = out_row(p, head, row0, nt, row);
#pragma unroll
            for (int s = 0; s < kKSteps; ++s) q[r][s] = __builtin_bit_cast(bf16x8, keep_if(real, ld16(p.q + at * D + quad * (D / 4) + s * 8)));
            m[r] = kNoReference;
            l[r] = 0.f;
#pragma unroll
            for (int i = 0; i < kOut; ++i) acc[r][i] = f32x4{0.f, 0.f, 0.f, 0.f};
        }
    }
    __device__ __forceinline__ void scores(Scores &x, const char *k, int lane) const {
#pragma unroll
        for (int pg = 0; pg < kStepPages; ++pg) {
#pragma unroll
            for (int r = 0; r < kBlocks; ++r) x[r][pg] = f32x4{0.f, 0.f, 0.f, 0.f};
#pragma unroll
            for (int s = 0; s < kKSteps; ++s) {
                const bf16x8 key = *reinterpret_cast<const bf16x8 *>(k + (pg * kKSteps + s) * 1024 + lane * 16);
#pragma unroll
                for (int r = 0; r < kBlocks; ++r) x[r][pg] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(key, q[r][s], x[r][pg], 0, 0, 0);
            }
        }
    }
    __device__ __forceinline__ float weights(const Scores &x, float c2, float (&sum)[kBlocks]) {
        float most = 0.f;
#pragma unroll
        for (int r = 0; r < kBlocks; ++r) {
            float w[8];
            sum[r] = l[r];
#pragma unroll
            for (int e = 0; e < 8; ++e) {
                w[e] = __builtin_amdgcn_exp2f(x[r][e / 4][e % 4] * c2 - m[r]);
                sum[r] += w[e];
            }
#pragma unroll
            for (int e = 0; e < 4; ++e) pk[r][e] = pack_bf16x2(w[2 * e], w[2 * e + 1]);
            most = fmaxf(most, sum[r]);
        }
        return most;
    }
    __device__ __forceinline__ void products(const char *v, int lane) {
#pragma unroll
        for (int i = 0; i < kOut; ++i) {
            const bf16x8 val = *reinterpret_cast<const bf16x8 *>(v + i * 1024 + lane * 16);
#pragma unroll
            for (int r = 0; r < kBlocks; ++r) acc[r][i] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(val, __builtin_bit_cast(bf16x8, pk[r]), acc[r][i], 0, 0, 0);
        }
    }
    // Moves the references so that no weight of these scores is above one, nor a row's sum.
    __device__ __forceinline__ void move_references(const Scores &x, float c2) {
#pragma unroll
        for (int r = 0; r < kBlocks; ++r) {
            float mx = fmaxf(fmaxf(x[r][0][0], x[r][0][1]), fmaxf(x[r][0][2], x[r][0][3]));
            mx = fmaxf(mx, fmaxf(fmaxf(x[r][1][0], x[r][1][1]), fmaxf(x[r][1][2], x[r][1][3]))) * c2;
            mx = fmaxf(mx, m[r] + __builtin_amdgcn_logf(l[r]));              // (minus infinity where the sum is zero)
            mx = fmaxf(mx, __shfl_xor(mx, 16));
            mx = fmaxf(mx, __shfl_xor(mx, 32));
            const float top = fmaxf(m[r], mx), f = __builtin_amdgcn_exp2f(m[r] - top);
            l[r] *= f;
            m[r] = top;
#pragma unroll
            for (int i = 0; i < kOut; ++i) acc[r][i] *= f;
            __builtin_amdgcn_sched_barrier(0);
        }
    }
};

// This wavefront's part of a step's operands: `raw` holds the codes of two pages and their scales; valid0, valid1: keys of each page that
// somebody sees.
template <int D>
__device__ __forceinline__ void make_operands(const char *raw, char *to, int wave, int lane, int i16, int quad, int valid0, int valid1) {
    using W = WideLayout<D>;
    const int pg = wave >> 1, sub = wave & 1;
    const char *scales = raw + W::kCodes;
    {   // K: half of a page's k-steps
        const float sc = scale_of(*reinterpret_cast<const uint8_t *>(scales + pg * D + (D == 128 ? quad : quad >> 1) * 16 + i16));
#pragma unroll
        for (int h = 0; h < W::kKSteps / 2; ++h) {
            const uint32_t w = *reinterpret_cast<const uint32_t *>(raw + pg * (16 * D) + lane * (D / 8) + (sub * (W::kKSteps / 2) + h) * 4);
            *reinterpret_cast<u32x4 *>(to + (pg * W::kKSteps + sub * (W::kKSteps / 2) + h) * W::kFrag + lane * 16) =
                u32x4{two_values<0>(w, sc), two_values<1>(w, sc), two_values<2>(w, sc), two_values<3>(w, sc)};
        }
    }
    // V: a quarter of the columns of every chunk, of both pages
    u32x4 even, odd;
#pragma unroll
    for (int g = 0; g < kStepPages; ++g) {
        const char *v = raw + g * (16 * D) + 8 * D;
        uint32_t vs = *reinterpret_cast<const uint32_t *>(scales + g * D + D / 2 + quad * (D / 8) + (i16 * (D / 16) / 32) * 4);
        const int n = (g == 0 ? valid0 : valid1) - 4 * quad;
        uint32_t word[4];
        if constexpr (D == 128) {
            const u32x4 c = *reinterpret_cast<const u32x4 *>(v + lane * 16);
#pragma unroll
            for (int e = 0; e < 4; ++e) word[e] = c[e] >> (8 * wave);
        } else {
            const uint2 c = *reinterpret_cast<const uint2 *>(v + lane * 8);
            word[0] = c.x >> (8 * (wave >> 1)); word[1] = c.x >> (16 + 8 * (wave >> 1));
            word[2] = c.y >> (8 * (wave >> 1)); word[3] = c.y >> (16 + 8 * (wave >> 1));
        }
        uint32_t y[4];
#pragma unroll
        for (int e = 0; e < 4; ++e) {
            // (a key that nobody sees: what its bytes hold must not meet a weight of zero)
            y[e] = two_values<0>(word[e], scale_of(vs >> (8 * e) & 255u));
            y[e] = e < n ? y[e] : 0u;
        }
        even[2 * g] = __builtin_amdgcn_perm(y[1], y[0], 0x05040100);
        even[2 * g + 1] = __builtin_amdgcn_perm(y[3], y[2], 0x05040100);
        odd[2 * g] = __builtin_amdgcn_perm(y[1], y[0], 0x07060302);
        odd[2 * g + 1] = __builtin_amdgcn_perm(y[3], y[2], 0x07060302);
    }
    char *vt = to + W::kKFrags * W::kFrag + lane * 16;
    if constexpr (D == 128) {
        *reinterpret_cast<u32x4 *>(vt + (2 * wave) * W::kFrag) = even;
        *reinterpret_cast<u32x4 *>(vt + (2 * wave + 1) * W::kFrag) = odd;
    } else {
        *reinterpret_cast<u32x4 *>(vt + wave * W::kFrag) = sub ? odd : even;
    }
}

template <int D, int kBlocks, bool kTree>
__global__ __launch_bounds__(kThreadsWide) __attribute__((amdgpu_waves_per_eu(1, 1))) void kvq_attn_wide_kernel(KvqAttnParams p) {
    using Rows = WideRows<D, kBlocks>;
    using W = WideLayout<D>;
    constexpr int kWaveRows = kBlocks * 16, kRows = kWaveRows * kWaves, kMinRange = 4 * kStep;
    __shared__ __attribute__((aligned(1024))) char s_frag[W::kBuffers][W::kStepBytes];
    __shared__ __attribute__((aligned(1024))) char s_raw[W::kSlots][W::kRaw];
    __shared__ int s_ids[kWaves][2][64];
    __shared__ uint32_t s_mask[kTree ? READER_MAX_T : 1][4];
    __shared__ int s_up[kTree ? READER_MAX_T : 1];
    const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    const int i16 = lane & 15, quad = lane >> 4, tb = p.tokens_per_block;
    const Sequences seqs{p.seq_lens, p.cu_tokens, p.N, p.max_seq_len, kTree ? p.nodes : 0};
    const int range = blockIdx.x;
    WideBlock place;
    int t_place;
    if (!find_range<WideBlock, kMinRange, kTree>(p, seqs, lane, place, t_place)) return;
    const PromptRange<WideBlock> rg(place, t_place, p.Hkv);
    const RangeNote note = rg.note(seqs, p.B, tb, lane);
    if (threadIdx.x == 0) reinterpret_cast<RangeNote *>(p.workspace)[range] = note;
    int bad = 0;
    const unsigned raw_lds = (unsigned)(size_t)(lds_char *)&s_raw[0][0];
    // this lane's bytes of a step's copies: codes of page copy_page, 16 bytes; scales of both pages, 4 bytes
    const int copy_page = D == 128 ? wave >> 1 : wave & 1, copy_part = D == 128 ? wave & 1 : 0;
    const int scale_page = D == 128 ? lane >> 5 : lane >> 4 & 1, scale_word = D == 128 ? lane & 31 : lane & 15;

    WideBlock o = rg.at;
    for (bool first_block = true; !rg.behind(o); first_block = false) {
        int t0, t1;
        rg.share(o, first_block, tb, p.max_seq_len, t0, t1);
        const int keys = o.keys(tb, p.max_seq_len), nt = o.tokens(tb), row0 = o.c0 + o.k * tb, all = o.tiles(tb, p.max_seq_len);
        const long long p0 = (long long)o.L + o.k * tb;
        const bool last_block = rg.is_stop(o);
        if (t1 > t0) {
            if constexpr (kTree) {
                if ((long long)t1 * kStep > o.L) ancestors(p.parents + (size_t)o.b * p.nodes, p.nodes, s_mask, s_up, bad);
            }
            const int first = wave * kWaveRows, steps = t1 - t0;
            const int unmasked = kTree ? o.L : (int)min(p0 + 1, (long long)p.max_seq_len);     // keys that every row sees
            PageIds ids(p.page_table + (size_t)o.b * p.max_pages, t0 * kStepPages, p.max_pages, &s_ids[wave][0][0]);
            auto page_id = [&](int step, int now, int pg) { return ids.get(step * kStepPages + pg, now, keys, p.num_pages); };
            auto block_of = [&](int id) { return reinterpret_cast<const char *>(p.cache) + ((size_t)max(id, 0) * p.Hkv + o.head) * KvqBlock<D>::kBytes; };
            auto issue = [&](int step, int now) {        // (at step `now`) two copy instructions, whatever the pages are
                const unsigned slot = raw_lds + (step % W::kSlots) * W::kRaw;
                const char *b0 = block_of(page_id(step, now, 0)), *b1 = block_of(page_id(step, now, 1));
                copy16_uniform((copy_page ? b1 : b0) + copy_part * 1024, lane * 16, slot + copy_page * (16 * D) + copy_part * 1024);
                const char *from = (scale_page ? b1 : b0) + 16 * D + scale_word * 4;
                asm volatile("s_mov_b32 m0, %1\n\tglobal_load_lds_dword %0, off" :: "v"(from), "s"(slot + W::kCodes) : "memory", "m0");
            };
            auto make = [&](int step, int now) {         // (at step `now`) this wavefront's operands of a step
                const int j0 = (t0 + step) * kStep;
                const int v0 = page_id(step, now, 0) < 0 ? 0 : keys - j0, v1 = page_id(step, now, 1) < 0 ? 0 : keys - j0 - READER_PAGE_SIZE;
                make_operands<D>(s_raw[step % W::kSlots], s_frag[step % W::kBuffers], wave, lane, i16, quad, v0, v1);
            };
            auto meet = [&] {
                __builtin_amdgcn_fence(__ATOMIC_RELEASE, "workgroup", "local");
                __builtin_amdgcn_s_barrier();
                __builtin_amdgcn_fence(__ATOMIC_ACQUIRE, "workgroup", "local");
                asm volatile("" ::: "memory");
            };
            ids.load(0, lane);
            Rows rows;
            rows.load(p, o.head, row0, nt, first, i16, quad);
            wait_vmcnt<0>();                             // the first page ids are there
            asm volatile("" ::: "memory");
            ids.begin(lane);
            for (int s = 0; s < W::kDepth + 2; ++s) issue(s, 0);
            wait_vmcnt<2 * (W::kDepth - 1)>();           // steps 0, 1 and 2
            asm volatile("" ::: "memory");
            meet();
            make(0, 0);
            make(1, 0);
            meet();
            auto masked = [&](int s) {
                const int j0 = (t0 + s) * kStep;
                return j0 + kStep > unmasked || page_id(s, s, 0) < 0 || page_id(s, s, 1) < 0;
            };
            bool move = true;                            // (the references are yet to be found)
            int s = 0;
            typename Rows::Scores x0, x1;
            // One step: the weights of the scores `xa` of step s, the scores `xb` of step s + 1, the products.  true: on with the next one.
            auto step = [&](const typename Rows::Scores &xa, typename Rows::Scores &xb) -> bool {
                rows.scores(xb, s_frag[(s + 1) % W::kBuffers], lane);
                float sum[kBlocks];
                if (__any(rows.weights(xa, p.scale_log2, sum) > kMostSum)) {
                    move = true;
                    return false;
                }
#pragma unroll
                for (int r = 0; r < kBlocks; ++r) rows.l[r] = sum[r];
                issue(s + 2 + W::kDepth, s);
                make(s + 2, s);
                rows.products(s_frag[s % W::kBuffers] + W::kKFrags * W::kFrag, lane);
                wait_vmcnt<2 * (W::kDepth - 1)>();       // step s + 3 has come
                asm volatile("" ::: "memory");
                meet();
                ++s;
                if (s >= steps) return false;
                ids.template advance<1>(s, steps, lane);
                return !masked(s);
            };
            ids.template advance<1>(0, steps, lane);
            // (references are moved, and scores masked, outside the loop over the steps, with the scores computed again: a path around the
            // accumulators inside it is paid for in every step)
            while (s < steps) {
                rows.scores(x0, s_frag[s % W::kBuffers], lane);
                if (masked(s)) {
                    const int j0 = (t0 + s) * kStep;
                    const bool hole0 = page_id(s, s, 0) < 0, hole1 = page_id(s, s, 1) < 0;
                    if ((j0 < keys && hole0) || (j0 + READER_PAGE_SIZE < keys && hole1)) bad |= READER_STATUS_BAD_PAGE;
#pragma unroll
                    for (int r = 0; r < kBlocks; ++r) {
                        int row = first + r * 16 + i16;
                        asm("" : "+v"(row));
                        const int tok = min(Rows::token(p, row), nt - 1), lim = (int)min(p0 + tok + 1, (long long)p.max_seq_len);
                        const uint32_t *mask = s_mask[kTree ? o.k * tb + tok : 0];
#pragma unroll
                        for (int e = 0; e < 8; ++e) {
                            const int key = j0 + (e / 4) * READER_PAGE_SIZE + quad * 4 + e % 4, n = key - o.L;
                            // (no branches: with them the compiler has lost the assignment on one of the ways)
                            bool sees = !(e < 4 ? hole0 : hole1) & (key < lim);
                            if constexpr (kTree) sees &= (n < 0) | ((mask[(n >> 5) & 3] >> (n & 31) & 1u) != 0);
                            x0[r][e / 4][e % 4] = sees ? x0[r][e / 4][e % 4] : -INFINITY;
                        }
                        asm volatile("" ::: "memory");            // (all rows' masks at once do not fit the registers)
                        __builtin_amdgcn_sched_barrier(0);
                    }
                }
                if (move) {
                    rows.move_references(x0, p.scale_log2);
                    move = false;
                }
                while (step(x0, x1) && step(x1, x0)) {}
                // (one copy of these across the paths, not two: the second would not fit the registers)
#pragma unroll
                for (int r = 0; r < kBlocks; ++r) asm("" : "+v"(rows.m[r]), "+v"(rows.l[r]));
            }
            wait_vmcnt<0>();                             // copies that nobody needed
            asm volatile("" ::: "memory");
            meet();
            // ---- end of the segment: the whole block is normalised and written out, a part of one leaves a record
            const bool whole = t0 == 0 && t1 == all;
            float *rec = reinterpret_cast<float *>(reinterpret_cast<char *>(p.workspace) + kNotesBytes) +
                         (size_t)(2 * range + (t0 == 0 ? 1 : 0)) * ((size_t)kRows * (D + 2));
#pragma unroll
            for (int r = 0; r < kBlocks; ++r) {
                float sum = rows.l[r];
                sum += __shfl_xor(sum, 16);
                sum += __shfl_xor(sum, 32);
                const float inv = sum == 0.f ? 0.f : 1.f / sum;
                int row = first + r * 16 + i16;
                asm("" : "+v"(row));                     // (where the row goes is found again: kept through the steps, it would cost registers)
                const bool real = Rows::token(p, row) < nt;
                const size_t at = Rows::out_row(p, o.head, row0, nt, row);
#pragma unroll
                for (int n = 0; n < D / 16; ++n) {       // four values 4 piece .. + 3 of the row
                    constexpr int kHalves = D / 64;
                    const int k = n / kHalves, h = n % kHalves, piece = (4 * quad + k) * kHalves + h;
                    const f32x4 v = f32x4{rows.acc[r][4 * h][k], rows.acc[r][4 * h + 1][k], rows.acc[r][4 * h + 2][k], rows.acc[r][4 * h + 3][k]} * inv;
                    if (!whole) reinterpret_cast<f32x4 *>(rec)[piece * kRows + row] = v;
                    else if (real) *reinterpret_cast<uint2 *>(p.out + at * D + piece * 4) = make_uint2(pack_bf16x2(v[0], v[1]), pack_bf16x2(v[2], v[3]));
                }
                if (quad == 0) {
                    if (!whole) {
                        rec[(size_t)kRows * D + row] = sum == 0.f ? -INFINITY : rows.m[r];
                        rec[(size_t)kRows * (D + 1) + row] = sum;
                    } else if (real && p.lse) {
                        p.lse[lse_at(p, at)] = sum == 0.f ? -INFINITY : (rows.m[r] + __builtin_amdgcn_logf(sum)) * kLn2;
                    }
                }
            }
        }
        if (last_block) break;
        o.next(seqs, p.B, tb);
        o = o.of_lane(0);
    }
    if (p.status && bad) atomicOr(p.status, bad);
}

template <int D, int kBlocks>
hipError_t launch_wide(KvqAttnParams p, hipStream_t stream) {
    constexpr int kRows = 16 * kBlocks * kWaves;
    p.n_ranges = kNumCU;
    p.tokens_per_block = kRows / p.G;
    if (p.nodes > 0) hipLaunchKernelGGL((kvq_attn_wide_kernel<D, kBlocks, true>), dim3(p.n_ranges), dim3(kThreadsWide), 0, stream, p);
    else hipLaunchKernelGGL((kvq_attn_wide_kernel<D, kBlocks, false>), dim3(p.n_ranges), dim3(kThreadsWide), 0, stream, p);
    const hipError_t e = hipGetLastError();
    if (e != hipSuccess) return note_hip_error("launch kvq_attn_wide_kernel", e);
    return launch_prompt_merge(p, kRows, stream);
}

}  // namespace

hipError_t launch_kvq_attn_wide(const KvqAttnParams &p, int rows, hipStream_t stream) {
    if (rows == 128) return p.D == 64 ? launch_wide<64, 2>(p, stream) : launch_wide<128, 2>(p, stream);
    return p.D == 64 ? launch_wide<64, 4>(p, stream) : launch_wide<128, 4>(p, stream);
}

}  // namespace reader

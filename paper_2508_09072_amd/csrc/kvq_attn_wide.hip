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
typedef float f32x16 __attribute__((ext_vector_type(16)));
constexpr int kWaveRows = 32;

template <int D>
struct WideLayout {
    static constexpr int kFrag = 1024;                                            // an operand: 16 bytes a lane
    static constexpr int kFrags = D / 16;                                         // of K in a step, and of V
    static constexpr int kStepBytes = 2 * kFrags * kFrag, kBuffers = 3;
    static constexpr int kCodes = kStepPages * 16 * D, kRaw = kCodes + 256;       // codes of two pages, their scales (D bytes each)
    static constexpr int kSlots = 6, kDepth = 3;                                  // raw steps in the ring; asked for as many steps before they are used
};

// 32 query rows of a wavefront.  S^T = K.Q^T, 32 keys x 32 rows, leaves lane (half, row) with keys 8 g + 4 half + i in register 4 g + i:
// as they stand, the operand of O^T += V^T.P^T for the 16 keys of page g / 2, if lane (half, column) of the other one holds the same.
template <int D>
struct WideRows {
    using W = WideLayout<D>;
    static constexpr int kOut = D / 32;
    bf16x8 q[W::kFrags];                 // step t: values ((t / (D/32)) * 2 + half) D / 4 + t % (D/32) * 8 .. + 7 of the row
    f32x16 acc[kOut];                    // [b][4 g + i]: with rho = 8 g + 4 half + i, value rho % 16 * D / 16 + 2 b + rho / 16 of the row
    float m, l;                          // reference (exponent of two), this lane's part of the sum
    u32x4 pk[kStepPages];

    __device__ static __forceinline__ int token(const PromptParams &p, int row) { return (int)(((float)row + 0.5f) * p.g_rcp); }   // row / G
    __device__ static __forceinline__ size_t out_row(const PromptParams &p, int head, int row0, int nt, int row) {
        const int tok = token(p, row);
        return ((size_t)row0 + min(tok, nt - 1)) * p.Hq + (size_t)head * p.G + (row - tok * p.G);
    }
    __device__ __forceinline__ void load(const PromptParams &p, int head, int row0, int nt, int row, int half) {
        const bool real = token(p, row) < nt;
        const size_t at = out_row(p, head, row0, nt, row);
#pragma unroll
        for (int t = 0; t < W::kFrags; ++t)
            q[t] = __builtin_bit_cast(bf16x8, keep_if(real, ld16(p.q + at * D + (t / (D / 32) * 2 + half) * (D / 4) + t % (D / 32) * 8)));
        m = kNoReference;
        l = 0.f;
#pragma unroll
        for (int b = 0; b < kOut; ++b)
#pragma unroll
            for (int e = 0; e < 16; ++e) acc[b][e] = 0.f;
    }
    __device__ __forceinline__ void scores(f32x16 &x, const char *k, int lane) const {
#pragma unroll
        for (int e = 0; e < 16; ++e) x[e] = 0.f;
#pragma unroll
        for (int t = 0; t < W::kFrags; ++t)
            x = __builtin_amdgcn_mfma_f32_32x32x16_bf16(*reinterpret_cast<const bf16x8 *>(k + t * W::kFrag + lane * 16), q[t], x, 0, 0, 0);
    }
    // Weights of the scores, and what the lane's sum becomes with them.
    __device__ __forceinline__ float weights(const f32x16 &x, float c2) {
        float sum[2] = {l, 0.f};
#pragma unroll
        for (int e = 0; e < 16; e += 2) {
            const float w0 = __builtin_amdgcn_exp2f(x[e] * c2 - m), w1 = __builtin_amdgcn_exp2f(x[e + 1] * c2 - m);
            sum[0] += w0;
            sum[1] += w1;
            pk[e / 8][e / 2 % 4] = pack_bf16x2(w0, w1);
        }
        return sum[0] + sum[1];
    }
    __device__ __forceinline__ void products(const char *v, int lane) {
#pragma unroll
        for (int pg = 0; pg < kStepPages; ++pg)
#pragma unroll
            for (int b = 0; b < kOut; ++b)
                acc[b] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(*reinterpret_cast<const bf16x8 *>(v + (pg * kOut + b) * W::kFrag + lane * 16),
                                                                 __builtin_bit_cast(bf16x8, pk[pg]), acc[b], 0, 0, 0);
    }
    // Moves the reference so that no weight of these scores is above one, nor the row's sum.
    __device__ __forceinline__ void move_reference(const f32x16 &x, float c2) {
        float mx = x[0];
#pragma unroll
        for (int e = 1; e < 16; ++e) mx = fmaxf(mx, x[e]);
        mx = fmaxf(mx * c2, m + __builtin_amdgcn_logf(l));                   // (minus infinity where the sum is zero)
        mx = fmaxf(mx, __shfl_xor(mx, 32));
        const float top = fmaxf(m, mx), f = __builtin_amdgcn_exp2f(m - top);
        l *= f;
        m = top;
#pragma unroll
        for (int b = 0; b < kOut; ++b)
#pragma unroll
            for (int e = 0; e < 16; ++e) acc[b][e] *= f;
    }
};

// A quarter (`part`) of a step's K operands: half of the words of one page's lanes.
template <int D>
__device__ __forceinline__ void make_keys(const char *raw, char *to, int part, int lane, int i16, int quad) {
    using W = WideLayout<D>;
    constexpr int kWords = D / 32;                           // of eight codes, a lane's; half of them are taken here
    const int pg = part >> 1, first = (part & 1) * (kWords / 2);
    const float sc = scale_of(*reinterpret_cast<const uint8_t *>(raw + W::kCodes + pg * D + (D == 128 ? quad : quad >> 1) * 16 + i16));
    char *at = to + (quad >> 1) * kWords * W::kFrag + (pg * 16 + i16 + 32 * (quad & 1)) * 16;
#pragma unroll
    for (int h = 0; h < kWords / 2; ++h) {
        const uint32_t w = *reinterpret_cast<const uint32_t *>(raw + pg * (16 * D) + lane * (D / 8) + (first + h) * 4);
        *reinterpret_cast<u32x4 *>(at + (first + h) * W::kFrag) = u32x4{two_values<0>(w, sc), two_values<1>(w, sc), two_values<2>(w, sc), two_values<3>(w, sc)};
    }
}

// ... and of its V operands: columns 2 b, 2 b + 1 of every chunk of both pages (D 64: of one page).  valid: keys of each page that
// somebody sees; what the others' bytes hold must not meet a weight of zero.
template <int D>
__device__ __forceinline__ void make_values(const char *raw, char *to, int part, int lane, int i16, int quad, int valid0, int valid1) {
    using W = WideLayout<D>;
    constexpr int kOut = D / 32;
    const int b = D == 128 ? part : part & 1;
#pragma unroll
    for (int turn = 0; turn < (D == 128 ? 2 : 1); ++turn) {
        const int pg = D == 128 ? turn : part >> 1;
        const char *v = raw + pg * (16 * D) + 8 * D;
        const uint32_t vs = *reinterpret_cast<const uint32_t *>(raw + W::kCodes + pg * D + D / 2 + quad * (D / 8) + (i16 * (D / 16) / 32) * 4);
        uint32_t word[4];
        if constexpr (D == 128) {
            const u32x4 c = *reinterpret_cast<const u32x4 *>(v + lane * 16);
#pragma unroll
            for (int e = 0; e < 4; ++e) word[e] = c[e] >> (8 * b);
        } else {
            const uint2 c = *reinterpret_cast<const uint2 *>(v + lane * 8);
            word[0] = c.x >> (8 * b); word[1] = c.x >> (16 + 8 * b); word[2] = c.y >> (8 * b); word[3] = c.y >> (16 + 8 * b);
        }
        uint32_t y[4];
#pragma unroll
        for (int e = 0; e < 4; ++e) y[e] = two_values<0>(word[e], scale_of(vs >> (8 * e) & 255u));
        const int n = (pg == 0 ? valid0 : valid1) - 4 * quad;
        if (n < 4) {
#pragma unroll
            for (int e = 0; e < 4; ++e) y[e] = e < n ? y[e] : 0u;
        }
        // (keys 4 quad .. + 3: half quad & 1 of the operand, place quad / 2 of its lanes)
        char *at = to + (W::kFrags + pg * kOut + b) * W::kFrag + (i16 + 32 * (quad & 1)) * 16 + (quad >> 1) * 8;
        *reinterpret_cast<uint2 *>(at) = make_uint2(__builtin_amdgcn_perm(y[1], y[0], 0x05040100), __builtin_amdgcn_perm(y[3], y[2], 0x05040100));
        *reinterpret_cast<uint2 *>(at + 16 * 16) = make_uint2(__builtin_amdgcn_perm(y[1], y[0], 0x07060302), __builtin_amdgcn_perm(y[3], y[2], 0x07060302));
    }
}

template <int D, int kWaves, bool kTree>
__global__ __launch_bounds__(64 * kWaves) __attribute__((amdgpu_waves_per_eu(2, 2))) void kvq_attn_wide_kernel(KvqAttnParams p) {
    using Rows = WideRows<D>;
    using W = WideLayout<D>;
    constexpr int kRows = kWaveRows * kWaves, kMinRange = 4 * kStep;
    constexpr int kCopies = 8 / kWaves;                  // copy instructions of a wavefront in a step
    __shared__ __attribute__((aligned(1024))) char s_frag[W::kBuffers][W::kStepBytes];
    __shared__ __attribute__((aligned(1024))) char s_raw[W::kSlots][W::kRaw];
    __shared__ int s_ids[kWaves][2][64];
    __shared__ uint32_t s_mask[kTree ? READER_MAX_T : 1][4];
    __shared__ int s_up[kTree ? READER_MAX_T : 1];
    const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    const int i16 = lane & 15, quad = lane >> 4, half = lane >> 5, tb = p.tokens_per_block;
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
    const int copy_page = D == 128 ? (wave >> 1) & 1 : wave & 1, copy_part = D == 128 ? wave & 1 : 0;
    const int scale_page = D == 128 ? lane >> 5 : lane >> 4 & 1, scale_word = D == 128 ? lane & 31 : lane & 15;
    const unsigned num_pages = (unsigned)(p.num_pages < 0x7fffffffLL ? p.num_pages : 0x7fffffffLL);

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
            const int steps = t1 - t0;
            const int unmasked = kTree ? o.L : (int)min(p0 + 1, (long long)p.max_seq_len);     // keys that every row sees
            PageIds ids(p.page_table + (size_t)o.b * p.max_pages, t0 * kStepPages, p.max_pages, &s_ids[wave][0][0]);
            auto raw_id = [&](int step, int now, int pg) {
                const int at = step * kStepPages + pg, id_now = __builtin_amdgcn_readlane(ids.now, at & 63), id_then = __builtin_amdgcn_readlane(ids.then, at & 63);
                return (unsigned)((at >> 6) == (now >> 5) ? id_now : id_then);
            };
            // keys of page pg of a step that somebody sees (above 16: all)
            auto valid = [&](int step, int now, int pg) {
                return raw_id(step, now, pg) < num_pages ? keys - (t0 + step) * kStep - pg * READER_PAGE_SIZE : 0;
            };
            unsigned whole_steps = 0;                    // bit of a step, by its number modulo 32: both pages are there, all keys seen
            const char *const cache = reinterpret_cast<const char *>(p.cache) + (size_t)o.head * KvqBlock<D>::kBytes;
            const size_t page_bytes = (size_t)p.Hkv * KvqBlock<D>::kBytes;
            auto issue = [&](int step, int now) {        // (at step `now`) kCopies copy instructions, whatever the pages are
                unsigned id0 = raw_id(step, now, 0), id1 = raw_id(step, now, 1);
                const bool there0 = id0 < num_pages, there1 = id1 < num_pages;
                id0 = there0 ? id0 : 0u; id1 = there1 ? id1 : 0u;
                whole_steps = (whole_steps & ~(1u << (step & 31))) | (unsigned)(there0 && there1 && (t0 + step + 1) * kStep <= keys) << (step & 31);
                const unsigned slot = raw_lds + (step % W::kSlots) * W::kRaw;
                const char *b0 = cache + id0 * page_bytes, *b1 = cache + id1 * page_bytes;
                if (kWaves == 4 || wave < 4) copy16_uniform((copy_page ? b1 : b0) + copy_part * 1024, lane * 16, slot + copy_page * (16 * D) + copy_part * 1024);
                if (kWaves == 4 || wave >= 4) {
                    const char *from = (scale_page ? b1 : b0) + 16 * D + scale_word * 4;
                    asm volatile("s_mov_b32 m0, %1\n\tglobal_load_lds_dword %0, off" :: "v"(from), "s"(slot + W::kCodes) : "memory", "m0");
                }
            };
            auto make = [&](int step, int now) {         // (at step `now`) this wavefront's part of a step's operands
                const char *raw = s_raw[step % W::kSlots];
                char *to = s_frag[step % W::kBuffers];
                if (kWaves == 4 || wave < 4) make_keys<D>(raw, to, wave & 3, lane, i16, quad);
                if (kWaves == 4 || wave >= 4) {
                    int v0 = READER_PAGE_SIZE, v1 = READER_PAGE_SIZE;
                    if (!(whole_steps >> (step & 31) & 1)) { v0 = valid(step, now, 0); v1 = valid(step, now, 1); }
                    make_values<D>(raw, to, wave & 3, lane, i16, quad, v0, v1);
                }
            };
            auto meet = [&] {
                __builtin_amdgcn_fence(__ATOMIC_RELEASE, "workgroup", "local");
                __builtin_amdgcn_s_barrier();
                __builtin_amdgcn_fence(__ATOMIC_ACQUIRE, "workgroup", "local");
                asm volatile("" ::: "memory");
            };
            ids.load(0, lane);
            Rows rows;
            int row = wave * kWaveRows + (lane & 31);
            rows.load(p, o.head, row0, nt, row, half);
            wait_vmcnt<0>();                             // the first page ids are there
            asm volatile("" ::: "memory");
            ids.begin(lane);
            for (int s = 0; s < W::kDepth + 2; ++s) issue(s, 0);
            wait_vmcnt<kCopies * (W::kDepth - 1)>();     // steps 0, 1 and 2
            asm volatile("" ::: "memory");
            meet();
            make(0, 0);
            make(1, 0);
            meet();
            auto masked = [&](int s) { return (t0 + s + 1) * kStep > unmasked || !(whole_steps >> (s & 31) & 1); };
            bool move = true;                            // (the reference is yet to be found)
            int s = 0;
            f32x16 x0, x1;
            // One step: the weights of the scores `xa` of step s, the scores `xb` of step s + 1, the products.  true: on with the next one.
            auto step = [&](const f32x16 &xa, f32x16 &xb) -> bool {
                rows.scores(xb, s_frag[(s + 1) % W::kBuffers], lane);
                const float sum = rows.weights(xa, p.scale_log2);
                if (__any(sum > kMostSum)) {
                    move = true;
                    return false;
                }
                rows.l = sum;
                issue(s + 2 + W::kDepth, s);
                make(s + 2, s);
                rows.products(s_frag[s % W::kBuffers] + W::kFrags * W::kFrag, lane);
                wait_vmcnt<kCopies * (W::kDepth - 1)>();     // step s + 3 has come
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
                    const int j0 = (t0 + s) * kStep, valid0 = valid(s, s, 0), valid1 = valid(s, s, 1);
                    if ((j0 < keys && valid0 <= 0) || (j0 + READER_PAGE_SIZE < keys && valid1 <= 0)) bad |= READER_STATUS_BAD_PAGE;
                    asm("" : "+v"(row));                 // (what follows from the row is found again: kept through the steps, it would cost registers)
                    const int tok = min(Rows::token(p, row), nt - 1), lim = (int)min(p0 + tok + 1, (long long)p.max_seq_len);
                    const uint32_t *mask = s_mask[kTree ? o.k * tb + tok : 0];
#pragma unroll
                    for (int e = 0; e < 16; ++e) {
                        const int at = e / 4 * 8 + half * 4 + e % 4, key = j0 + at, n = key - o.L;
                        // (no branches: with them the compiler has lost the assignment on one of the ways)
                        bool sees = ((e < 8 ? valid0 : valid1) > 0) & (key < lim);
                        if constexpr (kTree) sees &= (n < 0) | ((mask[(n >> 5) & 3] >> (n & 31) & 1u) != 0);
                        x0[e] = sees ? x0[e] : -INFINITY;
                    }
                }
                if (move) {
                    rows.move_reference(x0, p.scale_log2);
                    move = false;
                }
                while (step(x0, x1) && step(x1, x0)) {}
            }
            wait_vmcnt<0>();                             // copies that nobody needed
            asm volatile("" ::: "memory");
            meet();
            // ---- end of the segment: the whole block is normalised and written out, a part of one leaves a record
            const bool whole = t0 == 0 && t1 == all;
            float *rec = reinterpret_cast<float *>(reinterpret_cast<char *>(p.workspace) + kNotesBytes) +
                         (size_t)(2 * range + (t0 == 0 ? 1 : 0)) * ((size_t)kRows * (D + 2));
            asm("" : "+v"(row));
            const float sum = rows.l + __shfl_xor(rows.l, 32), inv = sum == 0.f ? 0.f : 1.f / sum;
            const bool real = Rows::token(p, row) < nt;
            const size_t at = Rows::out_row(p, o.head, row0, nt, row);
#pragma unroll
            for (int g = 0; g < 2; ++g)
#pragma unroll
                for (int i = 0; i < 4; ++i) {            // the D / 16 values of chunk 8 g + 4 half + i
                    const int chunk = 8 * g + 4 * half + i;
#pragma unroll
                    for (int h = 0; h < D / 64; ++h) {
                        const f32x4 v = f32x4{rows.acc[2 * h][4 * g + i], rows.acc[2 * h][4 * g + 8 + i], rows.acc[2 * h + 1][4 * g + i],
                                              rows.acc[2 * h + 1][4 * g + 8 + i]} * inv;
                        const int piece = chunk * (D / 64) + h;
                        if (!whole) reinterpret_cast<f32x4 *>(rec)[piece * kRows + row] = v;
                        else if (real) *reinterpret_cast<uint2 *>(p.out + at * D + piece * 4) = make_uint2(pack_bf16x2(v[0], v[1]), pack_bf16x2(v[2], v[3]));
                    }
                }
            if (half == 0) {
                if (!whole) {
                    rec[(size_t)kRows * D + row] = sum == 0.f ? -INFINITY : rows.m;
                    rec[(size_t)kRows * (D + 1) + row] = sum;
                } else if (real && p.lse) {
                    p.lse[lse_at(p, at)] = sum == 0.f ? -INFINITY : (rows.m + __builtin_amdgcn_logf(sum)) * kLn2;
                }
            }
        }
        if (last_block) break;
        o.next(seqs, p.B, tb);
        o = o.of_lane(0);
    }
    if (p.status && bad) atomicOr(p.status, bad);
}

template <int D, int kWaves>
hipError_t launch_wide(KvqAttnParams p, hipStream_t stream) {
    constexpr int kRows = kWaveRows * kWaves;
    p.n_ranges = kNumCU * 8 / kWaves;                    // (as many as run at once)
    p.tokens_per_block = kRows / p.G;
    if (p.nodes > 0) hipLaunchKernelGGL((kvq_attn_wide_kernel<D, kWaves, true>), dim3(p.n_ranges), dim3(64 * kWaves), 0, stream, p);
    else hipLaunchKernelGGL((kvq_attn_wide_kernel<D, kWaves, false>), dim3(p.n_ranges), dim3(64 * kWaves), 0, stream, p);
    const hipError_t e = hipGetLastError();
    if (e != hipSuccess) return note_hip_error("launch kvq_attn_wide_kernel", e);
    return launch_prompt_merge(p, kRows, stream);
}

}  // namespace

hipError_t launch_kvq_attn_wide(const KvqAttnParams &p, int rows, hipStream_t stream) {
    if (rows == 128) return p.D == 64 ? launch_wide<64, 4>(p, stream) : launch_wide<128, 4>(p, stream);
    return p.D == 64 ? launch_wide<64, 8>(p, stream) : launch_wide<128, 8>(p, stream);
}

}  // namespace reader

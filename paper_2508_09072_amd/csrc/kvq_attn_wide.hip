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
    using Frags = bf16x8[W::kFrags];
    __device__ static __forceinline__ void read(Frags &f, const char *from, int lane) {
#pragma unroll
        for (int t = 0; t < W::kFrags; ++t) f[t] = *reinterpret_cast<const bf16x8 *>(from + t * W::kFrag + lane * 16);
    }
    __device__ __forceinline__ void scores(f32x16 &x, const Frags &k) const {
#pragma unroll
        for (int e = 0; e < 16; ++e) x[e] = 0.f;
#pragma unroll
        for (int t = 0; t < W::kFrags; ++t) x = __builtin_amdgcn_mfma_f32_32x32x16_bf16(k[t], q[t], x, 0, 0, 0);
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
    __device__ __forceinline__ void products(const Frags &v) {
#pragma unroll
        for (int pg = 0; pg < kStepPages; ++pg)
#pragma unroll
            for (int b = 0; b < kOut; ++b)
                acc[b] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(v[pg * kOut + b], __builtin_bit_cast(bf16x8, pk[pg]), acc[b], 0, 0, 0);
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

// What one of D / 16 parts of a step's operands is made of: eight codes a lane of a page's K, and columns 2 b, 2 b + 1 of every chunk
// of a page's V for the lane's four keys.
template <int D>
struct Part {
    using W = WideLayout<D>;
    static constexpr int kWords = D / 32, kParts = D / 16;
    uint32_t k, ks, vs, v[D == 128 ? 4 : 2];
    __device__ __forceinline__ void read(const char *raw, int part, int lane, int i16, int quad) {
        const int pg = part / kWords, w = part % kWords;
        const char *codes = raw + pg * (16 * D), *scales = raw + W::kCodes + pg * D;
        k = *reinterpret_cast<const uint32_t *>(codes + lane * (D / 8) + w * 4);
        ks = *reinterpret_cast<const uint8_t *>(scales + (D == 128 ? quad : quad >> 1) * 16 + i16);
        vs = *reinterpret_cast<const uint32_t *>(scales + D / 2 + quad * (D / 8) + (i16 * (D / 16) / 32) * 4);
        if constexpr (D == 128) {
            const u32x4 c = *reinterpret_cast<const u32x4 *>(codes + 8 * D + lane * 16);
#pragma unroll
            for (int e = 0; e < 4; ++e) v[e] = c[e];
        } else {
            const uint2 c = *reinterpret_cast<const uint2 *>(codes + 8 * D + lane * 8);
            v[0] = c.x; v[1] = c.y;
        }
    }
    __device__ __forceinline__ void write(char *to, int part, int i16, int quad) const {
        const int pg = part / kWords, w = part % kWords;
        const float sc = scale_of(ks);
        *reinterpret_cast<u32x4 *>(to + ((quad >> 1) * kWords + w) * W::kFrag + (pg * 16 + i16 + 32 * (quad & 1)) * 16) =
            u32x4{two_values<0>(k, sc), two_values<1>(k, sc), two_values<2>(k, sc), two_values<3>(k, sc)};
        uint32_t y[4];
#pragma unroll
        for (int e = 0; e < 4; ++e) y[e] = two_values<0>((D == 128 ? v[e] : v[e / 2] >> (e % 2 * 16)) >> (8 * w), scale_of(vs >> (8 * e) & 255u));
        // (keys 4 quad .. + 3: half quad & 1 of the operand, place quad / 2 of its lanes)
        char *at = to + (W::kFrags + pg * (D / 32) + w) * W::kFrag + (i16 + 32 * (quad & 1)) * 16 + (quad >> 1) * 8;
        *reinterpret_cast<uint2 *>(at) = make_uint2(__builtin_amdgcn_perm(y[1], y[0], 0x05040100), __builtin_amdgcn_perm(y[3], y[2], 0x05040100));
        *reinterpret_cast<uint2 *>(at + 16 * 16) = make_uint2(__builtin_amdgcn_perm(y[1], y[0], 0x07060302), __builtin_amdgcn_perm(y[3], y[2], 0x07060302));
    }
};

// Page ids of a segment's keys, 64 (32 steps) at a time, a lane each: of the window that the wavefront is in and of the one behind it,
// which has come through LDS by an asynchronous copy.  A page that is not there, or whose first key nobody sees, is page 0 and has no
// bit in `ok`.
struct PageWindow {
    const int32_t *table;
    int page0, max_pages, keys;
    unsigned num_pages;
    int *window;                         // [2][64] in LDS, the wavefront's own
    int now, then;
    unsigned long long ok_now, ok_then;
    __device__ __forceinline__ void ask(int c, int lane) const {
        const int32_t *src = table + min(page0 + c * 64 + lane, max_pages - 1);
        const unsigned dst = (unsigned)(size_t)(lds_char *)reinterpret_cast<char *>(window) + (c & 1) * 256;
        asm volatile("s_mov_b32 m0, %1\n\tglobal_load_lds_dword %0, off" :: "v"(src), "s"(dst) : "memory", "m0");
    }
    __device__ __forceinline__ void take(int c, int lane) {
        const int id = window[(c & 1) * 64 + lane];
        const bool there = (unsigned)id < num_pages && (page0 + c * 64 + lane) * READER_PAGE_SIZE < keys;
        ok_then = __ballot(there);
        then = there ? id : 0;
    }
    // at the head of step i: a window is asked for when the one in front of it begins, and taken 20 steps later
    __device__ __forceinline__ void advance(int i, int steps, int lane) {
        const int c = i >> 5, in = i & 31;
        if (in == 0) {
            if (i > 0) { now = then; ok_now = ok_then; }
            if ((c + 1) * 32 < steps) ask(c + 1, lane);
            else ok_then = 0, then = 0;
        }
        if (in == 20 && (c + 1) * 32 < steps) take(c + 1, lane);
    }
    // page pg of a step at most 8 ahead of step i; whether both pages of it are there
    __device__ __forceinline__ unsigned id(int step, int i, int pg) const {
        const int from = (step ^ i) & 32 ? then : now;
        return (unsigned)__builtin_amdgcn_readlane(from, (step * 2 + pg) & 63);
    }
    __device__ __forceinline__ unsigned there(int step, int i) const { return (unsigned)(((step ^ i) & 32 ? ok_then : ok_now) >> (step * 2 & 63)) & 3u; }
};

template <int D, int kWaves, bool kTree>
__global__ __launch_bounds__(64 * kWaves) __attribute__((amdgpu_waves_per_eu(2, 2))) void kvq_attn_wide_kernel(KvqAttnParams p) {
    using Rows = WideRows<D>;
    using W = WideLayout<D>;
    constexpr int kRows = kWaveRows * kWaves, kMinRange = 4 * kStep;
    constexpr int kCopies = 8 / kWaves;                  // copy instructions of a wavefront in a step
    constexpr int kParts = (Part<D>::kParts + kWaves - 1) / kWaves;          // parts of the operands that it makes
    __shared__ __attribute__((aligned(1024))) char s_frag[W::kBuffers * W::kStepBytes];
    __shared__ __attribute__((aligned(1024))) char s_raw[W::kSlots * W::kRaw];
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
    const unsigned raw_lds = (unsigned)(size_t)(lds_char *)&s_raw[0];
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
            PageWindow ids = {p.page_table + (size_t)o.b * p.max_pages, t0 * kStepPages, p.max_pages, keys, num_pages, &s_ids[wave][0][0], 0, 0, 0, 0};
            const int full = keys / kStep - t0;          // steps in front of this one have 32 keys that somebody sees
            auto whole_step = [&](int step, int now) { return (step < full) & (ids.there(step, now) == 3u); };
            const char *const cache = reinterpret_cast<const char *>(p.cache) + (size_t)o.head * KvqBlock<D>::kBytes;
            const unsigned page_bytes = (unsigned)p.Hkv * KvqBlock<D>::kBytes;
            auto issue = [&](int step, int now, unsigned slot) {     // (at step `now`) kCopies copy instructions, whatever the pages are
                const char *b0 = cache + (size_t)ids.id(step, now, 0) * page_bytes, *b1 = cache + (size_t)ids.id(step, now, 1) * page_bytes;
                if (kWaves == 4 || wave < 4) copy16_uniform((copy_page ? b1 : b0) + copy_part * 1024, lane * 16, raw_lds + slot + copy_page * (16 * D) + copy_part * 1024);
                if (kWaves == 4 || wave >= 4) {
                    const char *from = (scale_page ? b1 : b0) + 16 * D + scale_word * 4;
                    asm volatile("s_mov_b32 m0, %1\n\tglobal_load_lds_dword %0, off" :: "v"(from), "s"(raw_lds + slot + W::kCodes) : "memory", "m0");
                }
            };
            // What this wavefront has copied of keys that nobody sees becomes zeros: their bytes must not meet a weight of zero.
            auto blank = [&](int step, int now, unsigned slot) {
                const unsigned there = ids.there(step, now);
                const int j0 = (t0 + step) * kStep;
                int l = lane;
                asm("" : "+v"(l));                       // (addresses are found here: kept through the steps, they would cost registers)
#pragma unroll 1
                for (int pg = 0; pg < kStepPages; ++pg) {
                    const int n = there >> pg & 1 ? keys - j0 - pg * READER_PAGE_SIZE : 0;
                    char *codes = s_raw + slot + pg * (16 * D);
                    if ((kWaves == 4 || wave < 4) && copy_page == pg && (D == 64 || copy_part == 1)) {
#pragma unroll
                        for (int e = 0; e < 4; ++e) {
                            if (4 * (l >> 4) + e < n) continue;
                            if constexpr (D == 128) *reinterpret_cast<uint32_t *>(codes + 8 * D + l * 16 + e * 4) = 0;
                            else *reinterpret_cast<uint16_t *>(codes + 8 * D + l * 8 + e * 2) = 0;
                        }
                    }
                    if (kWaves == 4 || wave >= 4) {          // a byte of the scales a lane, of the first D / 2
                        if (l < D / 2 && (l / (D / 8)) * 4 + l % 4 >= n) s_raw[slot + W::kCodes + pg * D + D / 2 + l] = 127;
                    }
                }
            };
            auto read_parts = [&](Part<D> (&part)[kParts], unsigned slot) {
#pragma unroll
                for (int i = 0; i < kParts; ++i) part[i].read(s_raw + slot, (wave + i * kWaves) % Part<D>::kParts, lane, i16, quad);
            };
            auto write_parts = [&](const Part<D> (&part)[kParts], unsigned buffer) {
#pragma unroll
                for (int i = 0; i < kParts; ++i) part[i].write(s_frag + buffer, (wave + i * kWaves) % Part<D>::kParts, i16, quad);
            };
            auto meet = [&] {
                __builtin_amdgcn_fence(__ATOMIC_RELEASE, "workgroup", "local");
                __builtin_amdgcn_s_barrier();
                __builtin_amdgcn_fence(__ATOMIC_ACQUIRE, "workgroup", "local");
                asm volatile("" ::: "memory");
            };
            ids.ask(0, lane);
            Rows rows;
            int row = wave * kWaveRows + (lane & 31);
            rows.load(p, o.head, row0, nt, row, half);
            wait_vmcnt<0>();                             // the first page ids are there
            asm volatile("" ::: "memory");
            ids.take(0, lane);
            ids.now = ids.then; ids.ok_now = ids.ok_then;
            for (int s = 0; s < W::kDepth + 2; ++s) issue(s, 0, s * W::kRaw);
            wait_vmcnt<kCopies * (W::kDepth - 1)>();     // steps 0, 1 and 2
            asm volatile("" ::: "memory");
            for (int s = 0; s < 3; ++s)
                if (!whole_step(s, 0)) blank(s, 0, s * W::kRaw);
            meet();
            Part<D> part[kParts];
            for (int s = 0; s < 2; ++s) {
                read_parts(part, s * W::kRaw);
                write_parts(part, s * W::kStepBytes);
            }
            meet();
            auto masked = [&](int s) { return (t0 + s + 1) * kStep > unmasked || !whole_step(s, s); };
            bool move = true;                            // (the reference is yet to be found)
            int s = 0;
            // where the operands of steps s, s + 1, s + 2 are, and the bytes of steps s + 2, s + 3, s + 2 + kDepth
            unsigned at0 = 0, at1 = W::kStepBytes, at2 = 2 * W::kStepBytes, raw2 = 2 * W::kRaw, raw5 = (2 + W::kDepth) * W::kRaw;
            auto behind = [](unsigned slot) { return slot == (W::kSlots - 1) * W::kRaw ? 0u : slot + W::kRaw; };
            f32x16 x0, x1;
            // One step: the weights of the scores `xa` of step s, the scores `xb` of step s + 1, the products.  true: on with the next one.
            auto step = [&](const f32x16 &xa, f32x16 &xb) -> bool {
                typename Rows::Frags k, v;
                Rows::read(k, s_frag + at1, lane);
                rows.scores(xb, k);
                const float sum = rows.weights(xa, p.scale_log2);
                Rows::read(v, s_frag + at0 + W::kFrags * W::kFrag, lane);
                read_parts(part, raw2);
                // the order: K's operands, then a product and a part of the weights in turn, V's operands and the bytes between them
                __builtin_amdgcn_sched_group_barrier(0x100, W::kFrags, 0);
                __builtin_amdgcn_sched_group_barrier(0x002, 10, 0);
#pragma unroll
                for (int i = 0; i < W::kFrags; ++i) {
                    __builtin_amdgcn_sched_group_barrier(0x008, 1, 0);
                    __builtin_amdgcn_sched_group_barrier(0x002, 48 / W::kFrags, 0);
                    __builtin_amdgcn_sched_group_barrier(0x100, 2, 0);
                }
                if (__any(sum > kMostSum)) {
                    move = true;
                    return false;
                }
                rows.l = sum;
                rows.products(v);
                write_parts(part, at2);
#pragma unroll
                for (int i = 0; i < W::kFrags; ++i) {
                    __builtin_amdgcn_sched_group_barrier(0x008, 1, 1);
                    __builtin_amdgcn_sched_group_barrier(0x002, 4 * kParts, 1);
                }
                issue(s + 2 + W::kDepth, s, raw5);
                wait_vmcnt<kCopies * (W::kDepth - 1)>();     // step s + 3 has come
                asm volatile("" ::: "memory");
                raw2 = behind(raw2);
                raw5 = behind(raw5);
                if (!whole_step(s + 3, s)) blank(s + 3, s, raw2);
                meet();
                const unsigned free = at0;
                at0 = at1; at1 = at2; at2 = free;
                ++s;
                if (s >= steps) return false;
                ids.advance(s, steps, lane);
                return !masked(s);
            };
            ids.advance(0, steps, lane);
            // (references are moved, and scores masked, outside the loop over the steps, with the scores computed again: a path around the
            // accumulators inside it is paid for in every step)
            while (s < steps) {
                {
                    typename Rows::Frags k;
                    Rows::read(k, s_frag + at0, lane);
                    rows.scores(x0, k);
                }
                if (masked(s)) {
                    const int j0 = (t0 + s) * kStep;
                    const unsigned there = ids.there(s, s);
                    if ((j0 < keys && !(there & 1)) || (j0 + READER_PAGE_SIZE < keys && !(there & 2))) bad |= READER_STATUS_BAD_PAGE;
                    asm("" : "+v"(row));                 // (what follows from the row is found again: kept through the steps, it would cost registers)
                    const int tok = min(Rows::token(p, row), nt - 1), lim = (int)min(p0 + tok + 1, (long long)p.max_seq_len);
                    const uint32_t *mask = s_mask[kTree ? o.k * tb + tok : 0];
#pragma unroll
                    for (int e = 0; e < 16; ++e) {
                        const int at = e / 4 * 8 + half * 4 + e % 4, key = j0 + at, n = key - o.L;
                        // (no branches: with them the compiler has lost the assignment on one of the ways)
                        bool sees = ((there >> (e / 8) & 1u) != 0) & (key < lim);
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
            int half_ = half;
            asm("" : "+v"(row), "+v"(half_));
            const float sum = rows.l + __shfl_xor(rows.l, 32), inv = sum == 0.f ? 0.f : 1.f / sum;
            const bool real = Rows::token(p, row) < nt;
            const size_t at = Rows::out_row(p, o.head, row0, nt, row);
#pragma unroll
            for (int g = 0; g < 2; ++g)
#pragma unroll
                for (int i = 0; i < 4; ++i) {            // the D / 16 values of chunk 8 g + 4 half + i
                    const int chunk = 8 * g + 4 * half_ + i;
#pragma unroll
                    for (int h = 0; h < D / 64; ++h) {
                        const f32x4 v = f32x4{rows.acc[2 * h][4 * g + i], rows.acc[2 * h][4 * g + 8 + i], rows.acc[2 * h + 1][4 * g + i],
                                              rows.acc[2 * h + 1][4 * g + 8 + i]} * inv;
                        const int piece = chunk * (D / 64) + h;
                        if (!whole) reinterpret_cast<f32x4 *>(rec)[piece * kRows + row] = v;
                        else if (real) *reinterpret_cast<uint2 *>(p.out + at * D + piece * 4) = make_uint2(pack_bf16x2(v[0], v[1]), pack_bf16x2(v[2], v[3]));
                    }
                }
            if (half_ == 0) {
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

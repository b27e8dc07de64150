// Up to 32 query rows of the prompts' attention that a wavefront carries through keys in LDS, 32 at a time (prompt_attn_few.hip,
// prompt_attn_mid.hip).
#pragma once

#include "prompt_attn_scalar.h"
#include "prompt_ranges.h"

namespace reader {

namespace {

typedef float f32x4 __attribute__((ext_vector_type(4)));
constexpr int kStep = 32, kStepPages = kStep / READER_PAGE_SIZE;
constexpr float kNoReference = -1e30f;               // of a row that has seen no key
constexpr float kTooLarge = 0x1p100f;                // ... of a sum that is not added to others any more

// How a page of 16 K or V rows is copied to LDS and read back as an operand: whole, 1 KB a copy instruction; the 16-byte chunks of
// a row are swizzled by the row, so that the reads of an operand touch every bank once (K: 16 rows, one chunk; V: 8 rows, two
// chunks side by side).
template <int D>
struct PageLayout {
    static constexpr int kRowBytes = D * 2, kChunks = D / 8, kPageBytes = READER_PAGE_SIZE * kRowBytes;
    static constexpr int kCopies = kPageBytes / 1024, kRowsPerCopy = 64 / kChunks;
    __device__ static __forceinline__ int swizzle_v16(int row) { return D == 128 ? (row & 7) << 1 : ((row >> 1) & 3) << 1; }
    unsigned k_off[kCopies], v_off[kCopies];             // this lane's 16 bytes of copy i: of row i * kRowsPerCopy + lane / kChunks
    int lane_row;
    __device__ __forceinline__ explicit PageLayout(int lane) : lane_row(lane / kChunks) {
#pragma unroll
        for (int i = 0; i < kCopies; ++i) {
            const int r = i * kRowsPerCopy + lane_row;
            k_off[i] = r * kRowBytes + (((lane % kChunks) ^ swizzle_k<D>(r)) << 4);
            v_off[i] = r * kRowBytes + (((lane % kChunks) ^ swizzle_v16(r)) << 4);
        }
    }
    // The page at `src` to LDS byte address `dst`, kCopies instructions; only its first `rows` rows exist (all of a page that is
    // not there: none): the others are copied from a block of zeros, so that a weight of zero times them stays zero.
    __device__ __forceinline__ void copy(const char *src, const unsigned (&off)[kCopies], int rows, unsigned dst, int lane) const {
        const char *zeros = reinterpret_cast<const char *>(kZeroRow) + (lane & 15) * 16;
#pragma unroll
        for (int j = 0; j < kCopies; ++j) {
            if (rows >= READER_PAGE_SIZE) copy16_uniform(src, off[j], dst + j * 1024);
            else copy16_lane(j * kRowsPerCopy + lane_row < rows ? src + off[j] : zeros, dst + j * 1024);
        }
    }
};

// Page ids of a segment's keys, 64 (32 steps of keys) at a time: a lane each, of the window that the wavefront is in and of the one
// behind it, which has come through LDS by an asynchronous copy (a load into a register would be waited for together with all
// copies on their way; an id read from LDS where it is needed costs the step a trip there).
struct PageIds {
    const int32_t *table;
    int page0, max_pages;
    int *window;             // [2][64] in LDS, the wavefront's own
    int now = 0, then = 0;
    __device__ __forceinline__ PageIds(const int32_t *t, int first, int most, int *w) : table(t), page0(first), max_pages(most), window(w) {}
    __device__ __forceinline__ void load(int c, int lane) const {
        const int32_t *src = table + min(page0 + c * 64 + lane, max_pages - 1);
        const unsigned dst = (unsigned)(size_t)(lds_char *)reinterpret_cast<char *>(window) + (c & 1) * 256;
        asm volatile("s_mov_b32 m0, %1\n\tglobal_load_lds_dword %0, off" :: "v"(src), "s"(dst) : "memory", "m0");
    }
    // the first window has landed
    __device__ __forceinline__ void begin(int lane) { now = window[lane]; }
    // At the head of step i, kStride steps behind the wavefront's last one.  A window is asked for when the one in front of it begins
    // and is there 20 steps later.
    template <int kStride>
    __device__ __forceinline__ void advance(int i, int steps, int lane) {
        const int c = i >> 5, in = i & 31;
        if (in < kStride) {
            if (i >= 32) now = then;
            if ((c + 1) * 32 < steps) load(c + 1, lane);
        }
        if (in >= 20 && in < 20 + kStride) then = window[((c + 1) & 1) * 64 + lane];
    }
    // page `at` of the segment, asked for at step i (at most 8 ahead): its id, or -1 if it is none or its first key is not below `keys`
    __device__ __forceinline__ int get(int at, int i, int keys, int64_t num_pages) const {
        const int id = (at >> 6) == (i >> 5) ? __builtin_amdgcn_readlane(now, at & 63) : __builtin_amdgcn_readlane(then, at & 63);
        return (page0 + at) * READER_PAGE_SIZE < keys && id >= 0 && id < num_pages ? id : -1;
    }
};

// kBlocks blocks of 16 rows.  S^T = K.Q^T in blocks of 16 keys x 16 rows leaves lane (quad, i16) with four scores of row i16 of a
// block for each page, keys 4 quad .. + 3: as they stand, the operand of O^T += V^T.P^T, if key 8 quad' + j of that product is key
// 4 quad + j % 4 of page j / 4 in both operands.  A row's reference is its maximum over the first 32 keys and is never moved: a lower
// one makes all weights of the row larger by one factor, which fp32 sums and bf16 weights hold.  A row whose sum reaches kTooLarge is
// computed again: up to there hundreds of its parts add up without an overflow, and a part is below 2^-24 of the row where its factor,
// 2 to the difference of two references, becomes zero.  With a maximum that moves, were it only once in a thousand steps, the
// compiler copies all accumulators three times a step where the paths meet.  Weights are rounded to bf16 for the second product, their
// sums are not (what that costs: prompt_attn.hip).
template <int D, int kBlocks>
struct PromptRows {
    using Page = PageLayout<D>;
    static constexpr int kSteps = D / 32, kOut = D / 16;     // 32-deep steps of the first product, 16-wide blocks of the output
    bf16x8 q[kBlocks][kSteps];                                // block r, step s: row i16, values 32 s + 8 quad .. + 7
    int lim[kBlocks];                                         // keys that row i16 of block r sees
    bool real[kBlocks];
    f32x4 acc[kBlocks][kOut];                                 // output 16 db + 4 quad .. + 3 of row i16
    float m[kBlocks], l[kBlocks];                             // reference (exponent of two), this lane's part of the sum

    // row i16 of block r as a row of q, out and lse (rows behind the last token: one of its)
    __device__ static __forceinline__ size_t out_row(const PromptParams &p, int head, int row0, int nt, int first, int r, int i16) {
        const int row = first + r * 16 + i16, tok = (int)(((float)row + 0.5f) * p.g_rcp);
        return ((size_t)row0 + min(tok, nt - 1)) * p.Hq + (size_t)head * p.G + (row - tok * p.G);
    }
    // rows first .. first + 16 kBlocks - 1 of the block that starts at packed row row0 and position p0 and has nt tokens
    __device__ __forceinline__ void load(const PromptParams &p, int head, int row0, long long p0, int nt, int first, int i16, int quad) {
#pragma unroll
        for (int r = 0; r < kBlocks; ++r) {
            const int row = first + r * 16 + i16, tok = (int)(((float)row + 0.5f) * p.g_rcp);    // row / G
            real[r] = tok < nt;
            lim[r] = real[r] ? (int)min(p0 + tok + 1, (long long)p.max_seq_len) : 0;
            const size_t at = out_row(p, head, row0, nt, first, r, i16);
#pragma unroll
            for (int s = 0; s < kSteps; ++s) q[r][s] = __builtin_bit_cast(bf16x8, keep_if(real[r], ld16(p.q + at * D + s * 32 + quad * 8)));
            m[r] = kNoReference;
            l[r] = 0.f;
#pragma unroll
            for (int db = 0; db < kOut; ++db) acc[r][db] = f32x4{0.f, 0.f, 0.f, 0.f};
        }
    }
    f32x4 x[kBlocks][kStepPages];                             // scores of 32 keys
    u32x4 pk[kBlocks];                                        // ... their weights, as operands
    // scores of the keys whose pages are at `kp` in LDS
    __device__ __forceinline__ void scores(const char *kp, int i16, int quad) {
#pragma unroll
        for (int pg = 0; pg < kStepPages; ++pg) {
            bf16x8 key[kSteps];
#pragma unroll
            for (int s = 0; s < kSteps; ++s)
                key[s] = *reinterpret_cast<const bf16x8 *>(kp + pg * Page::kPageBytes + i16 * Page::kRowBytes + (((4 * s + quad) ^ swizzle_k<D>(i16)) << 4));
#pragma unroll
            for (int r = 0; r < kBlocks; ++r) {
                x[r][pg] = f32x4{0.f, 0.f, 0.f, 0.f};
#pragma unroll
                for (int s = 0; s < kSteps; ++s) x[r][pg] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(key[s], q[r][s], x[r][pg], 0, 0, 0);
            }
        }
    }
    // Their weights; the keys are j0 .. j0 + 31.  start: the first ones.  masked: some row does not see some of them; hole0, hole1:
    // nobody sees the first, the second page.
    __device__ __forceinline__ void weights(int j0, bool start, bool masked, bool hole0, bool hole1, float c2, int quad) {
#pragma unroll
        for (int r = 0; r < kBlocks; ++r) {
            if (masked) {
#pragma unroll
                for (int pg = 0; pg < kStepPages; ++pg)
#pragma unroll
                    for (int e = 0; e < 4; ++e)
                        if (j0 + pg * 16 + quad * 4 + e >= lim[r] || (pg == 0 ? hole0 : hole1)) x[r][pg][e] = -INFINITY;
            }
            if (start) {
                float mx = fmaxf(fmaxf(x[r][0][0], x[r][0][1]), fmaxf(x[r][0][2], x[r][0][3]));
                mx = fmaxf(mx, fmaxf(fmaxf(x[r][1][0], x[r][1][1]), fmaxf(x[r][1][2], x[r][1][3])));
                mx = fmaxf(mx, __shfl_xor(mx, 16));
                mx = fmaxf(mx, __shfl_xor(mx, 32));
                m[r] = fmaxf(mx * c2, kNoReference);
            }
            float w[8];
#pragma unroll
            for (int e = 0; e < 8; ++e) {
                w[e] = __builtin_amdgcn_exp2f(x[r][e / 4][e % 4] * c2 - m[r]);
                l[r] += w[e];
            }
#pragma unroll
            for (int e = 0; e < 4; ++e) pk[r][e] = pack_bf16x2(w[2 * e], w[2 * e + 1]);
        }
    }
    // O^T += V^T.P^T with the values whose pages are at `vp`; taken(): they have all been read
    template <bool kTells, class F>
    __device__ __forceinline__ void products(const char *vp, int i16, int quad, F &&taken) {
        const int row = quad * 4 + (i16 >> 2), chunk = (i16 & 3) >> 1;
        const char *v_at = vp + row * Page::kRowBytes + (i16 & 1) * 8;
        constexpr int kPart = 4;                             // output blocks whose values are in registers at a time
#pragma unroll
        for (int d0 = 0; d0 < kOut; d0 += kPart) {
            s16x4 vf[kPart][kStepPages];
#pragma unroll
            for (int db = 0; db < kPart; ++db)
#pragma unroll
                for (int pg = 0; pg < kStepPages; ++pg)
                    vf[db][pg] = lds_read_tr16(v_at + pg * Page::kPageBytes + ((((d0 + db) * 2 + chunk) ^ Page::swizzle_v16(row)) << 4));
            if constexpr (kTells) {
                if (d0 + kPart == kOut) {
#pragma unroll
                    for (int db = 0; db < kPart; ++db) asm volatile("" : "+v"(vf[db][0]), "+v"(vf[db][1]) :: "memory");
                    taken();
                }
            }
#pragma unroll
            for (int db = 0; db < kPart; ++db) {
                const bf16x8 v8 = __builtin_bit_cast(bf16x8, __builtin_shufflevector(vf[db][0], vf[db][1], 0, 1, 2, 3, 4, 5, 6, 7));
#pragma unroll
                for (int r = 0; r < kBlocks; ++r)
                    acc[r][d0 + db] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(v8, __builtin_bit_cast(bf16x8, pk[r]), acc[r][d0 + db], 0, 0, 0);
            }
        }
    }
    // the whole sum of row i16 of every block, in all its lanes
    __device__ __forceinline__ void finish_sums() {
#pragma unroll
        for (int r = 0; r < kBlocks; ++r) {
            l[r] += __shfl_xor(l[r], 16);
            l[r] += __shfl_xor(l[r], 32);
        }
    }
    // Normalised rows to `out` and `lse`.  True if a row has a value that is not a number.
    __device__ __forceinline__ bool write(const PromptParams &p, int head, int row0, int nt, int first, int i16, int quad) {
        bool odd = false;
#pragma unroll
        for (int r = 0; r < kBlocks; ++r) {
            const float inv = l[r] == 0.f ? 0.f : 1.f / l[r];
            float check = l[r] < kTooLarge ? 0.f : __builtin_nanf("");   // (not a number once any value is none)
            const size_t at = out_row(p, head, row0, nt, first, r, i16);
#pragma unroll
            for (int db = 0; db < kOut; ++db) {
                const f32x4 v = acc[r][db] * inv;
                check = check + v[0] * 0.f + v[1] * 0.f + v[2] * 0.f + v[3] * 0.f;
                if (real[r]) *reinterpret_cast<uint2 *>(p.out + at * D + db * 16 + quad * 4) = make_uint2(pack_bf16x2(v[0], v[1]), pack_bf16x2(v[2], v[3]));
            }
            if (real[r] && quad == 0 && p.lse) p.lse[at] = l[r] == 0.f ? -INFINITY : (m[r] + __builtin_amdgcn_logf(l[r])) * kLn2;
            odd = odd || (real[r] && !(check == 0.f));
        }
        return __any(odd);
    }
};

// A value that is not a number, maybe behind a mask (times a weight of zero): rows [lo, hi) of a block the plain way, one after the
// other, over keys [j0, j1).  rec: where the block's part is left, kRecordRows rows wide, or null: the rows go to `out`.
template <int D>
__device__ inline void rows_the_plain_way(const PromptParams &p, const int32_t *table, int head, int row0, long long p0, int lo, int hi, int j0,
                                          int j1, float *rec, int record_rows, int lane, int &bad) {
    // (what the wavefront has just written to the same places is there before it is written again)
    wait_vmcnt<0>();
    asm volatile("" ::: "memory");
    for (int row = lo; row < hi; ++row) {
        const int tok = row / p.G;
        const size_t at = ((size_t)row0 + tok) * p.Hq + (size_t)head * p.G + (row - tok * p.G);
        const int end = (int)min(min(p0 + tok + 1, (long long)p.max_seq_len), (long long)j1);
        const ScalarRow<D> s = prompt_row_scalar<D>(p, p.q + at * D, table, head, j0, end, lane, bad);
        const float inv = s.l == 0.f ? 0.f : 1.f / s.l;
#pragma unroll
        for (int e = 0; e < D / 64; ++e) {
            const int d = lane * (D / 64) + e;
            if (!rec) p.out[at * D + d] = (uint16_t)pack_bf16x2(s.o[e] * inv, 0.f);
            else rec[((size_t)(d / 4) * record_rows + row) * 4 + d % 4] = s.o[e] * inv;
        }
        if (lane == 0) {
            if (rec) {
                rec[(size_t)record_rows * D + row] = s.l == 0.f ? -INFINITY : s.m;
                rec[(size_t)record_rows * (D + 1) + row] = s.l;
            } else if (p.lse) {
                p.lse[at] = s.l == 0.f ? -INFINITY : (s.m + __builtin_amdgcn_logf(s.l)) * kLn2;
            }
        }
    }
}

}  // namespace

}  // namespace reader

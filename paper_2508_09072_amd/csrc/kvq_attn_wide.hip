// Attention over a cache in 4 bits for many query rows a kv head: trees of many nodes, chunks of prompts (the mathematics: kvq_attn.hip).
//
// A workgroup takes a range of the (head, sequence, block of rows, key) axis with one or two wavefronts a SIMD, each with 32 query rows or
// two times 32, through 32 keys a step.  Bytes come into a ring in LDS by asynchronous copies, steps ahead of their use.  K is
// multiplied as it is stored (QueryPieces); of V every wavefront makes a share of each step's operands (two codes an instruction, exact in
// bf16), because a scale belongs to 32 columns of one key and the matrix instructions scale along the keys; they are left in LDS as the
// products read them, 1 KB an operand, conflict-free.  The scores of step s + 1 are computed beside the weights of step s, V's operands
// of step s + 3 are made beside the second product of step s; two steps are a turn of the loop (16 copies a step less, 1 %).
//   128 rows: four wavefronts, two workgroups a compute unit, a barrier a step.
//   256 rows, head dimension 128: eight wavefronts, the second of each SIMD half a step behind the first, so that one has the
//     matrix unit while the other makes weights (priority to products: 1 to 2 %), a barrier every two steps (3 % of long calls).  Four
//     wavefronts of twice 32 rows read V half as often but have nothing to fill the gaps with: 889 instead of 756 us on the same card
//     (64 trees of 64 nodes on 2 K to 8 K positions).
//   256 rows, head dimension 64: four wavefronts of twice 32 rows (half the operands a row; their scores fill the gaps).
// What bounds it: exponentials and the other 76 vector instructions of a wavefront's step take 560 cycles, its 14 products 448, and the two
// wavefronts of a SIMD cover each other's only in part (1900 cycles); and power: the clock is at 2.0 of 2.4 GHz then.  64 trees of 64 nodes
// on 2 K to 8 K positions, 64 and 8 heads of 128: 652 to 720 us (0.97 to 1.07 PFLOP/s), 5 % of them in front of the five blocks of a
// workgroup (page ids, queries, first bytes, one after the other; with the queries split behind the asking there are no registers).  2
// chunks of 512 tokens behind 20 K to 28 K: 695 to 760 us (1.04 to 1.14), where a library's product of 8192^3 reaches 1.14.  Blocks of few
// steps are far from that (16 prompts of 1000 tokens from an empty cache 280 us, their products alone 115): what stands in front of a
// block's first step and behind its last takes 8 to 9 us, nothing of the next block is asked for meanwhile, and masked steps leave the
// pairs of steps.
#include "kvq_attn.h"

namespace reader {

namespace {

using WideBlock = PromptBlock<kStep, 2 * kStep, 8 * kStep>;
typedef float f32x16 __attribute__((ext_vector_type(16)));
constexpr int kWaveRows = 32;

template <int D>
struct WideLayout {
    static constexpr int kFrag = 1024;                                            // an operand: 16 bytes a lane
    static constexpr int kFrags = D / 16;                                         // of V in a step
    static constexpr int kStepFrags = kFrags * kFrag;
    static constexpr int kCodes = kStepPages * 16 * D, kRaw = kCodes + 2 * D;     // codes of two pages, their scales
};

// 32 values of a query row, as matrix instructions multiply them with codes of 4 bits as they are stored: three pieces of 6 bits (e2m3:
// sign, up to 7.5, steps of 1/8 below 2, of 1/4 and 1/2 above) with scales of their own, the rounding of each left to the next.  With E =
// floor(log2 of the largest magnitude) - 2 the pieces count in steps of 2^(E - 3), 2^(E - 7) and 2^(E - 12) at least, so that a value above
// 1/128 of the largest keeps all bits that bf16 has and no value is off by more than 2^(E - 13), 2^-15 of the largest.  E is -117 at least,
// so that the third scale's exponent is one that there is: below, no value is off by more than 2^-130.  The
// three products take 3/4 of the time of one with bf16 operands, and K needs no operands made of it (735 us without, 684 with: 64 trees
// of 64 nodes on 2 K to 8 K positions).  The few rows of kvq_attn.hip would gain 1 to 10 % where calls are long and lose 0.5 to
// 1 us to the splitting where they are short: bf16 there.
typedef uint32_t u32x6 __attribute__((ext_vector_type(6)));
typedef int i32x8 __attribute__((ext_vector_type(8)));
struct QueryPieces {
    u32x6 piece[3];
    uint32_t scales;                     // a byte each: exponent + 127
    __device__ __forceinline__ void make(const u32x4 (&bits)[4]) {
        typedef float f32x32 __attribute__((ext_vector_type(32)));
        uint32_t top = 0;
        f32x16 even, odd;
#pragma unroll
        for (int i = 0; i < 16; ++i) {
            const uint32_t w = bits[i / 4][i % 4];
            top = max(top, max(w & 0x7fffu, w >> 16 & 0x7fffu));
            even[i] = __uint_as_float(w << 16);
            odd[i] = __uint_as_float(w & 0xffff0000u);
        }
        const uint32_t e = (uint32_t)max((int)(top >> 7) - 2, 10);
        scales = top < 0x7f80u ? e | (e - 4) << 8 | (e - 9) << 16 : ~0u;         // (255: all products are NaN)
#pragma unroll
        for (int k = 0; k < 3; ++k) {
            const float s = __uint_as_float((e - (k == 0 ? 0u : k == 1 ? 4u : 9u)) << 23);
            piece[k] = __builtin_amdgcn_cvt_scalef32_2xpk16_fp6_f32(even, odd, s);
            // (the instruction writes before it has read all: its operands stay where they are)
            asm volatile("" :: "v"(even), "v"(odd), "v"(s), "v"(piece[k]));
            if (k == 2) break;
            const f32x32 was = __builtin_amdgcn_cvt_scalef32_pk32_f32_fp6(piece[k], s);
            asm volatile("" :: "v"(piece[k]), "v"(s), "v"(was));
#pragma unroll
            for (int i = 0; i < 16; ++i) {
                even[i] -= was[2 * i];
                odd[i] -= was[2 * i + 1];
            }
        }
    }
};
__device__ __forceinline__ i32x8 operand(u32x4 codes) { return i32x8{(int)codes[0], (int)codes[1], (int)codes[2], (int)codes[3], 0, 0, 0, 0}; }
__device__ __forceinline__ i32x8 operand(u32x6 piece) {
    return i32x8{(int)piece[0], (int)piece[1], (int)piece[2], (int)piece[3], (int)piece[4], (int)piece[5], 0, 0};
}

// 32 query rows of a wavefront.  S^T = K.Q^T, 32 keys x 32 rows, leaves lane (half, row) with keys 8 g + 4 half + i in register 4 g + i:
// as they stand, the operand of O^T += V^T.P^T for the 16 keys of page g / 2, if lane (half, column) of the other one holds the same.
template <int D>
struct WideRows {
    using W = WideLayout<D>;
    static constexpr int kOut = D / 32;
    QueryPieces q[D / 64];               // [t]: values 64 t + 32 half .. + 31 of the row
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
        for (int t = 0; t < D / 64; ++t) {
            u32x4 bits[4];
#pragma unroll
            for (int i = 0; i < 4; ++i) bits[i] = __builtin_bit_cast(u32x4, keep_if(real, ld16(p.q + at * D + t * 64 + half * 32 + i * 8)));
            q[t].make(bits);
        }
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

// K of a step, as it is stored: lane (half, key) holds the codes of values 64 t + 32 half .. + 31 and their scale.
template <int D>
struct WideKeys {
    u32x4 codes[D / 64];
    uint32_t scale[D / 64];
    __device__ __forceinline__ void read(const char *raw, int lane) {
        const int pg = lane >> 4 & 1, row = lane & 15, half = lane >> 5;
        const char *from = raw + (pg * (16 * D) + row * (D / 8) + half * (D == 128 ? 2 * D : 4 * D));
        const char *scales = raw + (WideLayout<D>::kCodes + pg * D + row + half * 16);
#pragma unroll
        for (int t = 0; t < D / 64; ++t) {
            if constexpr (D == 128) codes[t] = *reinterpret_cast<const u32x4 *>(from + t * (4 * D));
            else {
                const uint2 a = *reinterpret_cast<const uint2 *>(from), b = *reinterpret_cast<const uint2 *>(from + 2 * D);
                codes[t] = u32x4{a.x, a.y, b.x, b.y};
            }
            scale[t] = *reinterpret_cast<const uint8_t *>(scales + t * 32);
        }
    }
};

// Scores and products of kCols such groups of rows, each operand of the keys for all of them.
template <int D, int kCols>
__device__ __forceinline__ void scores(f32x16 (&x)[kCols], const WideRows<D> (&rows)[kCols], const WideKeys<D> &k) {
#pragma unroll
    for (int c = 0; c < kCols; ++c)
#pragma unroll
        for (int e = 0; e < 16; ++e) x[c][e] = 0.f;
    // (formats: 4 is e2m1, 2 is e2m3)
#pragma unroll
    for (int t = 0; t < D / 64; ++t)
#pragma unroll
        for (int c = 0; c < kCols; ++c) {
            const QueryPieces &q = rows[c].q[t];
            x[c] = __builtin_amdgcn_mfma_scale_f32_32x32x64_f8f6f4(operand(k.codes[t]), operand(q.piece[0]), x[c], 4, 2, 0, k.scale[t], 0, q.scales);
            x[c] = __builtin_amdgcn_mfma_scale_f32_32x32x64_f8f6f4(operand(k.codes[t]), operand(q.piece[1]), x[c], 4, 2, 0, k.scale[t], 1, q.scales);
            x[c] = __builtin_amdgcn_mfma_scale_f32_32x32x64_f8f6f4(operand(k.codes[t]), operand(q.piece[2]), x[c], 4, 2, 0, k.scale[t], 2, q.scales);
        }
}
// (operand t of the values)
template <int D, int kCols>
__device__ __forceinline__ void product(WideRows<D> (&rows)[kCols], const bf16x8 &v, int t) {
    constexpr int kOut = D / 32;
#pragma unroll
    for (int c = 0; c < kCols; ++c)
        rows[c].acc[t % kOut] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(v, __builtin_bit_cast(bf16x8, rows[c].pk[t / kOut]), rows[c].acc[t % kOut], 0, 0, 0);
}

// What one of D / 16 parts of a step's operands of V is made of: columns 2 b, 2 b + 1 of every chunk of a page for the lane's four keys.
template <int D>
struct Part {
    using W = WideLayout<D>;
    static constexpr int kWords = D / 32, kParts = D / 16;
    uint32_t vs, v[D == 128 ? 4 : 2];
    __device__ __forceinline__ void read(const char *raw, int part, int lane, int i16, int quad) {
        const int pg = part / kWords;
        const char *codes = raw + pg * (16 * D), *scales = raw + W::kCodes + pg * D;
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
    // in three pieces
    uint32_t y[4];
    __device__ __forceinline__ void write(int piece, char *v_to, int part, int i16, int quad) {
        const int pg = part / kWords, w = part % kWords;
        if (piece < 2) {
#pragma unroll
            for (int e = 2 * piece; e < 2 * piece + 2; ++e)
                y[e] = two_values<0>((D == 128 ? v[e] : v[e / 2] >> (e % 2 * 16)) >> (8 * w), scale_in(vs, e));
        } else {
            // (keys 4 quad .. + 3: half quad & 1 of the operand, place quad / 2 of its lanes)
            char *at = v_to + (pg * (D / 32) + w) * W::kFrag + (i16 + 32 * (quad & 1)) * 16 + (quad >> 1) * 8;
            *reinterpret_cast<uint2 *>(at) = make_uint2(__builtin_amdgcn_perm(y[1], y[0], 0x05040100), __builtin_amdgcn_perm(y[3], y[2], 0x05040100));
            *reinterpret_cast<uint2 *>(at + 16 * 16) = make_uint2(__builtin_amdgcn_perm(y[1], y[0], 0x07060302), __builtin_amdgcn_perm(y[3], y[2], 0x07060302));
        }
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
    int first_bad;                       // the first step, as far as windows have been taken, with a page that is not there
    __device__ __forceinline__ void ask(int c, int lane) const {
        asm("" : "+v"(lane));                            // (an address that is kept would cost registers)
        const int32_t *src = table + min(page0 + c * 64 + lane, max_pages - 1);
        const unsigned dst = (unsigned)(size_t)(lds_char *)reinterpret_cast<char *>(window) + (c & 1) * 256;
        asm volatile("s_mov_b32 m0, %1\n\tglobal_load_lds_dword %0, off" :: "v"(src), "s"(dst) : "memory", "m0");
    }
    __device__ __forceinline__ void take(int c, int lane) {
        const int id = window[(c & 1) * 64 + lane];
        const bool there = (unsigned)id < num_pages && (page0 + c * 64 + lane) * READER_PAGE_SIZE < keys;
        ok_then = __ballot(there);
        then = there ? id : 0;
        if (first_bad == 0x7fffffff && ~ok_then != 0) first_bad = c * 32 + (__builtin_ctzll(~ok_then) >> 1);
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
    // page pg of a step at most 11 ahead of step i; whether both pages of it are there
    __device__ __forceinline__ unsigned id(int step, int i, int pg) const {
        const int from = (step ^ i) & 32 ? then : now;
        return (unsigned)__builtin_amdgcn_readlane(from, (step * 2 + pg) & 63);
    }
    __device__ __forceinline__ unsigned there(int step, int i) const { return (unsigned)(((step ^ i) & 32 ? ok_then : ok_now) >> (step * 2 & 63)) & 3u; }
};

// Asynchronous copy to LDS: a lane of `lanes` moves 16 bytes to lds + 16 * lane.  (All lanes are active around it.)
__device__ __forceinline__ void copy_lanes(const char *base, unsigned lane_off, unsigned lds, unsigned long long lanes) {
    asm volatile("s_mov_b32 m0, %2\n\ts_mov_b64 exec, %3\n\tglobal_load_lds_dwordx4 %0, %1 nt\n\ts_mov_b64 exec, -1"
                 :: "v"(lane_off), "s"(base), "s"(lds), "s"(lanes) : "memory", "m0");
}

template <int D, int kWaves, int kCols, bool kTree>
__global__ __launch_bounds__(64 * kWaves) __attribute__((amdgpu_waves_per_eu(kCols == 1 ? 2 : 1, kCols == 1 ? 2 : 1))) void kvq_attn_wide_kernel(KvqAttnParams p) {
    using Rows = WideRows<D>;
    using W = WideLayout<D>;
    constexpr int kRows = kWaveRows * kCols * kWaves, kMinRange = 4 * kStep;
    constexpr int kCopies = 8 / kWaves;                  // copy instructions of a wavefront in a step
    constexpr int kParts = (Part<D>::kParts + kWaves - 1) / kWaves;          // parts of the operands that it makes
    // With eight wavefronts, the second of each SIMD is half a step behind the first: its barrier is in front of its second product, not
    // behind it, so that one of them has the matrix unit while the other makes weights.
    constexpr bool kOffset = kWaves == 8, kEarly = kCols == 2 || kOffset;
    // A barrier stands behind every kTurn steps: behind one step, or with eight wavefronts, which are not at the same place anyway, behind
    // two.  From one of them to the next, steps n to n + kTurn - 1, V's operands of these steps are read (by those behind from n - 1 on), K from
    // n + 2 on (n + 1), the operands of kTurn steps from n + 3 on are made, and the bytes of as many have to come that follow those.
    constexpr int kTurn = kOffset ? 2 : 1;
    constexpr int kVBuffers = kOffset ? 6 : 4;
    constexpr int kDepth = kOffset ? 5 : 3, kSlots = kOffset ? 9 : 6;         // bytes are asked for kDepth steps ahead of their use; steps of them in the ring
    __shared__ __attribute__((aligned(1024))) char s_frag[kVBuffers * W::kStepFrags];
    __shared__ __attribute__((aligned(1024))) char s_raw[kSlots * W::kRaw];
    __shared__ int s_ids[kWaves][2][64];
    __shared__ uint32_t s_mask[kTree ? READER_MAX_T : 1][4];
    __shared__ int s_up[kTree ? READER_MAX_T : 1];
    __shared__ int s_odd[kRows + 1];                     // in which turn a row, and any, was none that 32 bits hold
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
    int bad = 0, turn = 0;
    for (int i = threadIdx.x; i <= kRows; i += 64 * kWaves) s_odd[i] = 0;
    const unsigned raw_lds = (unsigned)(size_t)(lds_char *)&s_raw[0];
    // what this wavefront copies of a step: the first four 1 KB of codes each, the others the scales of a page; with four, both
    const int code_page = D == 128 ? (wave >> 1) & 1 : wave & 1, code_part = D == 128 ? wave & 1 : 0;
    constexpr unsigned long long scale_lanes = (1ull << (D / 16)) - 1;
    const int copy_page = wave < 4 ? code_page : wave & 1;
    const unsigned copy_from = wave < 4 ? code_part * 1024 : 16 * D;
    const unsigned copy_to = wave < 4 ? code_page * (16 * D) + code_part * 1024 : W::kCodes + (wave & 1) * D;
    const unsigned long long copy_which = wave < 4 ? ~0ull : scale_lanes;
    const bool late = kOffset && wave >= 4;
    const unsigned num_pages = (unsigned)(p.num_pages < 0x7fffffffLL ? p.num_pages : 0x7fffffffLL);

    WideBlock o = rg.at;
    for (bool first_block = true; !rg.behind(o); first_block = false) {
        int t0, t1;
        rg.share(o, first_block, tb, p.max_seq_len, t0, t1);
        const int keys = o.keys(tb, p.max_seq_len), nt = o.tokens(tb), row0 = o.c0 + o.k * tb, all = o.tiles(tb, p.max_seq_len);
        const long long p0 = (long long)o.L + o.k * tb;
        const bool last_block = rg.is_stop(o);
        if (t1 > t0) {
            ++turn;
            if constexpr (kTree) {
                if ((long long)t1 * kStep > o.L) ancestors(p.parents + (size_t)o.b * p.nodes, p.nodes, s_mask, s_up, bad);
            }
            const int steps = t1 - t0;
            const int unmasked = kTree ? o.L : (int)min(p0 + 1, (long long)p.max_seq_len);     // keys that every row sees
            PageWindow ids = {p.page_table + (size_t)o.b * p.max_pages, t0 * kStepPages, p.max_pages, keys, num_pages, &s_ids[wave][0][0], 0, 0, 0, 0, 0x7fffffff};
            const int full = keys / kStep - t0;          // steps in front of this one have 32 keys that somebody sees
            const int free = unmasked / kStep - t0;      // ... that every row sees
            auto whole_step = [&](int step) { return step < min(full, ids.first_bad); };
            const char *const cache = reinterpret_cast<const char *>(p.cache) + (size_t)o.head * KvqBlock<D>::kBytes;
            const unsigned page_bytes = (unsigned)p.Hkv * KvqBlock<D>::kBytes;
            auto issue = [&](int step, int now, unsigned slot) {     // (at step `now`) kCopies copy instructions, whatever the pages are
                if (kWaves == 4) {
                    copy_lanes(cache + (size_t)ids.id(step, now, code_page) * page_bytes + code_part * 1024, lane * 16, raw_lds + slot + code_page * (16 * D) + code_part * 1024, ~0ull);
                    copy_lanes(cache + (size_t)ids.id(step, now, wave & 1) * page_bytes + 16 * D, lane * 16, raw_lds + slot + W::kCodes + (wave & 1) * D, scale_lanes);
                } else {
                    copy_lanes(cache + (size_t)ids.id(step, now, copy_page) * page_bytes + copy_from, lane * 16, raw_lds + slot + copy_to, copy_which);
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
                    if ((kWaves == 4 || wave < 4) && code_page == pg && (D == 64 || code_part == 1)) {
#pragma unroll
                        for (int e = 0; e < 4; ++e) {
                            if (4 * (l >> 4) + e < n) continue;
                            if constexpr (D == 128) *reinterpret_cast<uint32_t *>(codes + 8 * D + l * 16 + e * 4) = 0;
                            else *reinterpret_cast<uint16_t *>(codes + 8 * D + l * 8 + e * 2) = 0;
                        }
                    }
                    if ((kWaves == 4 || wave >= 4) && (wave & 1) == pg) {        // a byte of the scales a lane, of the first D / 2
                        if (l < D / 2 && (l / (D / 8)) * 4 + l % 4 >= n) s_raw[slot + W::kCodes + pg * D + D / 2 + l] = 127;
                    }
                }
            };
            auto read_part = [&](Part<D> &part, int i, unsigned slot) { part.read(s_raw + slot, (wave + i * kWaves) % Part<D>::kParts, lane, i16, quad); };
            auto write_part = [&](Part<D> &part, int piece, int i, unsigned v_at) {
                part.write(piece, s_frag + v_at, (wave + i * kWaves) % Part<D>::kParts, i16, quad);
            };
            auto meet = [&] {
                __builtin_amdgcn_fence(__ATOMIC_RELEASE, "workgroup", "local");
                __builtin_amdgcn_s_barrier();
                __builtin_amdgcn_fence(__ATOMIC_ACQUIRE, "workgroup", "local");
                asm volatile("" ::: "memory");
            };
            ids.ask(0, lane);
            Rows rows[kCols];
            int row = lane;
            asm("" : "+v"(row));
            row = wave * (kWaveRows * kCols) + (row & 31);
#pragma unroll
            for (int c = 0; c < kCols; ++c) rows[c].load(p, o.head, row0, nt, row + c * kWaveRows, half);
            wait_vmcnt<0>();                             // the first page ids are there
            asm volatile("" ::: "memory");
            ids.take(0, lane);
            ids.now = ids.then; ids.ok_now = ids.ok_then;
            for (int s = 0; s < kDepth + 3; ++s) issue(s, 0, s * W::kRaw);
            wait_vmcnt<kCopies * (kDepth - kTurn)>();    // steps 0 to 2 + kTurn
            asm volatile("" ::: "memory");
            for (int s = 0; s < 3 + kTurn; ++s)
                if (!whole_step(s)) blank(s, 0, s * W::kRaw);
            meet();
            f32x16 x0[kCols], x1[kCols];
            WideKeys<D> k;                               // of step s + 1
            for (int s = 0; s < 4; ++s) {
                if (s == 2) {
                    meet();
                    k.read(s_raw, lane);
                    scores(x0, rows, k);
                    k.read(s_raw + W::kRaw, lane);
                    meet();
                }
                if (s == 3 && !late) break;              // (those behind make a step's part between the same barriers as the others)
                for (int i = 0; i < kParts; ++i) {
                    Part<D> part;
                    read_part(part, i, s * W::kRaw);
#pragma unroll
                    for (int piece = 0; piece < 3; ++piece) write_part(part, piece, i, s * W::kStepFrags);
                }
            }
            meet();
            if (late) issue(3 + kDepth, 0, (3 + kDepth) % kSlots * W::kRaw);      // (... and ask for one)
            auto masked = [&](int s) { return s >= min(free, ids.first_bad); };
            bool move = true;                            // (the reference is yet to be found)
            int s = 0;
            // (a step's reference is moved once: of scores so large that it cannot move by less, weights stay large)
            float most_now = kMostSum;
            // K of step s + 2 and the operands of V of step s are read; those of step s + 3 + late are made, of bytes that have come, and
            // bytes are asked for kDepth steps ahead of them.
            auto next = [](unsigned at, unsigned size, unsigned end) { return at + size == end ? 0u : at + size; };
            constexpr unsigned kVEnd = kVBuffers * W::kStepFrags, kRawEnd = kSlots * W::kRaw;
            const int behind = late ? 1 : 0;
            unsigned k_read = 2 * W::kRaw, v_read = 0, v_make = (3 + behind) % kVBuffers * W::kStepFrags;
            unsigned raw_make = (3 + behind) % kSlots * W::kRaw, raw_ask = (3 + behind + kDepth) % kSlots * W::kRaw;
            unsigned raw_new = (3 + kTurn) * W::kRaw;    // of the steps that come next
            auto barrier = [&] {
                if (kTurn == 2 && !(s & 1)) return;
                wait_vmcnt<kCopies * (kDepth - kTurn)>();    // steps s + 4 to s + 3 + kTurn have come
                asm volatile("" ::: "memory");
                for (int n = s + 4; n < s + 4 + kTurn; ++n) {
                    if (!whole_step(n)) blank(n, s, raw_new);
                    raw_new = next(raw_new, W::kRaw, kRawEnd);
                }
                meet();
            };
            // One step: the weights of the scores `xa` of step s, the scores `xb` of step s + 1, the products.  true: on with the next one.
            auto step = [&](const f32x16 (&xa)[kCols], f32x16 (&xb)[kCols]) -> bool {
                typename Rows::Frags v;
                Rows::read(v, s_frag + v_read, lane);
                Part<D> part[kEarly ? kParts : 1];
                if constexpr (kEarly && !kOffset) {
#pragma unroll
                    for (int i = 0; i < kParts; ++i) read_part(part[i], i, raw_make);
                }
                scores(xb, rows, k);
                float sum[kCols], most = 0.f;
#pragma unroll
                for (int c = 0; c < kCols; ++c) {
                    sum[c] = rows[c].weights(xa[c], p.scale_log2);
                    most = fmaxf(most, sum[c]);
                }
                // the order: a product and a part of the weights in turn, what is read between them
#pragma unroll
                for (int i = 0; i < 3 * D / 64 * kCols; ++i) {
                    __builtin_amdgcn_sched_group_barrier(0x008, 1, 0);
                    __builtin_amdgcn_sched_group_barrier(0x100, 2, 0);
                    __builtin_amdgcn_sched_group_barrier(0x002, 56 / (3 * D / 64), 0);
                }
                // (here, and not behind the branch, where nothing would be beside them)
#pragma unroll
                for (int c = 0; c < kCols; ++c) asm volatile("" : "+v"(xb[c]));
                if (__any(most > most_now)) {
                    move = true;
                    return false;
                }
#pragma unroll
                for (int c = 0; c < kCols; ++c) rows[c].l = sum[c];
                if (kOffset && late) barrier();
                __builtin_amdgcn_s_setprio(1);           // (products in front of the other wavefront's weights)
                issue(s + 3 + behind + kDepth, s, raw_ask);
                if constexpr (kOffset) read_part(part[0], 0, raw_make);
                k.read(s_raw + k_read, lane);
                if constexpr (kOffset) {
#pragma unroll
                    for (int i = 0; i < W::kFrags; ++i) product(rows, v[i], i);
#pragma unroll
                    for (int piece = 0; piece < 3; ++piece) write_part(part[0], piece, 0, v_make);
#pragma unroll
                    for (int i = 0; i < W::kFrags; ++i) {
                        __builtin_amdgcn_sched_group_barrier(0x100, 2, 1);
                        __builtin_amdgcn_sched_group_barrier(0x008, 1, 1);
                        __builtin_amdgcn_sched_group_barrier(0x002, 4, 1);
                    }
                } else {
                    // (the order is kept: a product, then a piece of the operands to come, while the matrix unit works on it; 2 to 4 % faster,
                    // but where another wavefront's weights fill the gaps 2 % slower)
#pragma unroll
                    for (int i = 0; i < W::kFrags; ++i) {
                        product(rows, v[i], i);
                        if (i < 3 * kParts) {
                            if (!kEarly && i % 3 == 0) read_part(part[0], i / 3, raw_make);  // (beside the scores there are no registers for them)
                            write_part(part[kEarly ? i / 3 : 0], i % 3, i / 3, v_make);
                        }
                        __builtin_amdgcn_sched_barrier(0);
                    }
                }
                __builtin_amdgcn_s_setprio(0);
                if (!(kOffset && late)) barrier();
                k_read = next(k_read, W::kRaw, kRawEnd);
                v_read = next(v_read, W::kStepFrags, kVEnd);
                v_make = next(v_make, W::kStepFrags, kVEnd);
                raw_make = next(raw_make, W::kRaw, kRawEnd);
                raw_ask = next(raw_ask, W::kRaw, kRawEnd);
                most_now = kMostSum;
                ++s;
                if (s >= steps) return false;
                ids.advance(s, steps, lane);
                return !masked(s);
            };
            ids.advance(0, steps, lane);
            // (references are moved, and scores masked, outside the loop over the steps: a path around the accumulators inside it is paid for in
            // every step)
            while (s < steps) {
                if (masked(s)) {
                    const int j0 = (t0 + s) * kStep;
                    const unsigned there = ids.there(s, s);
                    if ((j0 < keys && !(there & 1)) || (j0 + READER_PAGE_SIZE < keys && !(there & 2))) bad |= READER_STATUS_BAD_PAGE;
#pragma unroll
                    for (int c = 0; c < kCols; ++c) {
                        int r = row + c * kWaveRows;
                        asm volatile("" : "+v"(r) :: "memory");      // (what follows from the row is found again: kept through the steps, it would cost registers)
                        const int tok = min(Rows::token(p, r), nt - 1), lim = (int)min(p0 + tok + 1, (long long)p.max_seq_len);
                        const uint32_t *mask = s_mask[kTree ? o.k * tb + tok : 0];
#pragma unroll
                        for (int e = 0; e < 16; ++e) {
                            const int at = e / 4 * 8 + half * 4 + e % 4, key = j0 + at, n = key - o.L;
                            // (no branches: with them the compiler has lost the assignment on one of the ways)
                            bool sees = ((there >> (e / 8) & 1u) != 0) & (key < lim);
                            if constexpr (kTree) sees &= (n < 0) | ((mask[(n >> 5) & 3] >> (n & 31) & 1u) != 0);
                            x0[c][e] = sees ? x0[c][e] : -INFINITY;
                        }
                    }
                }
                if (move) {
#pragma unroll
                    for (int c = 0; c < kCols; ++c) rows[c].move_reference(x0[c], p.scale_log2);
                    move = false;
                    most_now = INFINITY;
                }
                bool on;
                // (the loop's first products start in front of a line of 64 bytes or well inside one: across its end, long calls take 3 % more)
                asm volatile(".p2align 6");
                do {
                    on = step(x0, x1);
                    if (move) break;
                    if (on) {
                        on = step(x1, x0);
                        if (!move) continue;
                        on = false;
                    }
#pragma unroll
                    for (int c = 0; c < kCols; ++c) x0[c] = x1[c];
                } while (on);
            }
#pragma unroll
            for (int c = 0; c < kCols; ++c) {
                float check[2] = {0.f, 0.f};             // (not a number once any value is none)
#pragma unroll
                for (int b = 0; b < Rows::kOut; ++b)
#pragma unroll
                    for (int e = 0; e < 16; e += 4) {
                        check[0] = no_number(check[0], rows[c].acc[b][e], rows[c].acc[b][e + 1]);
                        check[1] = no_number(check[1], rows[c].acc[b][e + 2], rows[c].acc[b][e + 3]);
                    }
                // (a sum that is none is a query's doing)
                if (check[0] + check[1] != 0.f && rows[c].l < INFINITY) {
                    int r = row + c * kWaveRows;
                    asm volatile("" : "+v"(r));
                    if (Rows::token(p, r) < nt) s_odd[r] = s_odd[kRows] = turn;
                }
            }
            wait_vmcnt<0>();                             // copies that nobody needed
            asm volatile("" ::: "memory");
            meet();
            // ---- end of the segment: the whole block is normalised and written out, a part of one leaves a record
            const bool whole = t0 == 0 && t1 == all;
            float *rec = reinterpret_cast<float *>(reinterpret_cast<char *>(p.workspace) + kNotesBytes) +
                         (size_t)(2 * range + (t0 == 0 ? 1 : 0)) * ((size_t)kRows * (D + 2));
#pragma unroll
            for (int c = 0; c < kCols; ++c) {
                int half_ = half, r = row + c * kWaveRows;
                asm volatile("" : "+v"(r), "+v"(half_) :: "memory");
                const float sum = rows[c].l + __shfl_xor(rows[c].l, 32), inv = sum == 0.f ? 0.f : 1.f / sum;
                const int tok = Rows::token(p, r);
                const bool real = tok < nt;
                const size_t at = Rows::out_row(p, o.head, row0, nt, r);
#pragma unroll
                for (int g = 0; g < 2; ++g)
#pragma unroll
                    for (int i = 0; i < 4; ++i) {        // the D / 16 values of chunk 8 g + 4 half + i
                        const int chunk = 8 * g + 4 * half_ + i;
#pragma unroll
                        for (int h = 0; h < D / 64; ++h) {
                            const f32x4 v = f32x4{rows[c].acc[2 * h][4 * g + i], rows[c].acc[2 * h][4 * g + 8 + i], rows[c].acc[2 * h + 1][4 * g + i],
                                                  rows[c].acc[2 * h + 1][4 * g + 8 + i]} * inv;
                            const int piece = chunk * (D / 64) + h;
                            if (!whole) reinterpret_cast<f32x4 *>(rec)[piece * kRows + r] = v;
                            else if (real) *reinterpret_cast<uint2 *>(p.out + at * D + piece * 4) = make_uint2(pack_bf16x2(v[0], v[1]), pack_bf16x2(v[2], v[3]));
                        }
                    }
                if (half_ == 0) {
                    if (!whole) {
                        rec[(size_t)kRows * D + r] = sum == 0.f ? -INFINITY : rows[c].m;
                        rec[(size_t)kRows * (D + 1) + r] = sum;
                    } else if (real && p.lse) {
                        p.lse[lse_at(p, o.b, row0, o.k * tb, tok, o.head * p.G + r - tok * p.G)] = sum == 0.f ? -INFINITY : (rows[c].m + __builtin_amdgcn_logf(sum)) * kLn2;
                    }
                }
            }
            if (__builtin_expect(s_odd[kRows] == turn, 0)) {
                wait_vmcnt<0>();
                asm volatile("" ::: "memory");
                meet();
                rows_as_means<D, kTree>(p, o, nt * p.G, s_odd, turn, wave, kWaves, t0 * kStep, min(t1 * kStep, keys), s_mask, whole ? nullptr : rec, kRows, lane);
            }
        }
        if (last_block) break;
        o.next(seqs, p.B, tb);
        o = o.of_lane(0);
    }
    if (p.status && bad) atomicOr(p.status, bad);
}

template <int D, int kWaves, int kCols>
hipError_t launch_wide(KvqAttnParams p, hipStream_t stream) {
    constexpr int kRows = kWaveRows * kCols * kWaves;
    p.n_ranges = kNumCU * 8 / (kWaves * kCols);          // (as many as run at once)
    p.tokens_per_block = kRows / p.G;
    if (p.nodes > 0) hipLaunchKernelGGL((kvq_attn_wide_kernel<D, kWaves, kCols, true>), dim3(p.n_ranges), dim3(64 * kWaves), 0, stream, p);
    else hipLaunchKernelGGL((kvq_attn_wide_kernel<D, kWaves, kCols, false>), dim3(p.n_ranges), dim3(64 * kWaves), 0, stream, p);
    const hipError_t e = hipGetLastError();
    if (e != hipSuccess) return note_hip_error("launch kvq_attn_wide_kernel", e);
    return launch_prompt_merge(p, kRows, stream);
}

}  // namespace

hipError_t launch_kvq_attn_wide(const KvqAttnParams &p, int rows, hipStream_t stream) {
    if (rows == 128) return p.D == 64 ? launch_wide<64, 4, 1>(p, stream) : launch_wide<128, 4, 1>(p, stream);
    return p.D == 64 ? launch_wide<64, 4, 2>(p, stream) : launch_wide<128, 8, 1>(p, stream);
}

}  // namespace reader

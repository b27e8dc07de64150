// Attention over a cache in 4 bits, of packed prompts, chunks and single tokens (causal) and of draft trees whose rows are in the
// cache behind their sequence (ancestors only): few query rows a kv head here, 128 and more in kvq_attn_wide.hip.
//
//   out = sum_j w_j V_j / sum_j w_j,  w_j = 2^(c q.K_j - m),  c = scale * log2(e),  one pass over the keys j that a row sees
//
// A value is its code's times a power of two, exact in bf16: codes become operands by one instruction for two of them, and everything
// behind is an attention in bf16 with 32-bit sums.  A lane's bytes of a page are one load of K and one of V, each wavefront's 1 KB in a
// piece, straight into registers two steps of 32 keys ahead: nothing is shared between wavefronts before their rows' ends, so there is
// no barrier in the loop and eight wavefronts can walk the keys of one block side by side.  The reference m is moved only where a
// lane's sum passes 2^16: a wavefront's exponentials do not wait for maxima.
//
// What bounds it: bytes where each kv head has a handful of rows (16 sequences of 1 K to 16 K positions, one token each, 32 and 8 heads of
// 128: 153 MB in 43 us, in 41 if the last-level cache holds them; 6 to find the work and the first pages, 5 for the second launch, in
// between at the rate of a copy); the chain page id, page, products, exponentials, sums of wavefronts in small calls (a tree of 16
// nodes on 512 positions, 8 heads of 64: 7.3 us, the launch 4 of them); exponentials and the making of operands, which every block of
// rows does anew, in between: the more rows a workgroup has, the fewer times (64 trees of 32 nodes on 6000 positions: 540 us
// with 16 rows a workgroup, 329 with 32, 303 with 64, 225 with the wide kernel's 128).
#include <math.h>

#include "kvq_attn.h"

namespace reader {

namespace {

using Block = PromptBlock<kStep, 2 * kStep, 4 * kStep>;

// One lane's bytes of a page: K of row i16 and quarter `quad`, V of rows 4 quad .. + 3 and chunk i16.
template <int D>
struct KvqPage {
    static constexpr int kWords = D / 32;
    uint32_t k[kWords], v[kWords], ks, vs;
    // kOnce: nobody else reads these bytes in this call: past the caches, which they would only fill (16 tokens on 9000 positions each, keys that
    // no call in front has read: 36.7 us instead of 40.3; 64 on 6000: 75.4 instead of 88.9; where blocks share keys 5 to 8 % slower).
    template <bool kOnce>
    __device__ __forceinline__ void load(const uint8_t *block, int lane, int i16, int quad) {
        using B = KvqBlock<D>;
        typedef uint32_t words __attribute__((ext_vector_type(kWords)));
        const words *const k_at = reinterpret_cast<const words *>(block + lane * (kWords * 4));
        const words *const v_at = reinterpret_cast<const words *>(block + B::kV + lane * (kWords * 4));
        const words kw = kOnce ? __builtin_nontemporal_load(k_at) : *k_at, vw = kOnce ? __builtin_nontemporal_load(v_at) : *v_at;
#pragma unroll
        for (int w = 0; w < kWords; ++w) { k[w] = kw[w]; v[w] = vw[w]; }
        ks = block[B::kKScales + (D == 128 ? quad : quad >> 1) * 16 + i16];
        vs = *reinterpret_cast<const uint32_t *>(block + B::kVScales + quad * (D / 8) + (i16 * B::kChunk / 32) * 4);
    }
    // takes row e of the lane's four out of V
    __device__ __forceinline__ void drop(int e) {
        if constexpr (D == 128) v[e] = 0;
        else v[e / 2] &= 0xffffu << (e % 2 ? 0 : 16);
        vs = (vs & ~(255u << (8 * e))) | (127u << (8 * e));
    }
};

// kBlocks blocks of 16 query rows, carried through 32 keys at a time.  S^T = K.Q^T leaves lane (quad, i16) with four scores of row
// i16 for each page, keys 4 quad .. + 3: as they stand, the operand of O^T += V^T.P^T whose other one is the lane's V.
template <int D, int kBlocks>
struct KvqRows {
    static constexpr int kSteps = D / 32, kOut = D / 16;
    bf16x8 q[kBlocks][kSteps];                                // step s: values (D / 4) quad + 8 s .. + 7 of row i16
    int lim[kBlocks], node[kBlocks];                          // keys that row i16 sees (trees: at most), its node
    bool real[kBlocks];
    f32x4 acc[kBlocks][kOut];                                 // [i][k]: output value (4 quad + k) D / 16 + i of row i16
    float m[kBlocks], l[kBlocks];                             // reference (exponent of two), this lane's part of the sum
    f32x4 x[kBlocks][kStepPages];                             // scores
    u32x4 pk[kBlocks];                                        // weights of 32 keys, an operand

    __device__ static __forceinline__ size_t out_row(const PromptParams &p, int head, int row0, int nt, int row) {
        const int tok = (int)(((float)row + 0.5f) * p.g_rcp);
        return ((size_t)row0 + min(tok, nt - 1)) * p.Hq + (size_t)head * p.G + (row - tok * p.G);
    }
    __device__ __forceinline__ void load(const PromptParams &p, int head, int row0, long long p0, int node0, int nt, int first, int i16, int quad) {
#pragma unroll
        for (int r = 0; r < kBlocks; ++r) {
            const int row = first + r * 16 + i16, tok = (int)(((float)row + 0.5f) * p.g_rcp);    // row / G
            real[r] = tok < nt;
            node[r] = node0 + min(tok, nt - 1);
            lim[r] = real[r] ? (int)min(p0 + tok + 1, (long long)p.max_seq_len) : 0;
            const size_t at = out_row(p, head, row0, nt, row);
#pragma unroll
            for (int s = 0; s < kSteps; ++s) q[r][s] = __builtin_bit_cast(bf16x8, keep_if(real[r], ld16(p.q + at * D + quad * (D / 4) + s * 8)));
            m[r] = kNoReference;
            l[r] = 0.f;
#pragma unroll
            for (int i = 0; i < kOut; ++i) acc[r][i] = f32x4{0.f, 0.f, 0.f, 0.f};
        }
    }
    __device__ __forceinline__ void scores(const KvqPage<D> (&pages)[kStepPages]) {
#pragma unroll
        for (int pg = 0; pg < kStepPages; ++pg) {
            const float sc = scale_of(pages[pg].ks);
#pragma unroll
            for (int r = 0; r < kBlocks; ++r) x[r][pg] = f32x4{0.f, 0.f, 0.f, 0.f};
#pragma unroll
            for (int s = 0; s < kSteps; ++s) {
                const uint32_t w = pages[pg].k[s];
                const u32x4 k = {two_values<0>(w, sc), two_values<1>(w, sc), two_values<2>(w, sc), two_values<3>(w, sc)};
#pragma unroll
                for (int r = 0; r < kBlocks; ++r)
                    x[r][pg] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(__builtin_bit_cast(bf16x8, k), q[r][s], x[r][pg], 0, 0, 0);
            }
        }
    }
    // Weights of the scores, and what the lane's sums become with them: the largest of those.
    __device__ __forceinline__ float weights(float c2, float (&sum)[kBlocks]) {
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
    // Moves the references so that no weight of the scores at hand is above one, nor a row's sum.
    __device__ __forceinline__ void move_references(float c2) {
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
        }
    }
    __device__ __forceinline__ void products(const KvqPage<D> (&pages)[kStepPages]) {
        float sc[kStepPages][4];
#pragma unroll
        for (int pg = 0; pg < kStepPages; ++pg)
#pragma unroll
            for (int e = 0; e < 4; ++e) sc[pg][e] = scale_in(pages[pg].vs, e);
        two_columns<0>(pages, sc);
        two_columns<1>(pages, sc);
        if constexpr (D == 128) {
            two_columns<2>(pages, sc);
            two_columns<3>(pages, sc);
        }
    }
    // columns 2 kPair and 2 kPair + 1 of every chunk
    template <int kPair>
    __device__ __forceinline__ void two_columns(const KvqPage<D> (&pages)[kStepPages], const float (&sc)[kStepPages][4]) {
        u32x4 even, odd;
#pragma unroll
        for (int pg = 0; pg < kStepPages; ++pg) {
            uint32_t y[4];
            if constexpr (D == 128) {
#pragma unroll
                for (int e = 0; e < 4; ++e) y[e] = two_values<kPair>(pages[pg].v[e], sc[pg][e]);
            } else {
                y[0] = two_values<kPair>(pages[pg].v[0], sc[pg][0]);
                y[1] = two_values<2 + kPair>(pages[pg].v[0], sc[pg][1]);
                y[2] = two_values<kPair>(pages[pg].v[1], sc[pg][2]);
                y[3] = two_values<2 + kPair>(pages[pg].v[1], sc[pg][3]);
            }
            even[2 * pg] = __builtin_amdgcn_perm(y[1], y[0], 0x05040100);
            even[2 * pg + 1] = __builtin_amdgcn_perm(y[3], y[2], 0x05040100);
            odd[2 * pg] = __builtin_amdgcn_perm(y[1], y[0], 0x07060302);
            odd[2 * pg + 1] = __builtin_amdgcn_perm(y[3], y[2], 0x07060302);
        }
#pragma unroll
        for (int r = 0; r < kBlocks; ++r) {
            acc[r][2 * kPair] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(__builtin_bit_cast(bf16x8, even), __builtin_bit_cast(bf16x8, pk[r]), acc[r][2 * kPair], 0, 0, 0);
            acc[r][2 * kPair + 1] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(__builtin_bit_cast(bf16x8, odd), __builtin_bit_cast(bf16x8, pk[r]), acc[r][2 * kPair + 1], 0, 0, 0);
        }
    }
    // Four output values of row i16, number n of the lane's kOut / 4 * 4 such pieces, and the piece's place among the row's D / 4.
    __device__ __forceinline__ f32x4 piece(int r, int n) const {
        const int k = n / (kOut / 4), h = n % (kOut / 4);
        return f32x4{acc[r][4 * h][k], acc[r][4 * h + 1][k], acc[r][4 * h + 2][k], acc[r][4 * h + 3][k]};
    }
    __device__ static __forceinline__ int piece_at(int n, int quad) { return (4 * quad + n / (kOut / 4)) * (kOut / 4) + n % (kOut / 4); }
    __device__ __forceinline__ void finish_sums() {
#pragma unroll
        for (int r = 0; r < kBlocks; ++r) {
            l[r] += __shfl_xor(l[r], 16);
            l[r] += __shfl_xor(l[r], 32);
        }
    }
};

// kRowWaves groups of 16 kBlocks rows, each carried by kKeyWaves wavefronts that take the steps of 32 keys in turn.  kCut: a workgroup
// takes a range of the (head, sequence, block of query rows, key) axis, and blocks that are cut leave records for a second launch;
// else it takes a block.  kOnce: a sequence's keys are read by one block of a kv head.
template <int D, int kBlocks, int kRowWaves, int kKeyWaves, bool kTree, bool kCut, bool kOnce>
__global__ __launch_bounds__(64 * kRowWaves * kKeyWaves) void kvq_attn_kernel(KvqAttnParams p) {
    using Rows = KvqRows<D, kBlocks>;
    constexpr int kWaveRows = kBlocks * 16, kRows = kWaveRows * kRowWaves, kWaves = kRowWaves * kKeyWaves;
    constexpr int kMinRange = 8 * kStep;
    __shared__ __attribute__((aligned(16))) f32x4 s_part[kWaves][kWaveRows * D / 4];
    __shared__ float s_sum[kWaves][2][kWaveRows];
    __shared__ uint32_t s_mask[kTree ? READER_MAX_T : 1][4];
    __shared__ int s_up[kTree ? READER_MAX_T : 1];
    __shared__ int s_odd[kRows + 1];                     // in which turn a row, and any, was none that 32 bits hold
    const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    const int row_wave = wave / kKeyWaves, key_wave = wave % kKeyWaves;
    const int i16 = lane & 15, quad = lane >> 4, tb = p.tokens_per_block;
    RangeNote *const notes = reinterpret_cast<RangeNote *>(p.workspace);
    const Sequences seqs{p.seq_lens, p.cu_tokens, p.N, p.max_seq_len, kTree ? p.nodes : 0};
    const int range = blockIdx.x;
    int bad = 0, turn = 0;
    for (int i = threadIdx.x; i <= kRows; i += 64 * kWaves) s_odd[i] = 0;
    Block o;
    PromptRange<Block> rg;
    if constexpr (kCut) {
        int t_place;
        if (!find_range<Block, kMinRange, kTree>(p, seqs, lane, o, t_place)) return;
        rg = PromptRange<Block>(o, t_place, p.Hkv);
        const RangeNote note = rg.note(seqs, p.B, tb, lane);
        if (threadIdx.x == 0) notes[range] = note;
        o = rg.at;
    } else {
        if (blockIdx.x == 0 && blockIdx.y == 0) report_sequences<kTree>(p, blockDim.x);
        o.head = blockIdx.y;
        if (!find_block<kTree>(p, seqs, blockIdx.x, lane, o)) return;
    }
    for (bool first_block = true; !kCut || !rg.behind(o); first_block = false) {
        const int keys = o.keys(tb, p.max_seq_len), nt = o.tokens(tb), row0 = o.c0 + o.k * tb, all = o.tiles(tb, p.max_seq_len);
        int t0 = 0, t1 = all;
        if constexpr (kCut) rg.share(o, first_block, tb, p.max_seq_len, t0, t1);
        const long long p0 = (long long)o.L + o.k * tb;
        const bool last_block = !kCut || rg.is_stop(o);
        if (t1 > t0) {
            ++turn;
            if constexpr (kTree) {
                if ((long long)t1 * kStep > o.L) ancestors(p.parents + (size_t)o.b * p.nodes, p.nodes, s_mask, s_up, bad);
            }
            const int first = row_wave * kWaveRows;
            // steps key_wave, key_wave + kKeyWaves, ... of the segment are this wavefront's (none, if it has no rows)
            const int steps = first < nt * p.G ? (t1 - t0 - key_wave + kKeyWaves - 1) / kKeyWaves : 0;
            // (through the scalar cache: among the loads of keys, an id that is waited for would wait for all of them)
            const auto *table = (const __attribute__((address_space(4))) int32_t *)(uintptr_t)(p.page_table + (size_t)o.b * p.max_pages);
            const int unmasked = kTree ? o.L : (int)min(p0 + 1, (long long)p.max_seq_len);     // keys that every row sees
            // pages of step j: their ids, -1 for one that is not there (nobody sees its keys)
            auto page_id = [&](int j, int pg) {
                const int at = (t0 + key_wave + j * kKeyWaves) * kStepPages + pg;
                const bool there = j < steps && at * READER_PAGE_SIZE < keys;
                const int id = table[there ? at : 0];
                return there && id >= 0 && id < p.num_pages ? id : -1;
            };
            auto load = [&](KvqPage<D> (&to)[kStepPages], const int (&id)[kStepPages]) {
#pragma unroll
                for (int pg = 0; pg < kStepPages; ++pg)
                    to[pg].template load<kOnce>(p.cache + ((size_t)max(id[pg], 0) * p.Hkv + o.head) * KvqBlock<D>::kBytes, lane, i16, quad);
            };
            Rows rows;
            rows.load(p, o.head, row0, p0, o.k * tb, nt, first, i16, quad);
            if (steps > 0) {
                int id[kStepPages] = {page_id(0, 0), page_id(0, 1)}, id1[kStepPages] = {page_id(1, 0), page_id(1, 1)};
                int id2[kStepPages] = {page_id(2, 0), page_id(2, 1)};
                KvqPage<D> now[kStepPages], next[kStepPages], then[kStepPages];
                load(now, id);
                load(next, id1);
                int j = 0, moved_at = -1;
                // (a step's references are moved once: of scores so large that a reference cannot move by less, weights may stay large)
                // (the references are moved outside the loop over the steps: a path around its accumulators inside it is paid for in every step)
                while (true) {
                    bool move = false;
                    for (; j < steps; ++j) {
                        load(then, id2);
                        const int id3[kStepPages] = {page_id(j + 3, 0), page_id(j + 3, 1)};
                        const int j0 = (t0 + key_wave + j * kKeyWaves) * kStep;
                        rows.scores(now);
                        if (j0 + kStep > unmasked || id[0] < 0 || id[1] < 0) {
#pragma unroll
                            for (int pg = 0; pg < kStepPages; ++pg) {
                                const int jp = j0 + pg * READER_PAGE_SIZE;
                                if (jp < keys && id[pg] < 0) bad |= READER_STATUS_BAD_PAGE;
#pragma unroll
                                for (int e = 0; e < 4; ++e) {
                                    const int key = jp + quad * 4 + e, n = key - o.L;
                                    const bool nobody = id[pg] < 0 || key >= keys;
                                    if (nobody) now[pg].drop(e);
#pragma unroll
                                    for (int r = 0; r < kBlocks; ++r) {
                                        // (no branches: with them the compiler has lost the assignment on one of the ways)
                                        bool sees = !nobody & (key < rows.lim[r]);
                                        if constexpr (kTree) sees &= (n < 0) | ((s_mask[rows.node[r]][(n >> 5) & 3] >> (n & 31) & 1u) != 0);
                                        rows.x[r][pg][e] = sees ? rows.x[r][pg][e] : -INFINITY;
                                    }
                                }
                            }
                        }
                        float sum[kBlocks];
                        if (__any(rows.weights(p.scale_log2, sum) > kMostSum) & (j != moved_at)) {
                            move = true;
                            break;
                        }
#pragma unroll
                        for (int r = 0; r < kBlocks; ++r) rows.l[r] = sum[r];
                        rows.products(now);
#pragma unroll
                        for (int pg = 0; pg < kStepPages; ++pg) {
                            now[pg] = next[pg];
                            next[pg] = then[pg];
                            id[pg] = id1[pg];
                            id1[pg] = id2[pg];
                            id2[pg] = id3[pg];
                        }
                    }
                    if (!move) break;
                    rows.move_references(p.scale_log2);
                    moved_at = j;
                }
            }
            rows.finish_sums();
            // ---- end of the segment: the whole block is normalised and written out, a part of one leaves a record
            const bool whole = t0 == 0 && t1 == all;
            float *rec = reinterpret_cast<float *>(reinterpret_cast<char *>(p.workspace) + kNotesBytes) +
                         (size_t)(2 * range + (t0 == 0 ? 1 : 0)) * ((size_t)kRows * (D + 2));
            constexpr int kPieces = D / 16;                  // a lane's of a row
            auto write = [&](int r, int piece, f32x4 v) {
                const int row = first + r * 16 + i16;
                if (!whole) reinterpret_cast<f32x4 *>(rec)[piece * kRows + row] = v;
                else if (rows.real[r])
                    *reinterpret_cast<uint2 *>(p.out + Rows::out_row(p, o.head, row0, nt, row) * D + piece * 4) = make_uint2(pack_bf16x2(v[0], v[1]), pack_bf16x2(v[2], v[3]));
            };
            auto write_sums = [&](int r, float top, float sum) {
                const int row = first + r * 16 + i16;
                if (!whole) {
                    rec[(size_t)kRows * D + row] = sum == 0.f ? -INFINITY : top;
                    rec[(size_t)kRows * (D + 1) + row] = sum;
                } else if (rows.real[r] && p.lse) {
                    const int tok = (int)(((float)row + 0.5f) * p.g_rcp);
                    p.lse[lse_at(p, o.b, row0, o.k * tb, tok, o.head * p.G + row - tok * p.G)] = sum == 0.f ? -INFINITY : (top + __builtin_amdgcn_logf(sum)) * kLn2;
                }
            };
            // the wavefronts that share rows add them up: [D / 4 pieces][rows], a part of the pieces each
#pragma unroll
            for (int r = 0; r < kBlocks; ++r) {
#pragma unroll
                for (int n = 0; n < kPieces; ++n) s_part[wave][Rows::piece_at(n, quad) * kWaveRows + r * 16 + i16] = rows.piece(r, n);
                if (quad == 0) { s_sum[wave][0][r * 16 + i16] = rows.m[r]; s_sum[wave][1][r * 16 + i16] = rows.l[r]; }
            }
            __syncthreads();
#pragma unroll
            for (int r = 0; r < kBlocks; ++r) {
                const int row = r * 16 + i16, w0 = row_wave * kKeyWaves;
                float top = kNoReference, sum = 0.f, f[kKeyWaves];
#pragma unroll
                for (int w = 0; w < kKeyWaves; ++w) top = fmaxf(top, s_sum[w0 + w][0][row]);
#pragma unroll
                for (int w = 0; w < kKeyWaves; ++w) {
                    // (a wavefront whose rows saw nothing has no say, whatever its reference)
                    const float lw = s_sum[w0 + w][1][row];
                    f[w] = lw == 0.f ? 0.f : __builtin_amdgcn_exp2f(s_sum[w0 + w][0][row] - top);
                    sum += lw * f[w];
                }
                const float inv = sum == 0.f ? 0.f : 1.f / sum;
                float check = 0.f;                       // (not a number once any value is none)
                constexpr int kMine = (D / 4 + 4 * kKeyWaves - 1) / (4 * kKeyWaves);
#pragma unroll
                for (int c = 0; c < kMine; ++c) {
                    const int piece = (key_wave * kMine + c) * 4 + quad;
                    if (D / 4 % (4 * kKeyWaves) != 0 && piece >= D / 4) break;
                    f32x4 v = {0.f, 0.f, 0.f, 0.f};
#pragma unroll
                    for (int w = 0; w < kKeyWaves; ++w) v += s_part[w0 + w][piece * kWaveRows + row] * f[w];
                    v *= inv;
                    check = no_number(no_number(check, v[0], v[1]), v[2], v[3]);
                    write(r, piece, v);
                }
                // (a sum that is none is a query's doing)
                if (rows.real[r] && check != 0.f && sum < INFINITY) s_odd[first + row] = s_odd[kRows] = turn;
                if (key_wave == 0 && quad == 0) write_sums(r, top, sum);
            }
            __syncthreads();                             // everybody is done with the others' rows
            if (__builtin_expect(s_odd[kRows] == turn, 0)) {
                wait_vmcnt<0>();
                __syncthreads();
                rows_as_means<D, kTree>(p, o, nt * p.G, s_odd, turn, wave, kWaves, t0 * kStep, min(t1 * kStep, keys), s_mask, whole ? nullptr : rec, kRows, lane);
            }
        }
        if (last_block) break;
        if constexpr (kCut) {
            o.next(seqs, p.B, tb);
            o = o.of_lane(0);
        }
    }
    if (p.status && bad) atomicOr(p.status, bad);
}

// Blocks of a kv head, at most, whatever the bounds are: every sequence has one that is not full, and no row is in two (find_block).
int block_count(const KvqAttnParams &p) {
    if (p.nodes > 0) return p.B * ((p.nodes + p.tokens_per_block - 1) / p.tokens_per_block);
    return (int)min((long long)p.N, (long long)p.N / p.tokens_per_block + p.B);
}

template <int D, int kBlocks, int kRowWaves, int kKeyWaves, bool kCut>
hipError_t launch(KvqAttnParams p, int ranges, hipStream_t stream) {
    constexpr int kRows = 16 * kBlocks * kRowWaves;
    p.n_ranges = ranges;
    p.tokens_per_block = kRows / p.G;
    const dim3 grid = kCut ? dim3(ranges) : dim3(block_count(p), p.Hkv), block(64 * kRowWaves * kKeyWaves);
    // single tokens, and as many as a block holds of every sequence (if they have alike)
    const bool once = kRows == 16 && p.nodes == 0 && p.N <= (long long)p.B * p.tokens_per_block;
    if (p.nodes > 0) hipLaunchKernelGGL((kvq_attn_kernel<D, kBlocks, kRowWaves, kKeyWaves, true, kCut, false>), grid, block, 0, stream, p);
    else if (once) hipLaunchKernelGGL((kvq_attn_kernel<D, kBlocks, kRowWaves, kKeyWaves, false, kCut, kRows == 16>), grid, block, 0, stream, p);
    else hipLaunchKernelGGL((kvq_attn_kernel<D, kBlocks, kRowWaves, kKeyWaves, false, kCut, false>), grid, block, 0, stream, p);
    const hipError_t e = hipGetLastError();
    if (e != hipSuccess) return note_hip_error("launch kvq_attn_kernel", e);
    return kCut ? launch_prompt_merge(p, kRows, stream) : e;
}

template <int D>
hipError_t launch_rows(const KvqAttnParams &p, hipStream_t stream) {
    const int rows = kvq_attn_rows(p);
    switch (rows) {
        case 16: return launch<D, 1, 1, 4, true>(p, 2 * kNumCU, stream);
        case kFew16: return launch<D, 1, 1, 8, true>(p, kNumCU, stream);
        case kUncut16: return launch<D, 1, 1, 8, false>(p, 0, stream);
        case kUncut32: return launch<D, 2, 1, 8, false>(p, 0, stream);
        case kUncut64: return launch<D, 2, 2, 4, false>(p, 0, stream);
        default: return launch_kvq_attn_wide(p, rows, stream);
    }
}

}  // namespace

// Query rows of a kv head that a workgroup takes: the shortest of seven estimates, in us, of what the host knows (sequences of one
// length, max_seq_len with their last tokens).
//   16, 32, 64 rows, blocks that are not cut: a launch, and per block that a compute unit takes its ends and its wavefronts' steps of
//     32 keys; keys of a call that do not stay in the caches come from memory;
//   16 rows, keys cut into ranges: start and merge, steps that all compute units share out evenly, blocks' ends; 256 ranges of eight
//     wavefronts where no compute unit has a second block (a step's loads are out sooner, half the records), else 512 of four;
//   128, 256 rows, keys cut into ranges: the same, a range a workgroup; parts beyond four of a block cost the merge.
// The constants were fitted to 122 shapes (32 query and 8 kv heads of 128, 8 and 8 of 64; 1 to 64 sequences of one length, trees of 8 to
// 128 nodes, 1 to 1000 tokens, up to 12 K positions); other groups of heads and mixed batches go by the same estimates, unmeasured.  They pick
// the fastest on 109 of the 122 and are 0.7 % behind it on average, 12 % at most (16 prompts of 300 tokens, 64 trees of 128 nodes on 300
// positions).  Some of them, in us (all of them: profiles/kvq_rows_sweep.txt):
//                                              16  16 few  16 uncut  32 uncut  64 uncut    128    256
//   one token on 700 positions                 16.5    15.9       8.7      11.2      10.6   19.7   21.4
//   one token on 12 K positions                25.8    20.8      52.9      63.6      79.3   38.0   33.7
//   16 trees of 32 nodes on 1500               48.2    60.0      56.0      35.0      25.0   50.1   45.7
//   16 trees of 64 nodes on 6000                265     270       244       159       142    129    117
//   64 trees of 32 nodes on 6000                651     540       529       329       303    225    358
//   4 prompts of 1000 tokens                    244     337       219       157       117   93.5    101
// A bound that is loose is taken for the longest sequence.
int kvq_attn_rows(const KvqAttnParams &p) {
    const int forced = tuning(READER_TUNE_PROMPT_ROWS);
    // (blocks that are not cut are counted with the threads of a launch)
    const bool countable = (long long)p.N < (1 << 22);
    if (forced == 16 || forced == kFew16 || forced == 128 || forced == 256) return forced;
    if ((forced == kUncut16 || forced == kUncut32 || forced == kUncut64) && countable) return forced;
    const bool large = p.D == 128;
    const double tokens = p.nodes > 0 ? p.nodes : (double)p.N / p.B, longest = p.max_seq_len > tokens ? p.max_seq_len : tokens;
    const double longest_tiles = ceil(longest / kStep), tiles = (p.nodes > 0 ? longest : longest - 0.5 * tokens) / kStep + 0.5;
    auto blocks = [&](int rows) { return (double)p.Hkv * p.B * ceil(tokens / (rows / p.G)); };
    const double values = (double)p.B * p.Hkv * longest * p.D, from_memory = values > 1e8 ? 8.0 + values * (17.0 / 16.0) / 5.3e6 : 0.0;
    double best = 1e30;
    int rows = 16;
    auto offer = [&](int r, double us) {
        if (us < best) { best = us; rows = r; }
    };
    auto uncut = [&](int r, double ends, double step, int waves) {
        const double turns = ceil(blocks(r) / kNumCU), one = ends + step * ceil(longest_tiles / waves);
        const double each = ends + (turns > 1 ? (large ? 2.2 : 1.1) : 0.0) + step * (tiles > waves ? tiles / waves : 1.0);
        const double us = turns * each > one ? turns * each : one;
        return 2.5 + (us > from_memory ? us : from_memory);
    };
    if (countable) {
        offer(kUncut16, large ? uncut(16, 3.3, 1.0, 8) : uncut(16, 2.9, 0.73, 8));
        offer(kUncut32, large ? uncut(32, 4.1, 1.32, 8) : uncut(32, 3.2, 0.92, 8));
        offer(kUncut64, large ? uncut(64, 4.8, 1.29, 4) : uncut(64, 3.5, 0.95, 4));
    }
    auto parts = [&](int r, int ranges, int least) {      // of a block
        const double n = blocks(r) * tiles / least;
        return (n < ranges ? n : ranges) / blocks(r);
    };
    auto over = [](double n, double free) { return n > free ? n - free : 0.0; };
    const bool few = blocks(16) <= kNumCU;
    offer(few ? kFew16 : 16, (large ? (few ? 13.0 : 15.0) : (few ? 12.0 : 13.0)) + (large ? 0.195 : 0.095) * blocks(16) * tiles / kNumCU +
                                 0.15 * over(parts(16, few ? kNumCU : 2 * kNumCU, 8), 8) + (large ? 1.4 : 1.1) * blocks(16) / kNumCU);
    auto wide = [&](int r, int ranges, double start, double step, double ends) {
        const double steps = blocks(r) * tiles / ranges;
        return start + step * (steps > 4 ? steps : 4.0) + ends * blocks(r) / ranges + 0.3 * over(parts(r, ranges, 4), 4);
    };
    offer(128, large ? wide(128, 2 * kNumCU, 20, 1.25, 8) : wide(128, 2 * kNumCU, 16, 0.70, 8));
    offer(256, large ? wide(256, kNumCU, 22, 1.09, 9) : wide(256, kNumCU, 17, 0.84, 9));
    return rows;
}

size_t kvq_attn_workspace_bytes(int D) { return ranges_workspace_bytes(kNumCU, 256, D); }

hipError_t launch_kvq_attn(const KvqAttnParams &p, hipStream_t stream) {
    return p.D == 64 ? launch_rows<64>(p, stream) : launch_rows<128>(p, stream);
}

}  // namespace reader

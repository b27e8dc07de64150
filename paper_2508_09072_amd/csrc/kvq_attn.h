// What the kernels of the attention over the cache in 4 bits share (kvq_attn.hip, kvq_attn_wide.hip).
#pragma once

#include "kvq_common.h"
#include "prompt_rows.h"
#include "tree_attn_common.h"

namespace reader {

namespace {

constexpr float kMostSum = 0x1p16f;                  // of a lane's part of a row's sum, before its reference moves

// Two codes of byte `kByte` of a word, times 2^(scale - 127) in the exponent bits of `scale`: exact.
template <int kByte>
__device__ __forceinline__ uint32_t two_values(uint32_t word, float scale) {
    return __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(word, scale, kByte));
}
__device__ __forceinline__ float scale_of(uint32_t byte) { return __uint_as_float(byte << 23); }
// ... in byte e of a word.  (What else the word holds is in the sign and the mantissa: the instruction does not look at them.)
__device__ __forceinline__ float scale_in(uint32_t word, int e) { return __uint_as_float(e < 3 ? word << (23 - 8 * e) : word >> 1); }

// Which nodes every node of a draft tree sees: itself and its ancestors, a bit each.  By doubling the links, seven times for 128 nodes;
// a node whose link is wrong is a root.  All threads of the workgroup; barriers at both ends.
__device__ inline void ancestors(const int32_t *parents, int T, uint32_t (&s_mask)[READER_MAX_T][4], int (&s_up)[READER_MAX_T], int &bad) {
    int i = threadIdx.x;
    asm("" : "+v"(i));                                   // (nothing here is worth a register outside)
    uint32_t mine[4] = {};
    int up = i < T ? parents[i] : -1;
    __syncthreads();
    if (i < T) {
        if (i == 0 ? up != -1 : (up < 0 || up >= i)) { up = -1; bad |= READER_STATUS_BAD_TREE; }
        mine[i >> 5] = 1u << (i & 31);
    }
#pragma unroll 1
    for (int reach = 1;; reach *= 2) {                   // (nodes of a path that a mask holds, at most)
        if (i < T) {
#pragma unroll
            for (int w = 0; w < 4; ++w) s_mask[i][w] = mine[w];
            s_up[i] = up;
        }
        __syncthreads();
        if (reach >= T) break;
        if (up >= 0) {
#pragma unroll
            for (int w = 0; w < 4; ++w) mine[w] |= s_mask[up][w];
            up = s_up[up];
        }
        __syncthreads();
    }
}

// Where the log-sum-exp of token `tok` of a block goes that starts at packed row row0, and at node node0 of sequence b.
__device__ __forceinline__ size_t lse_at(const PromptParams &p, int b, int row0, int node0, int tok, int hq) {
    return p.nodes == 0 ? ((size_t)row0 + tok) * p.Hq + hq : ((size_t)b * p.Hq + hq) * p.nodes + node0 + tok;
}

// What is wrong with the lengths and bounds of all sequences (threads side by side).
template <bool kTree>
__device__ __forceinline__ int wrong_sequence(const KvqAttnParams &p, int b) {
    if constexpr (kTree) return p.seq_lens[b] < 0 || p.seq_lens[b] > p.max_seq_len - p.nodes ? READER_STATUS_BAD_LENGTH : 0;
    else return bad_sequence(p, b);
}
template <bool kTree>
__device__ __forceinline__ void report_sequences(const KvqAttnParams &p, int threads) {
    int bad = 0;
    for (int b = threadIdx.x; b < p.B; b += threads) bad |= wrong_sequence<kTree>(p, b);
    if (bad && p.status) atomicOr(p.status, bad);
}

// Largest of the lanes up to each, of values that are not negative.
template <int kControl, int kRows>
__device__ __forceinline__ int max_from(int v) { return max(v, __builtin_amdgcn_update_dpp(0, v, kControl, kRows, 0xf, kRows == 0xf)); }
__device__ __forceinline__ int max_scan(int v) {         // (scan64's steps)
    v = max_from<0x118, 0xf>(max_from<0x114, 0xf>(max_from<0x112, 0xf>(max_from<0x111, 0xf>(v))));
    return max_from<0x143, 0xc>(max_from<0x142, 0xa>(v));
}

// Block number `at` of a kv head, of all sequences' (o.head is set): false if there are not as many.  Rows that a sequence in front has
// too, where bounds go back, are that one's: the blocks are as many as N rows make, whatever the bounds are.  (Numbers that need no
// sums, cu[b] / tb + b and on, leave workgroups without a block between the others, and compute units with one more than their share: 64 tokens
// on 700 positions 26 instead of 19 us.)
template <bool kTree, class Block>
__device__ __forceinline__ bool find_block(const KvqAttnParams &p, const Sequences &seqs, int at, int lane, Block &o) {
    const int tb = p.tokens_per_block;
    if constexpr (kTree) {
        const int each = (p.nodes + tb - 1) / tb;
        o.b = at / each;
        o.k = at - o.b * each;
        if (o.b >= p.B) return false;
    } else {
        bool back = false;                               // a bound so far, and maybe the next, goes back
        for (int base = 0, before = 0, taken = 0;; base += 64) {
            if (base >= p.B) return false;
            const int b = base + lane;
            int from = 0, n = 0;
            if (b < p.B) {
                from = seqs.first(b);
                n = seqs.first(b + 1) - from;
            }
            back = back || __any(n < 0);
            if (back) {
                if (b > 0 && b < p.B && seqs.first(b - 1) < from) taken = max(taken, from);
                taken = max_scan(taken);                 // (the end of any sequence in front)
                n += from;
                from = max(from, taken);
                n = max(n - from, 0);
            }
            const int mine = (n + tb - 1) / tb, upto = before + (int)scan64(mine);
            const unsigned long long in = __ballot(at < upto);
            if (in) {
                const int i = (int)__builtin_ctzll(in);
                o.b = base + i;
                o.k = at - (__builtin_amdgcn_readlane(upto, i) - __builtin_amdgcn_readlane(mine, i));
                o.load(seqs);
                const int others = __builtin_amdgcn_readlane(from, i) - o.c0;
                o.c0 += others; o.L += others; o.n -= others;
                return true;
            }
            before = __builtin_amdgcn_readlane(upto, 63);
            // (in order, the last one's end is that of all who have tokens)
            const bool ends = __any(n > 0 && (!back || lane == 63));
            taken = max(__builtin_amdgcn_readlane(taken, 63), ends ? __builtin_amdgcn_readlane(from + n, 63) : 0);
        }
    }
    o.load(seqs);
    return true;
}

// This workgroup's range of the (head, sequence, block, key) axis, found by every wavefront for itself: false if there is none.  Its
// note is written, and what the first workgroup finds wrong with lengths and bounds.
template <class Block, int kMinRange, bool kTree>
__device__ __forceinline__ bool find_range(const KvqAttnParams &p, const Sequences &seqs, int lane, Block &place, int &t_place) {
    RangeNote *const notes = reinterpret_cast<RangeNote *>(p.workspace);
    const int tb = p.tokens_per_block;
    int bad = 0;
    auto cost_up_to = [&](int base) {                    // of sequences `base` .. base + lane
        const int b = base + lane;
        long long c = 0;
        if (b < p.B) {
            c = Block::sequence_cost(seqs.length(b), seqs.tokens(b), tb);
            bad |= wrong_sequence<kTree>(p, b);
        }
        return scan64(c);
    };
    const long long upto0 = cost_up_to(0);
    long long per_head = lane64(upto0, 63);
    for (int base = 64; base < p.B; base += 64) per_head += lane64(cost_up_to(base), 63);
    if (bad && blockIdx.x == 0 && p.status) atomicOr(p.status, bad);
    const long long total = per_head * p.Hkv;
    long long n_ranges = total / kMinRange;
    n_ranges = n_ranges > (long long)gridDim.x ? gridDim.x : (n_ranges < 1 ? 1 : n_ranges);
    const int range = blockIdx.x;
    if (range >= n_ranges || total == 0) {
        if (threadIdx.x == 0) notes[range] = RangeNote{};
        return false;
    }
    const PromptAxis axis(per_head, p.Hkv, (int)n_ranges);
    place = Block{p.Hkv, 0, 0, 0, 0, 0};
    t_place = 0;
    const long long at = axis.begin(range + (lane >> 5));
    long long r = 0, before = 0;
    if (at < total) place.head = axis.head(at, r);
#pragma unroll
    for (int half = 0; half < 2; ++half) {
        const long long r_half = lane64(r, 32 * half);
        long long carry = 0, upto = upto0;
        for (int base = 0;; base += 64) {
            if (base > 0) upto = cost_up_to(base);
            const long long all = carry + lane64(upto, 63);
            if (r_half < all) {                          // (the last of these 64 at the latest: r is below per_head)
                const int i = (int)__popcll(__ballot(carry + upto <= r_half));
                if (i > 0) carry += lane64(upto, i - 1);
                if ((lane >> 5) == half) place.b = base + i, before = carry;
                break;
            }
            carry = all;
        }
    }
    if (at < total) {
        place.load(seqs);
        t_place = place.locate(r - before, seqs, p.B, tb);
    } else place.b = 0;
    return true;
}

// Rows of a segment whose products have passed the largest number of 32 bits, though their mean does not: a lane's weights go up to
// kMostSum and are divided by their sum at the end, so that values from about 2^107 on can.  Such a row is gone through again over keys
// [j0, j1) by one wavefront as a running mean, which no value is larger than: 64 keys at a time, a lane each, then D / 64 columns a lane.
// Row numbers of the block, marked with `turn` in `odd`; the wavefronts share them out.  rec: where the block's part is left, record_rows wide,
// or null: the rows are written to `out`, behind what is written there already (a barrier in front).
template <int D, bool kTree, class Block>
__device__ __forceinline__ void rows_as_means(const KvqAttnParams &p, const Block &o, int rows, const int *odd, int turn, int wave, int waves, int j0, int j1,
                                              const uint32_t (*s_mask)[4], float *rec, int record_rows, int lane) {
    using B = KvqBlock<D>;
    constexpr int kPer = D / 64;
    asm("" : "+v"(lane));                                // (nothing here is worth a register outside)
    const int tb = p.tokens_per_block, d = lane * kPer;
    const int32_t *table = p.page_table + (size_t)o.b * p.max_pages;
#pragma unroll 1
    for (int row = wave; row < rows; row += waves) {
        if (odd[row] != turn) continue;
        const int tok = row / p.G, g = row - tok * p.G, node = o.k * tb + tok;
        const size_t at = ((size_t)(o.c0 + node)) * p.Hq + (size_t)o.head * p.G + g;
        const uint16_t *q = p.q + at * D;
        const int end = (int)min(min((long long)o.L + node + 1, (long long)p.max_seq_len), (long long)j1);
        float m = -INFINITY, l = 0.f, mean[kPer] = {};
#pragma unroll 1
        for (int base = j0; base < end; base += 64) {
            const int j = base + lane, n = j - o.L;
            const int id = j < end ? table[j / READER_PAGE_SIZE] : -1;
            bool sees = id >= 0 && id < p.num_pages;
            if constexpr (kTree) sees = sees && (n < 0 || (s_mask[node][(n >> 5) & 3] >> (n & 31) & 1u) != 0);
            const size_t block = ((size_t)(sees ? id : 0) * p.Hkv + o.head) * B::kBytes;
            const int s = j & (READER_PAGE_SIZE - 1);
            float x = -INFINITY;
            if (sees) {
                float dot = 0.f;
#pragma unroll 1
                for (int c = 0; c < D; c += 8) {
                    const uint32_t codes = *reinterpret_cast<const uint32_t *>(p.cache + block + B::k_code(s, c));
                    const float scale = scale_of(p.cache[block + B::k_scale(s, c / 32)]);
                    const u32x4 k = {two_values<0>(codes, scale), two_values<1>(codes, scale), two_values<2>(codes, scale), two_values<3>(codes, scale)}, w = ld16(q + c);
#pragma unroll
                    for (int i = 0; i < 4; ++i) {
                        dot += __uint_as_float(k[i] << 16) * __uint_as_float(w[i] << 16);
                        dot += __uint_as_float(k[i] & 0xffff0000u) * __uint_as_float(w[i] & 0xffff0000u);
                    }
                }
                x = dot * p.scale_log2;
            }
            float top = x;
#pragma unroll
            for (int off = 32; off >= 1; off >>= 1) top = fmaxf(top, __shfl_xor(top, off));
            top = fmaxf(top, m);
            const float keep = l == 0.f ? 0.f : l * __builtin_amdgcn_exp2f(m - top);
            const float w = sees && x > -INFINITY ? __builtin_amdgcn_exp2f(x - top) : 0.f;
            float sum = w;
#pragma unroll
            for (int off = 32; off >= 1; off >>= 1) sum += __shfl_xor(sum, off);
            if (sum == 0.f) continue;
            l = keep + sum;
            m = top;
#pragma unroll
            for (int e = 0; e < kPer; ++e) mean[e] *= keep / l;
            const float part = w / l;
            for (unsigned long long todo = __ballot(w > 0.f); todo; todo &= todo - 1) {
                const int k = (int)__builtin_ctzll(todo), ks = (base + k) & (READER_PAGE_SIZE - 1);
                const float wk = __shfl(part, k);
                const uint8_t *v_block = p.cache + __shfl((unsigned long long)block, k);
                const uint32_t v = two_values<0>(v_block[B::v_code(ks, d & ~1)], scale_of(v_block[B::v_scale(ks, d / 32)]));
                if constexpr (kPer == 2) {
                    mean[0] += wk * __uint_as_float(v << 16);
                    mean[1] += wk * __uint_as_float(v & 0xffff0000u);
                } else mean[0] += wk * __uint_as_float(d & 1 ? v & 0xffff0000u : v << 16);
            }
        }
#pragma unroll
        for (int e = 0; e < kPer; ++e) {
            if (rec) rec[((size_t)((d + e) / 4) * record_rows + row) * 4 + (d + e) % 4] = mean[e];
            else p.out[at * D + d + e] = (uint16_t)pack_bf16x2(mean[e], 0.f);
        }
        if (lane == 0) {
            if (rec) {
                rec[(size_t)record_rows * D + row] = m;
                rec[(size_t)record_rows * (D + 1) + row] = l;
            } else if (p.lse) p.lse[lse_at(p, o.b, o.c0 + o.k * tb, o.k * tb, tok, o.head * p.G + g)] = l == 0.f ? -INFINITY : (m + __builtin_amdgcn_logf(l)) * kLn2;
        }
    }
}

}  // namespace

}  // namespace reader

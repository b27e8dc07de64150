// The (head, sequence, block of query rows, key) axis of the prompts' attention, and what the ranges it is cut into leave for the
// launch that folds their parts together.
#pragma once

#include "prompt_common.h"

namespace reader {

namespace {

// What a range leaves for the launch behind it.
struct RangeNote {
    int tiles;            // 0: no record
    int ends;             // its first segment continues a block of an earlier range, and ends it
    int open;             // its last segment starts a block and does not end it: the block is
    int head, row0, nt;   // ... this one: kv head, first packed row, tokens
    int pad[2];
};
constexpr int kMaxRanges = kNumCU * 2;               // of any launch
constexpr size_t kNotesBytes = (size_t)kMaxRanges * sizeof(RangeNote);   // in front of the records, two a range
constexpr size_t ranges_workspace_bytes(int n_ranges, int record_rows, int D) {
    return kNotesBytes + (size_t)2 * n_ranges * record_rows * (D + 2) * sizeof(float);
}

// Sums of the lanes up to each.
template <int kControl, int kRows>
__device__ __forceinline__ long long add_from(long long v) {
    const int lo = __builtin_amdgcn_update_dpp(0, (int)v, kControl, kRows, 0xf, kRows == 0xf);
    const int hi = __builtin_amdgcn_update_dpp(0, (int)(v >> 32), kControl, kRows, 0xf, kRows == 0xf);
    return v + (((long long)hi << 32) | (unsigned)lo);
}
__device__ __forceinline__ long long scan64(long long v) {
    v = add_from<0x111, 0xf>(v);             // row_shr:1, 2, 4, 8
    v = add_from<0x112, 0xf>(v);
    v = add_from<0x114, 0xf>(v);
    v = add_from<0x118, 0xf>(v);
    v = add_from<0x142, 0xa>(v);             // row_bcast:15 into rows 1 and 3
    return add_from<0x143, 0xc>(v);          // row_bcast:31 into rows 2 and 3
}
__device__ __forceinline__ long long lane64(long long v, int lane) {
    return ((long long)__builtin_amdgcn_readlane((int)(v >> 32), lane) << 32) | (unsigned)__builtin_amdgcn_readlane((int)v, lane);
}

// Lengths and bounds of the sequences, from LDS or from memory.
struct Sequences {
    const int32_t *lens, *cu;
    int N, max_len;
    int nodes = 0;        // > 0: draft trees, each sequence has as many rows (cu is not read), behind which max_len leaves room for them
    // (rows behind the bound on the lengths see what lies in front of it)
    __device__ __forceinline__ int length(int b) const { return min(max(lens[b], 0), max_len - nodes); }
    __device__ __forceinline__ int first(int b) const { return nodes > 0 ? b * nodes : clamp_row(cu[b], N); }
    __device__ __forceinline__ int tokens(int b) const { return nodes > 0 ? nodes : max(clamp_row(cu[b + 1], N) - first(b), 0); }
};

// A block of query rows: `tb` tokens of a sequence (the last one of it: what is left) with all query heads of a kv head.  On the
// axis it takes as many positions as its last token sees keys, and kCost for what it costs beyond them: positions of a
// sequence's blocks add up to a closed form.
template <int kTileKeys, int kFront, int kCost>
struct PromptBlock {
    int head, b, k;       // kv head, sequence, number of the block there
    int L, n, c0;         // the sequence: cached positions, new tokens, first packed row
    __device__ __forceinline__ void load(const Sequences &s) { L = s.length(b); n = s.tokens(b); c0 = s.first(b); }
    __device__ __forceinline__ int tokens(int tb) const { return min(tb, n - k * tb); }
    // keys that the block's last token sees
    __device__ __forceinline__ int keys(int tb, int max_len) const {
        const long long end = (long long)L + k * tb + tokens(tb);
        return (int)(end < max_len ? end : max_len);
    }
    __device__ __forceinline__ int tiles(int tb, int max_len) const { return max(1, (keys(tb, max_len) + kTileKeys - 1) / kTileKeys); }
    __device__ __forceinline__ void next(const Sequences &s, int B, int tb) {
        if (++k * tb < n) return;
        k = 0;
        do {
            if (++b == B) { b = 0; ++head; }
        } while (s.tokens(b) == 0);          // (some sequence has tokens, or there would be no block)
        load(s);
    }
    // positions of the first k blocks of a sequence, none of them its last; of all of them
    __device__ static __forceinline__ long long blocks_cost(int L, int tb, long long k) { return k * ((long long)L + kCost) + tb * (k * (k + 1) / 2); }
    __device__ static __forceinline__ long long sequence_cost(int L, int n, int tb) {
        if (n <= 0) return 0;
        const long long nb = (n + tb - 1) / tb;
        return blocks_cost(L, tb, nb - 1) + (long long)L + kCost + n;
    }
    // The first tile at or behind position r of this sequence's part of the axis (head, b and what load() reads are set): its
    // block is set, its number returned.  Positions behind the block's tiles: the next block's first.
    __device__ __forceinline__ int locate(long long r, const Sequences &s, int B, int tb) {
        const int nb = (n + tb - 1) / tb;
        // k with blocks_cost(k) <= r < blocks_cost(k + 1): the root of a parabola, then a step either way for its rounding
        const double a = 0.5 * tb, q = (double)L + kCost + a;
        long long i = (long long)((sqrt(q * q + 4.0 * a * (double)r) - q) / (2.0 * a));
        i = i < 0 ? 0 : (i > nb - 1 ? nb - 1 : i);
        while (i > 0 && blocks_cost(L, tb, i) > r) --i;
        while (i < nb - 1 && blocks_cost(L, tb, i + 1) <= r) ++i;
        k = (int)i;
        const long long in = r - blocks_cost(L, tb, i) - kFront;
        const int all = tiles(tb, s.max_len);
        const int t = in <= 0 ? 0 : (int)((in + kTileKeys - 1) / kTileKeys < all ? (in + kTileKeys - 1) / kTileKeys : all);
        if (t < all) return t;
        next(s, B, tb);                      // (may step behind the last head: the end)
        return 0;
    }
    // the place that a lane has found, for all of them
    __device__ __forceinline__ PromptBlock of_lane(int lane) const {
        return PromptBlock{__builtin_amdgcn_readlane(head, lane), __builtin_amdgcn_readlane(b, lane), __builtin_amdgcn_readlane(k, lane),
                           __builtin_amdgcn_readlane(L, lane), __builtin_amdgcn_readlane(n, lane), __builtin_amdgcn_readlane(c0, lane)};
    }
};

// The axis: `per_head` positions for each of `heads` kv heads, cut into n ranges.
struct PromptAxis {
    long long per_head, total;
    double width, per_head_rcp;
    int n;
    __device__ __forceinline__ PromptAxis(long long head_positions, int heads, int n_ranges)
        : per_head(head_positions), total(head_positions * heads), width((double)total / n_ranges), per_head_rcp(1.0 / (double)per_head), n(n_ranges) {}
    // where range r begins (in floating point, which is as good as any other rule that all workgroups share: 64-bit division costs a
    // workgroup a microsecond)
    __device__ __forceinline__ long long begin(int r) const { return r >= n ? total : (long long)(r * width); }
    // kv head of position x, and the position within it
    __device__ __forceinline__ int head(long long x, long long &r) const {
        int h = (int)((double)x * per_head_rcp);
        r = x - h * per_head;
        while (r < 0) { --h; r += per_head; }
        while (r >= per_head) { ++h; r -= per_head; }
        return h;
    }
};

// A range: from tile t_lo of block `at` up to tile t_hi of block `stop`.
template <class Block>
struct PromptRange {
    Block at;
    int t_lo, t_hi, stop_head, stop_b, stop_k, heads;
    PromptRange() = default;
    // `o` and `t`: lanes 0..31 have found the first tile, the others the one behind the last.  (Side by side: a search costs as much
    // for one place as for two, a microsecond and a half.)
    __device__ __forceinline__ PromptRange(const Block &o, int t, int Hkv) : at(o.of_lane(0)), heads(Hkv) {
        t_lo = __builtin_amdgcn_readlane(t, 0); t_hi = __builtin_amdgcn_readlane(t, 32);
        stop_head = __builtin_amdgcn_readlane(o.head, 32); stop_b = __builtin_amdgcn_readlane(o.b, 32); stop_k = __builtin_amdgcn_readlane(o.k, 32);
    }
    __device__ __forceinline__ bool is_stop(const Block &o) const { return o.head == stop_head && (o.head == heads || (o.b == stop_b && o.k == stop_k)); }
    __device__ __forceinline__ bool behind(const Block &o) const { return o.head >= heads || (is_stop(o) && t_hi == 0); }
    // tiles of a block of the range that belong to it, [from, to)
    __device__ __forceinline__ void share(const Block &o, bool first, int tb, int max_len, int &from, int &to) const {
        from = first ? t_lo : 0;
        to = is_stop(o) ? t_hi : o.tiles(tb, max_len);
    }
    // its tiles, and what it leaves to the merge: blocks of a sequence 64 at a time, a lane each
    __device__ __forceinline__ RangeNote note(const Sequences &s, int B, int tb, int lane) const {
        RangeNote r = {};
        if (behind(at)) return r;
        const int from0 = t_lo, all0 = at.tiles(tb, s.max_len), to0 = is_stop(at) ? t_hi : all0;
        if (from0 > 0 && to0 > from0 && to0 == all0) r.ends = 1;
        int tiles = 0;
        Block o = at;
        for (bool first = true; !behind(o); first = false) {
            const bool here = o.head == stop_head && o.b == stop_b;         // (the range's last sequence)
            const int last = here ? stop_k : (o.n + tb - 1) / tb - 1;
            for (int k = o.k + lane; k <= last; k += 64) {
                Block c = o;
                c.k = k;
                const int from = first && k == o.k ? t_lo : 0, to = here && k == last ? t_hi : c.tiles(tb, s.max_len);
                tiles += max(to - from, 0);
            }
            const int begun = first && last == o.k ? t_lo : 0;              // of its last block there
            o.k = last;
            if (here) {
                if (begun == 0 && t_hi > 0 && t_hi < o.tiles(tb, s.max_len)) {
                    r.open = 1;
                    r.head = o.head; r.row0 = o.c0 + o.k * tb; r.nt = o.tokens(tb);
                }
                break;
            }
            o.next(s, B, tb);
        }
        r.tiles = (int)lane64(scan64(tiles), 63);
        return r;
    }
};

}  // namespace

}  // namespace reader

// Causal attention of packed prompts over the paged cache, on the matrix cores.
//
// Rows: a block is 256 query rows of one kv head, the `tb` = 256 / G tokens in a row of one sequence with all G heads of the
// group, so that a key tile that is in LDS serves them all and the causal edge costs one tile in L / 64.  A workgroup is 4
// wavefronts, one per SIMD, of 64 rows each (two blocks of 32): a K or V fragment read from LDS then feeds two matrix
// instructions, without which the LDS reads (32 KB a tile and wavefront) take as long as the matrix work; what 64 rows take of the
// register file needs the accumulation registers managed by hand (wide_registers.h).
// Work: blocks of one head are as long as their last token is far in, and lengths are known on the device only.  So the (head,
// sequence, block, key) axis is cut evenly into one range per compute unit, whatever the lengths; a block that is cut leaves
// partial records (fp32: outputs normalised by their own sum, reference, sum) that a second launch folds together.  Positions on
// the axis are keys, not tiles: blocks of one sequence then add up to a closed form, and nobody has to count them.
// Tiles travel HBM/L2 -> LDS through a ring of four, asked for three tiles ahead.  Tiles run as a software pipeline over two of
// them (see tile_pipelined): scores of the next tile, products of the current one and softmax weights alternate.
// Bound by power where prompts are long: 16384 tokens, 32 query and 8 kv heads of 128, 2.03 to 2.18 ms, 1.01 to 1.08 PFLOP/s, at 1.5
// GHz and 2750 cycles a tile, 2048 of them matrix work; heads of 64 2230, exponentials first.  Beyond its tiles a workgroup spends
// 7 to 10 us before the first one and 5 to 8 us a block (measured with a clock in a copy of this file: masked tile, first tile's maxima,
// outputs, query rows).
//
// Softmax weights are rounded to bf16 in front of the second product, which has no wider operand at this rate: scores, references
// and sums are fp32, but the output's error against 64 bits is 0.0020 to 0.0023 of its size where fp32 weights give 0.0016, the
// output's own rounding (dims.variant = 1).  Sums are of the weights before that rounding.
// A row's softmax reference is its maximum in the first tile of its range and is never moved: a lower reference makes all weights
// larger by one factor, which fp32 sums and bf16 weights hold up to 2^100.  Rows that this cannot hold, and rows with an output
// that is not a number (a masked value that is not one, times a weight of zero, is the other way to get there) are computed
// again, the plain way, by the wavefront that meets them.
#include <mutex>

#include "prompt_attn_scalar.h"
#include "prompt_ranges.h"
#include "wide_registers.h"

namespace reader {

namespace {

constexpr int kPromptThreads = 256, kPromptStages = 4, kPromptRows = 256;
constexpr int kPromptSlots = 256;                    // tiles of the list that are kept in LDS
constexpr int kPromptSeqsInLds = 2048;               // batches up to this size keep lengths and bounds in LDS
// What a block costs beyond its tiles, in keys (the query rows to fetch and the first tile's maxima in front, masks, normalising
// and writing behind), when the axis is cut.  (Six tiles instead of eight: the range with the first, short blocks of a head of 16384
// tokens took 13 % longer than the others, the whole call 4 %; ten: the same there, ragged prompts 3 % longer.)
constexpr int kBlockFront = 4 * kTile, kBlockCost = 8 * kTile;
constexpr int kMinRange = 4 * kTile;                 // no range is shorter than this: a range costs as much before its first tile
using Block = PromptBlock<kTile, kBlockFront, kBlockCost>;
constexpr int kMaxDevices = 64;                      // whose LDS limit is remembered

// One tile of a workgroup's list.
struct PromptTile {
    int blk[4];      // page * Hkv + kv head of each 16-key quarter, -1 where it reads as zeros
    int n_valid;     // keys of the tile that some row of the block sees (0..64)
    int flags;       // kTile*; from bit 8 up which quarters are missing
    int head, t;     // kv head, number of the tile
    int row0, p0, nt;   // the block: its first packed row, that token's position, its tokens
    int b;           // ... its sequence
};
enum {
    kTileFresh = 1,       // first tile of a segment (the part of a block inside the range)
    kTileEnds = 2,        // last tile of its segment
    kTileBlockStart = 4,  // first tile of its block
    kTileBlockEnd = 8,    // last tile of its block
    kTileMasked = 16,     // some row does not see some of its keys
    kTileHoles = 32,      // quarters behind a page id that does not exist
};

__host__ __device__ constexpr size_t prompt_record_floats(int D) { return (size_t)kPromptRows * (D + 2); }

}  // namespace

template <int D>
__global__ __launch_bounds__(kPromptThreads) void prompt_attn_kernel(PromptParams p, const int32_t *__restrict__ page_table) {
    constexpr int CW = 4;                            // every wavefront copies a quarter (16 rows) of each tile
    using G = Geometry<D, CW>;
    constexpr int kCopiesPerTile = 2 * G::kCopies;   // per wavefront
    constexpr int kS = kPromptStages;
    using Acc = AccMap<D>;
    static_assert(AccMap<128>::kEnd == 206 && AccMap<64>::kEnd == 106, "the register count below is the map's last register");
    if constexpr (D == 128) asm volatile("" ::: "a0", "a205");
    else asm volatile("" ::: "a0", "a105");

    extern __shared__ __attribute__((aligned(1024))) char smem[];
    char *ring = smem;                                                                   // [kS][kStageBytes]
    PromptTile *s_tile = reinterpret_cast<PromptTile *>(smem + kS * G::kStageBytes);     // [kPromptSlots]
    float *s_sink = reinterpret_cast<float *>(s_tile + kPromptSlots);                    // [64] landing zone of cache-warming copies
    int *s_seq = reinterpret_cast<int *>(s_sink + 64);                                   // lengths, then bounds
    const unsigned ring_lds = (unsigned)(size_t)(lds_char *)ring;
    const unsigned prefetch_lds = (unsigned)(size_t)(lds_char *)reinterpret_cast<char *>(s_sink);

    const int tid = threadIdx.x, lane = tid & 63;
    const int wave_s = __builtin_amdgcn_readfirstlane(tid >> 6);
    const int cw = wave_s, n = lane & 31, h = lane >> 5;
    const int tb = p.tokens_per_block;
    RangeNote *const notes = reinterpret_cast<RangeNote *>(p.workspace);
    int bad = 0;

    // ---- this workgroup's range of the axis
    // (costs of the sequences as prefix sums, in ring stages that are idle until the first copies)
    long long *s_pref = reinterpret_cast<long long *>(ring);                             // [B + 1]
    __shared__ long long s_wave[4];
    Sequences seqs{p.seq_lens, p.cu_tokens, p.N, p.max_seq_len};
    {
        const bool in_lds = p.B <= kPromptSeqsInLds;
        long long carry = 0;
        if (tid == 0) s_pref[0] = 0;
        for (int base = 0; base < p.B; base += kPromptThreads) {
            const int b = base + tid;
            long long c = 0;
            if (b < p.B) {
                const int len = p.seq_lens[b], lo = p.cu_tokens[b], hi = p.cu_tokens[b + 1];
                if (in_lds) {
                    s_seq[b] = len;
                    s_seq[p.B + b] = lo;
                    if (b == p.B - 1) s_seq[2 * p.B] = hi;
                }
                c = Block::sequence_cost(seqs.length(b), seqs.tokens(b), tb);
                bad |= bad_sequence(p, b);
            }
            c = scan64(c);
            if (lane == 63) s_wave[wave_s] = c;
            __syncthreads();
            long long before = carry;
            for (int w = 0; w < 4; ++w) {
                if (w < wave_s) before += s_wave[w];
                carry += s_wave[w];
            }
            if (b < p.B) s_pref[b + 1] = before + c;
            __syncthreads();
        }
        if (in_lds) { seqs.lens = s_seq; seqs.cu = s_seq + p.B; }
    }
    const long long per_head = s_pref[p.B], total = per_head * p.Hkv;
    long long n_ranges = total / kMinRange;
    n_ranges = n_ranges > (long long)gridDim.x ? gridDim.x : (n_ranges < 1 ? 1 : n_ranges);
    if (n_ranges >= kNumXCD) n_ranges -= n_ranges % kNumXCD;
    // ranges that follow one another (of one kv head, mostly) run on one XCD and share its L2
    const int range = n_ranges % kNumXCD == 0 ? (int)(blockIdx.x % kNumXCD * (n_ranges / kNumXCD) + blockIdx.x / kNumXCD) : (int)blockIdx.x;
    if (bad && blockIdx.x == 0 && p.status) atomicOr(p.status, bad);
    bad = 0;
    if ((int)blockIdx.x >= n_ranges || total == 0) {
        if (tid == 0) notes[blockIdx.x >= n_ranges ? blockIdx.x : range] = RangeNote{};
        return;
    }
    const PromptAxis axis(per_head, p.Hkv, (int)n_ranges);
    // first tile at or behind position x of the axis
    auto locate = [&](long long x, Block &o) {
        if (x >= total) {
            o = Block{p.Hkv, 0, 0, 0, 0, 0};
            return 0;
        }
        long long r;
        o.head = axis.head(x, r);
        int lo = 0, hi = p.B - 1;
        while (lo < hi) {                            // last sequence that starts at or in front of r
            const int mid = (lo + hi + 1) >> 1;
            if (s_pref[mid] <= r) lo = mid; else hi = mid - 1;
        }
        o.b = lo;
        o.load(seqs);
        return o.locate(r - s_pref[lo], seqs, p.B, tb);
    };
    Block place;
    const int t_place = locate(axis.begin(range + h), place);
    const PromptRange<Block> rg(place, t_place, p.Hkv);
    const RangeNote note = rg.note(seqs, p.B, tb, lane);
    if (tid == 0) notes[range] = note;
    const int n_iter = __builtin_amdgcn_readfirstlane(note.tiles);
    if (n_iter == 0) return;
    __syncthreads();                                 // (everybody is done with the prefix sums: the ring is free)

    // ---- this lane's two query rows: token within the block and head within the group, kept in accumulation registers
    static_for<2>([&](auto rc) {
        constexpr int r = decltype(rc)::value;
        const int row = wave_s * 64 + r * 32 + n;
        const int tok = (int)(((float)row + 0.5f) * p.g_rcp);         // row / G (half a row is far more than the product's rounding)
        acc_write<Acc::node(r)>((uint32_t)(row < tb * p.G ? tok : 0x3fffffff));   // (a row that no block uses: behind every token)
        acc_write<Acc::group(r)>((uint32_t)(row < tb * p.G ? row - tok * p.G : 0));
    });
    auto token_of = [](auto rc) { return (int)acc_read_u32<Acc::node(decltype(rc)::value)>(); };
    auto group_of = [](auto rc) { return (int)acc_read_u32<Acc::group(decltype(rc)::value)>(); };
    const int wave_token = wave_s * 64 < tb * p.G ? (int)(((float)(wave_s * 64) + 0.5f) * p.g_rcp) : 0x3fffffff;   // first token of this wavefront's rows

    // the segment that is being computed
    int seg_head = 0, seg_row0 = 0, seg_p0 = 0, seg_nt = 0, seg_t0 = 0;
    bool wave_active = false;
    auto q_row = [&](auto rc, int head, int row0, int nt) {
        const int tok = min(token_of(rc), nt - 1);                     // (rows behind the last token read its row)
        return p.q + (((size_t)row0 + tok) * p.Hq + (size_t)head * p.G + group_of(rc)) * D;
    };
    // The query rows as B operands of the first product: once per segment into the accumulation registers.
    struct QueryRows {
        u32x4 w[2][G::kKSteps];
    };
    auto fetch_q = [&](QueryRows &q, int head, int row0, int nt) {
        static_for<2>([&](auto rc) {
            constexpr int r = decltype(rc)::value;
            const uint16_t *src = q_row(rc, head, row0, nt);
#pragma unroll
            for (int kk = 0; kk < G::kKSteps; ++kk) q.w[r][kk] = ld16(src + kk * 16 + h * 8);
        });
    };
    auto put_q = [&](const QueryRows &q) {
        static_for<2>([&](auto rc) {
            constexpr int r = decltype(rc)::value;
            const bool real = token_of(rc) < seg_nt;
            static_for<G::kKSteps>([&](auto kc) {
                constexpr int kk = decltype(kc)::value;
                const u32x4 w = keep_if(real, q.w[r][kk]);
                acc_write<Acc::q(r, kk)>(w.x);
                acc_write<Acc::q(r, kk) + 1>(w.y);
                acc_write<Acc::q(r, kk) + 2>(w.z);
                acc_write<Acc::q(r, kk) + 3>(w.w);
            });
        });
        asm volatile("s_nop 3");
    };
    // (those of the first segment are on their way while the tile list is made: asked for behind the first tiles, they would be
    // waited for together with them)
    seg_head = rg.at.head; seg_row0 = rg.at.c0 + rg.at.k * tb; seg_nt = rg.at.tokens(tb);
    QueryRows first_q;
    fetch_q(first_q, seg_head, seg_row0, seg_nt);

    // ---- the tile list
    // Item i, found by walking the blocks from `walk`, whose first tile in the range is item walk_item; a thread each.
    Block walk = rg.at;
    int walk_item = 0;
    bool walk_first = true;
    auto write_item = [&](int i) {
        Block o = walk;
        bool first = walk_first;
        int from, to, item = walk_item;
        for (;;) {
            rg.share(o, first, tb, p.max_seq_len, from, to);
            if (i < item + (to - from)) break;
            item += to - from;
            first = false;
            o.next(seqs, p.B, tb);
        }
        const int t = from + (i - item), tiles = o.tiles(tb, p.max_seq_len), keys = o.keys(tb, p.max_seq_len);
        PromptTile *slot = s_tile + (i & (kPromptSlots - 1));
        const int n_valid = max(0, min(kTile, keys - t * kTile));
        int flags = (t == from ? kTileFresh : 0) | (t + 1 == to ? kTileEnds : 0) | (t == 0 ? kTileBlockStart : 0) | (t + 1 == tiles ? kTileBlockEnd : 0);
        const long long p0 = (long long)o.L + o.k * tb;
        if ((long long)(t + 1) * kTile > min(p0 + 1, (long long)p.max_seq_len)) flags |= kTileMasked;
        const int32_t *row = page_table + (size_t)o.b * p.max_pages + t * 4;
        int page[4];
#pragma unroll
        for (int j = 0; j < 4; ++j) page[j] = j * 16 < n_valid ? row[j] : 0;     // (position < keys <= 16 max_pages)
#pragma unroll
        for (int j = 0; j < 4; ++j) asm volatile("" : "+v"(page[j]));
#pragma unroll
        for (int j = 0; j < 4; ++j) {
            slot->blk[j] = -1;
            if (j * 16 >= n_valid) continue;
            if (page[j] >= 0 && page[j] < p.num_pages) slot->blk[j] = page[j] * p.Hkv + o.head;
            else { bad |= READER_STATUS_BAD_PAGE; flags |= kTileHoles | (1 << (8 + j)); }
        }
        slot->n_valid = n_valid; slot->flags = flags; slot->head = o.head; slot->t = t;
        slot->row0 = o.c0 + o.k * tb; slot->p0 = (int)min(p0, 0x7fffffffLL); slot->nt = o.tokens(tb); slot->b = o.b;
    };
    for (int i = tid; i < min(n_iter, kPromptSlots); i += kPromptThreads) write_item(i);
    // the next half of the list is written when half of it has been used; the walk then starts at the first item of that half
    auto move_walk = [&](int item) {
        for (;;) {
            int from, to;
            rg.share(walk, walk_first, tb, p.max_seq_len, from, to);
            if (item < walk_item + (to - from)) break;
            walk_item += to - from;
            walk_first = false;
            walk.next(seqs, p.B, tb);
            walk = walk.of_lane(0);
        }
    };
    __syncthreads();   // the list is written
    put_q(first_q);

    auto desc_of = [&](int i) -> const PromptTile * { return s_tile + (i & (kPromptSlots - 1)); };
    auto word = [](int v) { return __builtin_amdgcn_readfirstlane(v); };

    // touch the next segment's query rows one tile before they are needed
    auto prefetch_q = [&](int head, int row0, int nt) {
        static_for<2>([&](auto rc) {
            const uint16_t *src = q_row(rc, head, row0, nt) + (h * 64) % D;
            const unsigned dst = prefetch_lds;
            asm volatile("s_mov_b32 m0, %1\n\tglobal_load_lds_dword %0, off" :: "v"(src), "s"(dst) : "memory", "m0");
        });
    };

    // Byte offsets of this lane's part of the copies of a whole tile.
    const int rin = lane / G::kChunks, pchunk = lane % G::kChunks;
    static_for<G::kCopies>([&](auto ic) {
        constexpr int i = decltype(ic)::value;
        const int r = cw * G::kRowsPerWave + i * G::kRowsPerCopy + rin;
        acc_write<Acc::k_off(i)>((r & 15) * G::kRowBytes + ((unsigned)(pchunk ^ swizzle_k<D>(r)) << 4));
        acc_write<Acc::v_off(i)>((r & 15) * G::kRowBytes + ((unsigned)(pchunk ^ swizzle_v<D>(r)) << 4));
    });
    // Copies of this wavefront's 16 rows of a tile: exactly kCopiesPerTile copy instructions, whatever the tile looks like.  Rows
    // that nobody sees are copied from a block of zeros, so that a weight of zero times them stays zero.
    auto issue_tile = [&](int blk, int nv, unsigned stage_lds) {
        const bool page_ok = blk >= 0, whole = page_ok && (cw + 1) * G::kRowsPerWave <= nv;
        const size_t boff = (size_t)(page_ok ? blk : 0) * (16 * G::kRowBytes);
        const char *kb = reinterpret_cast<const char *>(p.k_cache) + boff, *vb = reinterpret_cast<const char *>(p.v_cache) + boff;
        const char *zeros = reinterpret_cast<const char *>(kZeroRow) + (lane & 15) * 16;
        static_for<kCopiesPerTile>([&](auto jc) {
            constexpr int j = decltype(jc)::value;
            constexpr bool is_v = j >= G::kCopies;
            constexpr int i = is_v ? j - G::kCopies : j;
            const unsigned dst = stage_lds + (is_v ? G::kTileBytes : 0) + cw * G::kRowsPerWave * G::kRowBytes + i * 1024;
            const unsigned off = acc_read_u32<is_v ? Acc::v_off(i) : Acc::k_off(i)>();
            if (whole) {
                copy16_uniform(is_v ? vb : kb, off, dst);
            } else {
                const bool ok = page_ok && cw * G::kRowsPerWave + i * G::kRowsPerCopy + rin < nv;
                copy16_lane(ok ? (is_v ? vb : kb) + off : zeros, dst);
            }
        });
    };
    auto issue_tile_at = [&](int i) {
        const PromptTile *d = desc_of(i);
        issue_tile(word(d->blk[cw]), word(d->n_valid), ring_lds + ((unsigned)i % kS) * G::kStageBytes);
    };
#pragma unroll
    for (int i = 0; i < kS - 1; ++i)
        if (i < n_iter) issue_tile_at(i);

    // per-lane LDS offsets of the operand reads (relative to the stage)
    int k_rd[G::kKSteps];   // K fragment of k-step kk, key block 0
#pragma unroll
    for (int kk = 0; kk < G::kKSteps; ++kk)
        k_rd[kk] = n * G::kRowBytes + (((2 * kk + h) ^ swizzle_k<D>(n)) << 4);
    int v_rd[G::kOBlocks];  // V fragment of output block db, keys 0..3 (+4h) of the first 16-key group
    {
        const int i16 = lane & 15, g16 = (lane >> 4) & 1;
        const int key_lo = 4 * h + (i16 >> 2);
        const int c_lo = 2 * g16 + ((i16 & 3) >> 1);
#pragma unroll
        for (int db = 0; db < G::kOBlocks; ++db)
            v_rd[db] = G::kTileBytes + key_lo * G::kRowBytes + ((((db * 4) | c_lo) ^ swizzle_v<D>(key_lo)) << 4) + (i16 & 1) * 8;
    }

    float mc[2] = {0.f, 0.f};                      // the rows' softmax references in the exp2 domain
    float lsum[2][2] = {{0.f, 0.f}, {0.f, 0.f}};   // per row block two partial sums of the segment's weights
    const float c2 = p.scale_log2;
    constexpr float kTooLarge = 0x1p100f;
    u32x4 pk[2][2][2];                    // [key block][row block][16-key step]: softmax weights as bf16 pairs, the B operands of the second product
    f32x16 s[2][2];                       // [key block][row block]: S^T of the current tile

    auto k_frag = [&](const char *stage, int kb, int kk) {
        return *reinterpret_cast<const bf16x8 *>(stage + k_rd[kk] + kb * 32 * G::kRowBytes);
    };
    // half `hf` of the V^T fragment of (16-key step ks, output block db): keys +0..3 (+4h) or +8..11 (+4h)
    auto v_half = [&](const char *stage, int ks, int db, int hf) {
        const int key_base = ((ks >> 1) * 32 + (ks & 1) * 16 + hf * 8) * G::kRowBytes;
        return lds_read_tr16(stage + v_rd[db] + key_base);
    };
    auto p_frag = [&](int kb, int r, int m2) { return __builtin_bit_cast(bf16x8, pk[kb][r][m2]); };
    // weights of scores i, i + 1 of block (kb, r) against the row's reference
    auto weight_pair = [&](int kb, int r, int i) {
        const float p0 = __builtin_amdgcn_exp2f(s[kb][r][i] * c2 - mc[r]);
        const float p1 = __builtin_amdgcn_exp2f(s[kb][r][i + 1] * c2 - mc[r]);
        lsum[r][0] += p0;
        lsum[r][1] += p1;
        pk[kb][r][i >> 3][(i >> 1) & 3] = pack_bf16x2(p0, p1);
    };
    // Which keys of a tile row block r sees: a bit for each (word 0 and 1: key blocks 0 and 1), the lane's 4 h taken off.
    // Score i of a key block has bit key_bit(i); a bit is spread over a register to choose between the score and minus infinity,
    // two instructions and no scalar register, of which comparisons would take two each.
    struct Sees { uint32_t w[2][2]; };   // [key block][row block]
    auto key_bit = [](int i) { return (i >> 2) * 8 + (i & 3); };
    auto sees_of = [&](int n_valid, int t) {
        Sees o;
        static_for<2>([&](auto rc) {
            constexpr int r = decltype(rc)::value;
            const int tok = token_of(rc), lim = (tok < seg_nt ? min(n_valid, seg_p0 + tok + 1 - t * kTile) : 0) - 4 * h;
#pragma unroll
            for (int kb = 0; kb < 2; ++kb) {
                const int n = min(max(lim - kb * 32, 0), 32);
                o.w[kb][r] = n == 32 ? ~0u : (1u << n) - 1u;
                asm volatile("" : "+v"(o.w[kb][r]));
            }
        });
        return o;
    };
    auto seen = [](uint32_t word, int bit, float x) {
        const uint32_t m = (uint32_t)__builtin_amdgcn_sbfe((int)word, bit, 1);
        return __uint_as_float((m & __float_as_uint(x)) | (~m & 0xff800000u));
    };
    auto mask = [&](int kb, const Sees &o) {
#pragma unroll
        for (int r = 0; r < 2; ++r)
#pragma unroll
            for (int i = 0; i < 16; ++i) s[kb][r][i] = seen(o.w[kb][r], key_bit(i), s[kb][r][i]);
    };
    // The weights of pipelined tiles are a pipeline of their own, one per matrix instruction: slot e takes the exponential of
    // the argument made in slot e - 1, makes the argument of weight e + 1, adds weight e - 1 to its row's sum and, when e is even,
    // packs weights e - 2 and e - 1, so that no instruction of a slot waits for another of it.  All of it is written out, so
    // that it stays in the slot it is written in and gets no wait states of the compiler's.
    float w_x = 0.f;                // argument of the exponential of the slot's own weight
    float w_p1 = 0.f, w_p2 = 0.f;   // the weights of one and two slots ago
    auto weight_arg = [&](float score, float ref) {
        float x;
        asm volatile("v_fma_f32 %0, %1, %2, -%3" : "=v"(x) : "v"(score), "v"(c2), "v"(ref));
        return x;
    };
    // masked: o[0] and o[1] say what of the current and of the next tile is seen
    auto weight_slot = [&](auto wkbc, auto ec, auto masked, const Sees (&o)[2]) {
        constexpr int wkb = decltype(wkbc)::value, e = decltype(ec)::value;
        float p_cur;
        asm volatile("v_exp_f32 %0, %1" : "=v"(p_cur) : "v"(w_x));
        constexpr int nb = e == 31 ? 1 - wkb : wkb, ne = (e + 1) & 31;
        w_x = weight_arg(s[nb][ne / 16][ne % 16], mc[ne / 16]);
        if constexpr (decltype(masked)::value) w_x = seen(o[wkb == 1 && e < 31 ? 0 : 1].w[nb][ne / 16], key_bit(ne % 16), w_x);
        constexpr int pe = (e + 31) & 31;
        asm volatile("v_add_f32 %0, %0, %1" : "+v"(lsum[pe / 16][pe & 1]) : "v"(w_p1));
        if constexpr ((e & 1) == 0) {
            constexpr int pb = e == 0 ? 1 - wkb : wkb, p2 = (e + 30) & 31, r = p2 / 16, i = p2 % 16;
            uint32_t both;
            asm volatile("v_cvt_pk_bf16_f32 %0, %1, %2" : "=v"(both) : "v"(w_p2), "v"(w_p1));
            pk[pb][r][i >> 3][(i >> 1) & 3] = both;
        }
        w_p2 = w_p1;
        w_p1 = p_cur;
    };

    // Slots e (even) and e + 1 in one piece, for tiles with two weights a matrix instruction (in pieces the compiler puts a wait state
    // between some of them: 16384 tokens with heads of 64 1392 -> 1349 us)
    auto weight_slots = [&](auto wkbc, auto ec) {
        constexpr int wkb = decltype(wkbc)::value, e = decltype(ec)::value;
        static_assert((e & 1) == 0, "a pair starts at an even slot");
        constexpr int nb = e + 1 == 31 ? 1 - wkb : wkb, ne = (e + 2) & 31;      // the argument of weight e + 2
        constexpr int pe = (e + 31) & 31, pb = e == 0 ? 1 - wkb : wkb, p2 = (e + 30) & 31, r = p2 / 16, i = p2 % 16;
        float p0, p1, x1, x2;
        uint32_t both;
        asm volatile("v_exp_f32 %0, %7\n\tv_fma_f32 %2, %8, %12, -%13\n\tv_add_f32 %5, %5, %10\n\tv_cvt_pk_bf16_f32 %4, %11, %10\n\t"
                     "v_exp_f32 %1, %2\n\tv_fma_f32 %3, %9, %12, -%14\n\tv_add_f32 %6, %6, %0"
                     : "=&v"(p0), "=&v"(p1), "=&v"(x1), "=&v"(x2), "=&v"(both), "+v"(lsum[pe / 16][pe & 1]), "+v"(lsum[e / 16][e & 1])
                     : "v"(w_x), "v"(s[wkb][(e + 1) / 16][(e + 1) % 16]), "v"(s[nb][ne / 16][ne % 16]), "v"(w_p1), "v"(w_p2), "v"(c2),
                       "v"(mc[(e + 1) / 16]), "v"(mc[ne / 16]));
        pk[pb][r][i >> 3][(i >> 1) & 3] = both;
        w_x = x2;
        w_p2 = p0;
        w_p1 = p1;
    };

    // S = K.Q^T of a tile
    auto scores = [&](const char *stage) {
        constexpr int kK = G::kKSteps;
        bf16x8 kf[3][2];
        kf[0][0] = k_frag(stage, 0, 0); kf[0][1] = k_frag(stage, 1, 0);
        kf[1][0] = k_frag(stage, 0, 1); kf[1][1] = k_frag(stage, 1, 1);
        static_for<kK>([&](auto kc) {
            constexpr int kk = decltype(kc)::value;
            if constexpr (kk + 2 < kK) { kf[(kk + 2) % 3][0] = k_frag(stage, 0, kk + 2); kf[(kk + 2) % 3][1] = k_frag(stage, 1, kk + 2); }
            static_for<4>([&](auto gc) {
                constexpr int kb = decltype(gc)::value >> 1, r = decltype(gc)::value & 1;
                if constexpr (kk == 0) mfma_s0<Acc::q(r, kk)>(s[kb][r], kf[kk % 3][kb]);
                else mfma_s<Acc::q(r, kk)>(s[kb][r], kf[kk % 3][kb]);
            });
        });
        READER_RESULT_WAIT();
    };
    // O^T += V^T.P^T of a tile whose weights are in pk: a V fragment serves both row blocks
    auto products = [&](const char *stage) {
        constexpr int kOB = G::kOBlocks;
        s16x4 vf[2][kOB][2];
#pragma unroll
        for (int db = 0; db < kOB; ++db) { vf[0][db][0] = v_half(stage, 0, db, 0); vf[0][db][1] = v_half(stage, 0, db, 1); }
        static_for<4>([&](auto kc) {
            constexpr int ks = decltype(kc)::value;
            if constexpr (ks + 1 < 4) {
#pragma unroll
                for (int db = 0; db < kOB; ++db) {
                    vf[(ks + 1) & 1][db][0] = v_half(stage, ks + 1, db, 0);
                    vf[(ks + 1) & 1][db][1] = v_half(stage, ks + 1, db, 1);
                }
            }
            static_for<2 * kOB>([&](auto jc) {
                constexpr int r = decltype(jc)::value / kOB, db = decltype(jc)::value % kOB;
                const s16x8 a8 = __builtin_shufflevector(vf[ks & 1][db][0], vf[ks & 1][db][1], 0, 1, 2, 3, 4, 5, 6, 7);
                mfma_o<Acc::o(r, db)>(__builtin_bit_cast(bf16x8, a8), p_frag(ks >> 1, r, ks & 1));
            });
        });
    };
    auto weights_of_key_block = [&](int kb) {
#pragma unroll
        for (int r = 0; r < 2; ++r)
#pragma unroll
            for (int i = 0; i < 16; i += 2) weight_pair(kb, r, i);
        asm volatile("s_nop 3");   // (weights written by the vector ALU are matrix operands next)
    };
    // Start of a run of whole tiles: the weights of key block 0, left the way slot 31 of a pipelined tile leaves them
    auto begin_run = [&]() {
#pragma unroll
        for (int r = 0; r < 2; ++r)
#pragma unroll
            for (int i = 0; i < (r == 0 ? 16 : 14); i += 2) weight_pair(0, r, i);
        w_p2 = __builtin_amdgcn_exp2f(s[0][1][14] * c2 - mc[1]);
        w_p1 = __builtin_amdgcn_exp2f(s[0][1][15] * c2 - mc[1]);
        lsum[1][0] += w_p2;
        w_x = weight_arg(s[1][0][0], mc[0]);
    };
    // End of a run: what slot 0 of a further pipelined tile would have done with key block 0
    auto end_run = [&]() {
        lsum[1][1] += w_p1;
        pk[0][1][1][3] = pack_bf16x2(w_p2, w_p1);
    };

    // One pipelined tile: products and key-block-1 weights of the tile in `stage`, scores and key-block-0 weights of the next
    // one in `next_stage`, in two half steps, one per block of 32 keys; half step kb of tile t holds, interleaved,
    //   S(t+1, kb) = K.Q^T          into the score registers of key block kb, whose weights were taken in the half step before;
    //   O += V(t, kb)^T.P(t, kb)^T  with the weights made in the half step before;
    //   weights of the other key block: of (t, 1) in half step 0, of (t+1, 0) in half step 1, one score per matrix instruction.
    // Operand fragments are read from LDS two groups of four matrix instructions ahead.  with_copy: the copies of a whole tile
    // (base addresses kbase / vbase, LDS address copy_stage_lds) are issued on the way, spread over the tile.  masked: rows do not see
    // some keys of the tile or of the next one.  (tree_attn_wide.hip runs its tiles in the same order, without masks: what is mended
    // in one belongs into the other.)
    auto tile_pipelined = [&](auto with_copy, auto masked, const Sees (&sees)[2], const char *stage, const char *next_stage, const char *kbase, const char *vbase,
                              unsigned copy_stage_lds) {
        constexpr int kK = G::kKSteps, kOB = G::kOBlocks;
        static_assert(kK == 2 * kOB, "a half step has as many score as product instructions");
        bf16x8 kf[3];
        s16x4 vf[3][2];
        auto load_part = [&](auto kbc, auto gc, auto part) {
            constexpr int kb = decltype(kbc)::value, g = decltype(gc)::value, w3 = (kb * kK + g) % 3;
            if constexpr (decltype(part)::value == 0) kf[w3] = k_frag(next_stage, kb, g);
            else vf[w3][decltype(part)::value - 1] = v_half(stage, 2 * kb + g / kOB, g % kOB, decltype(part)::value - 1);
        };
        static_for<3>([&](auto part) {
            load_part(std::integral_constant<int, 0>{}, std::integral_constant<int, 0>{}, part);
            load_part(std::integral_constant<int, 0>{}, std::integral_constant<int, 1>{}, part);
        });
        __builtin_amdgcn_sched_barrier(0);
        static_for<2 * kK>([&](auto gg) {
            constexpr int kb = decltype(gg)::value / kK, g = decltype(gg)::value % kK;
            static_for<4>([&](auto mc4) {
                constexpr int m = decltype(mc4)::value, j = g * 4 + m;      // slot j of 4 kK in this half step
                // Half step 0: P S P S (the first K fragment is the last to arrive); half step 1: S S P P.  Either way at
                // least two matrix instructions stand between the last score instruction of row block 0 and the first read of
                // those scores by the vector ALU, in the last slot of the half step.
                constexpr bool is_p = kb == 0 ? (m & 1) == 0 : m >= 2;
                constexpr int r = kb == 0 ? m >> 1 : m & 1;
                constexpr int w3 = (kb * kK + g) % 3;
                if constexpr (is_p) {
                    const s16x8 a8 = __builtin_shufflevector(vf[w3][0], vf[w3][1], 0, 1, 2, 3, 4, 5, 6, 7);
                    mfma_o<Acc::o(r, g % kOB)>(__builtin_bit_cast(bf16x8, a8), p_frag(kb, r, g / kOB));
                } else {
                    if constexpr (g == 0) mfma_s0<Acc::q(r, g)>(s[kb][r], kf[w3]);
                    else mfma_s<Acc::q(r, g)>(s[kb][r], kf[w3]);
                }
                if constexpr (m < 3) {
                    if constexpr (g + 2 < kK) load_part(std::integral_constant<int, kb>{}, std::integral_constant<int, g + 2>{}, mc4);
                    else if constexpr (kb == 0) load_part(std::integral_constant<int, 1>{}, std::integral_constant<int, g + 2 - kK>{}, mc4);
                }
                if constexpr (decltype(with_copy)::value) {
                    constexpr int J = kb * 4 * kK + j, kSpacing = 8 * kK / kCopiesPerTile;
                    if constexpr (J % kSpacing == 1) {
                        constexpr int c = J / kSpacing;
                        constexpr bool is_v = c >= G::kCopies;
                        constexpr int i = is_v ? c - G::kCopies : c;
                        copy16_uniform(is_v ? vbase : kbase, acc_read_u32<is_v ? Acc::v_off(i) : Acc::k_off(i)>(),
                                       copy_stage_lds + (is_v ? G::kTileBytes : 0) + cw * G::kRowsPerWave * G::kRowBytes + i * 1024);
                    }
                }
                // weights of the other key block (of the next tile in half step 1), 32 scores over 4 kK slots
                constexpr int lo = j * 32 / (4 * kK), hi = (j + 1) * 32 / (4 * kK);
                if constexpr (hi - lo == 2 && !decltype(masked)::value) weight_slots(std::integral_constant<int, 1 - kb>{}, std::integral_constant<int, lo>{});
                else static_for<hi - lo>([&](auto ic) { weight_slot(std::integral_constant<int, 1 - kb>{}, std::integral_constant<int, lo + decltype(ic)::value>{}, masked, sees); });
                __builtin_amdgcn_sched_barrier(0);
            });
        });
    };

    // The reference of row block r: the maximum of the scores in the registers, or kNoReference.  (A row that sees no key of the
    // segment's first tile sees none of a later one either, by its place; behind pages that do not exist, or keys that score minus
    // infinity, it may: its weights then are too large for the reference, and it is computed again.)
    constexpr float kNoReference = -1e30f;
    auto set_reference = [&](auto rc) {
        constexpr int r = decltype(rc)::value;
        float mx = fmaxf(s[0][r][0], s[1][r][0]);
#pragma unroll
        for (int i = 1; i < 16; ++i) mx = fmaxf(fmaxf(mx, s[0][r][i]), s[1][r][i]);
        // the other half of the row's keys sits in lane ^ 32
        const auto sw = __builtin_amdgcn_permlane32_swap(__float_as_uint(mx), __float_as_uint(mx), false, false);
        mx = fmaxf(__uint_as_float(sw[0]), __uint_as_float(sw[1]));
        const float ref = fmaxf(mx, kNoReference);
        acc_write<Acc::m_ref(r)>(__float_as_uint(ref));
        mc[r] = ref * c2;
    };

    // A tile with keys behind page ids that do not exist, one step after the other.
    auto tile_plain = [&](const char *stage, int flags, int n_valid, int t) {
        const int holes = (flags >> 8) & 15;
        scores(stage);
        const Sees o = sees_of(n_valid, t);
        mask(0, o);
        mask(1, o);
#pragma unroll
        for (int kb = 0; kb < 2; ++kb)
#pragma unroll
            for (int r = 0; r < 2; ++r)
#pragma unroll
                for (int i = 0; i < 16; ++i) s[kb][r][i] = (holes >> (kb * 2 + (i >> 3))) & 1 ? -INFINITY : s[kb][r][i];
        if (flags & kTileFresh) static_for<2>([&](auto rc) { set_reference(rc); });
        weights_of_key_block(0);
        weights_of_key_block(1);
        products(stage);
    };

    auto reset_state = [&]() {
#pragma unroll
        for (int r = 0; r < 2; ++r) {
            mc[r] = 0.f;
            lsum[r][0] = lsum[r][1] = 0.f;
        }
        acc_write<Acc::m_ref(0)>(__float_as_uint(-INFINITY));
        acc_write<Acc::m_ref(1)>(__float_as_uint(-INFINITY));
        static_for<2 * G::kOBlocks * 16>([&](auto ic) { acc_zero<decltype(ic)::value>(); });   // the output accumulators
    };

    // End of a segment: a block seen from its first to its last tile is normalised and written out, anything else leaves a
    // partial record.
    auto finish_segment = [&](int flags, int t_end, int table_b) {
        READER_RESULT_WAIT();   // the last products of the segment are about to be read by the vector ALU
        const bool whole = seg_t0 == 0 && (flags & kTileBlockEnd);
        float *rec = reinterpret_cast<float *>(reinterpret_cast<char *>(p.workspace) + kNotesBytes) +
                     (size_t)(2 * range + (seg_t0 == 0 ? 1 : 0)) * prompt_record_floats(D);
        bool again = false;
        static_for<2>([&](auto rc) {
            constexpr int r = decltype(rc)::value;
            const int row = wave_s * 64 + r * 32 + n, tok = token_of(rc);
            const bool real = tok < seg_nt;
            const float l_mine = lsum[r][0] + lsum[r][1];
            const auto both = __builtin_amdgcn_permlane32_swap(__float_as_uint(l_mine), __float_as_uint(l_mine), false, false);
            const float l = __uint_as_float(both[0]) + __uint_as_float(both[1]);
            const float inv = l == 0.f ? 0.f : __builtin_amdgcn_rcpf(l);    // (a row may see no key of a part; off by 2^-23 at most)
            const float ref = __uint_as_float(acc_read_u32<Acc::m_ref(r)>()) * c2;
            float check[4] = {l < kTooLarge ? 0.f : __builtin_nanf(""), 0.f, 0.f, 0.f};
            // values 4 i4 + 4 h .. + 3 and + 8 of them of block db: a lane holds, of two 8-wide chunks of the output row side by side,
            // 4 values of each, its partner lane (lane ^ 32) the others
            auto values = [&](auto dbc, auto i4c, float (&v)[8]) {
                static_for<8>([&](auto ec) {
                    constexpr int e = decltype(ec)::value;
                    v[e] = acc_read<Acc::o(r, decltype(dbc)::value) + 4 * decltype(i4c)::value + e>() * inv;
                    check[e % 4] = __builtin_fmaf(v[e], 0.f, check[e % 4]);   // (not a number once any value is none)
                });
            };
            if (whole) {
                // Four chunks of rows 0..15 and of 16..31 of the block change places, so that a store writes 64 bytes of a row in one go
                // (packed prompts with heads of 64 212 -> 207 us, more than to have the next query rows on their way meanwhile).
                auto place = [&](int at, bool &is) {
                    const int t = (int)(((float)at + 0.5f) * p.g_rcp);
                    is = at < tb * p.G && t < seg_nt;
                    return p.out + (((size_t)seg_row0 + t) * p.Hq + (size_t)seg_head * p.G + (at - t * p.G)) * D + (((lane >> 4) & 1) * 2 + h) * 8;
                };
                bool real_lo, real_hi;
                uint16_t *const to_lo = place(wave_s * 64 + r * 32 + (lane & 15), real_lo), *const to_hi = place(wave_s * 64 + r * 32 + 16 + (lane & 15), real_hi);
                static_for<G::kOBlocks>([&](auto dbc) {
                    constexpr int db = decltype(dbc)::value;
                    uint32_t w[2][4];
                    static_for<2>([&](auto ic) {
                        constexpr int i = decltype(ic)::value;
                        float v[8];
                        values(dbc, std::integral_constant<int, 2 * i>{}, v);
                        const auto s0 = __builtin_amdgcn_permlane32_swap(pack_bf16x2(v[0], v[1]), pack_bf16x2(v[4], v[5]), false, false);
                        const auto s1 = __builtin_amdgcn_permlane32_swap(pack_bf16x2(v[2], v[3]), pack_bf16x2(v[6], v[7]), false, false);
                        w[i][0] = s0[0]; w[i][1] = s1[0]; w[i][2] = s0[1]; w[i][3] = s1[1];
                    });
                    u32x4 lo, hi;
#pragma unroll
                    for (int j = 0; j < 4; ++j) {
                        const auto sw = __builtin_amdgcn_permlane16_swap(w[0][j], w[1][j], false, false);
                        lo[j] = sw[0]; hi[j] = sw[1];
                    }
                    if (real_lo) *reinterpret_cast<u32x4 *>(to_lo + db * 32) = lo;
                    if (real_hi) *reinterpret_cast<u32x4 *>(to_hi + db * 32) = hi;
                });
            } else {
                // [D / 4 chunks][rows][4 values], then the rows' references, then their sums
                static_for<G::kOBlocks * 2>([&](auto cc) {
                    constexpr int db = decltype(cc)::value / 2, i4 = (decltype(cc)::value % 2) * 2;
                    float v[8];
                    values(std::integral_constant<int, db>{}, std::integral_constant<int, i4>{}, v);
                    float4 *to = reinterpret_cast<float4 *>(rec) + (size_t)(db * 8 + 2 * i4 + h) * kPromptRows + row;
                    to[0] = make_float4(v[0], v[1], v[2], v[3]);
                    to[2 * kPromptRows] = make_float4(v[4], v[5], v[6], v[7]);
                });
            }
            if (h == 0) {
                if (!whole) {
                    float *ml = rec + (size_t)kPromptRows * D;
                    ml[row] = l == 0.f ? -INFINITY : ref;
                    ml[kPromptRows + row] = l;
                } else if (real && p.lse) {
                    p.lse[((size_t)seg_row0 + tok) * p.Hq + (size_t)seg_head * p.G + group_of(rc)] =
                        l == 0.f ? -INFINITY : (ref + __builtin_amdgcn_logf(l)) * kLn2;
                }
            }
            again = again || __any(real && !(check[0] + check[1] + check[2] + check[3] == 0.f));
        });
        if (!again) return;
        // the plain way, row after row: what has just been written is written again, behind it
        wait_vmcnt<0>();
        asm volatile("" ::: "memory");
        const int rows = min(64, min(tb, seg_nt) * p.G - wave_s * 64);
        for (int i = 0; i < rows; ++i) {
            const int row = wave_s * 64 + i, tok = (int)(((float)row + 0.5f) * p.g_rcp), g = row - tok * p.G;
            const size_t out_row = ((size_t)seg_row0 + tok) * p.Hq + (size_t)seg_head * p.G + g;
            const long long sees = min((long long)seg_p0 + tok + 1, (long long)p.max_seq_len);
            const int j1 = (int)min(sees, (long long)t_end * kTile);
            const ScalarRow<D> o = prompt_row_scalar<D>(p, p.q + out_row * D, page_table + (size_t)table_b * p.max_pages, seg_head,
                                                        seg_t0 * kTile, j1, lane, bad);
            const float inv = o.l == 0.f ? 0.f : 1.f / o.l;
#pragma unroll
            for (int e = 0; e < D / 64; ++e) {
                const int d = lane * (D / 64) + e;
                if (whole) p.out[out_row * D + d] = (uint16_t)pack_bf16x2(o.o[e] * inv, 0.f);
                else rec[((size_t)(d / 4) * kPromptRows + row) * 4 + d % 4] = o.o[e] * inv;
            }
            if (lane == 0) {
                if (!whole) {
                    rec[(size_t)kPromptRows * D + row] = o.l == 0.f ? -INFINITY : o.m;
                    rec[(size_t)kPromptRows * (D + 1) + row] = o.l;
                } else if (p.lse) {
                    p.lse[out_row] = o.l == 0.f ? -INFINITY : (o.m + __builtin_amdgcn_logf(o.l)) * kLn2;
                }
            }
        }
    };

    auto extend_list = [&](int it) {
        if ((it & (kPromptSlots / 2 - 1)) == 0 && it > 0) {
            const int first = it + kPromptSlots / 2;
            if (first < n_iter) {
                move_walk(first);
                if (tid < kPromptSlots / 2 && first + tid < n_iter) write_item(first + tid);
            }
        }
    };

    // words (keys, flags) of the tile to compute and of the one after it, and of the tile to copy, read ahead so that the LDS
    // latency hides behind the barrier
    int2 d_cur = *reinterpret_cast<const int2 *>(&desc_of(0)->n_valid);
    int2 d_nxt = *reinterpret_cast<const int2 *>(&desc_of(1)->n_valid);
    int2 d_cpy = *reinterpret_cast<const int2 *>(&desc_of(kS - 1)->n_valid);
    int d_blk = desc_of(kS - 1)->blk[cw];
    auto is_masked = [](int valid, int flags) { return ((valid ^ kTile) | (flags & kTileMasked)) != 0; };
    auto goes_on = [](int valid, int flags) { return ((valid ^ kTile) | (flags & (kTileFresh | kTileMasked | kTileHoles))) == 0; };

    struct Iter {
        int t_valid, t_flags;          // the tile to compute
        int c_blk;                     // first page block of the tile to copy (this wavefront's rows), or -1
        unsigned copy_stage_lds;
        bool last_iter, runs, masked;  // runs: tiles without holes
        bool pipelined, closing, copy_inside;   // the next tile of the run is whole; it, or this one, is masked
    };
    auto begin_iteration = [&](int it) {
        Iter I;
        I.t_valid = word(d_cur.x);
        I.t_flags = word(d_cur.y);
        const int n_valid = word(d_nxt.x), n_flags = word(d_nxt.y);
        const int c_valid = word(d_cpy.x);
        I.c_blk = word(d_blk);
        I.last_iter = it + 1 == n_iter;
        // Tiles up to it + 1 have to be complete in LDS (the pipelined tile code reads the next tile's K): this wavefront's
        // copies of them have landed once at most those of tile it + 2 are outstanding.
        if (it + 2 < n_iter) wait_vmcnt<kCopiesPerTile>();
        else wait_vmcnt<0>();
        __syncthreads();   // tiles it and it + 1 are complete in LDS; every wavefront is done with tile it - 1

        d_cur = d_nxt;
        d_nxt = *reinterpret_cast<const int2 *>(&desc_of(it + 2)->n_valid);
        d_cpy = *reinterpret_cast<const int2 *>(&desc_of(it + kS)->n_valid);
        d_blk = desc_of(it + kS)->blk[cw];
        extend_list(it);

        // Tile it + kS - 1 goes into the stage that tile it - 1 has left.
        const bool copy_next = it + kS - 1 < n_iter;
        I.copy_stage_lds = ring_lds + ((unsigned)(it + kS - 1) % kS) * G::kStageBytes;
        I.runs = (I.t_flags & kTileHoles) == 0;
        I.masked = is_masked(I.t_valid, I.t_flags);
        const bool more = wave_active && I.runs && !I.last_iter && (n_flags & (kTileFresh | kTileHoles)) == 0;
        I.pipelined = more && !I.masked && goes_on(n_valid, n_flags);
        I.closing = more && !I.pipelined;
        const bool whole_next = I.c_blk >= 0 && (cw + 1) * G::kRowsPerWave <= c_valid;
        I.copy_inside = copy_next && I.pipelined && whole_next;
        if (copy_next && !I.copy_inside) issue_tile(I.c_blk, c_valid, I.copy_stage_lds);
        if ((I.t_flags & kTileEnds) && !I.last_iter) {
            const PromptTile *d = desc_of(it + 1);
            prefetch_q(word(d->head), word(d->row0), word(d->nt));
        }
        return I;
    };
    auto whole_at = [&](int i) {
        const int2 d = *reinterpret_cast<const int2 *>(&desc_of(i)->n_valid);
        return goes_on(word(d.x), word(d.y));
    };
    auto stage_of = [&](int it) { return ring + ((unsigned)it % kS) * G::kStageBytes; };

    seg_p0 = word(desc_of(0)->p0); seg_t0 = word(desc_of(0)->t);
    wave_active = wave_token < seg_nt;
    reset_state();
    const Sees kNone[2] = {};
    for (int it = 0; it < n_iter; ++it) {
        Iter I = begin_iteration(it);
        if (!wave_active) {
        } else if (!I.runs) {
            tile_plain(stage_of(it), I.t_flags, I.t_valid, word(desc_of(it)->t));
        } else {
            // A run of tiles.  All but its last tile are pipelined, whole ones in a loop of their own.
            scores(stage_of(it));
            if (I.masked) {
                const Sees o = sees_of(I.t_valid, word(desc_of(it)->t));
                mask(0, o);
                mask(1, o);
            }
            if (I.t_flags & kTileFresh) static_for<2>([&](auto rc) { set_reference(rc); });
            begin_run();
            while (I.pipelined || I.closing) {
                if (I.copy_inside) {
                    // The middle of a run: as long as the tile after next and the tile to copy are whole too, a loop with one path
                    // through it and nothing between two tiles but the wait, the barrier and the words of the next tile to copy.
                    int blk = I.c_blk;
                    unsigned whole = (whole_at(it + 2) ? 1u : 0u) | (whole_at(it + 3) ? 2u : 0u);   // bit k: tile it + 2 + k
                    const int end = min(n_iter - kS + 1, (it | (kPromptSlots / 2 - 1)) + 1);         // (the list is extended by the general head)
                    for (;;) {
                        const size_t boff = (size_t)(unsigned)blk * (16 * G::kRowBytes);
                        tile_pipelined(std::true_type{}, std::false_type{}, kNone, stage_of(it), stage_of(it + 1), reinterpret_cast<const char *>(p.k_cache) + boff,
                                       reinterpret_cast<const char *>(p.v_cache) + boff, ring_lds + ((unsigned)(it + kS - 1) % kS) * G::kStageBytes);
                        ++it;
                        blk = word(d_blk);
                        const int c_valid = word(d_cpy.x), c_flags = word(d_cpy.y);
                        if (it >= end || (whole & 1u) == 0 || !goes_on(c_valid, c_flags)) break;
                        whole = (whole >> 1) | 2u;
                        wait_vmcnt<kCopiesPerTile>();
                        __syncthreads();        // tiles it and it + 1 are complete in LDS; every wavefront is done with tile it - 1
                        d_cpy = *reinterpret_cast<const int2 *>(&desc_of(it + kS)->n_valid);
                        d_blk = desc_of(it + kS)->blk[cw];
                    }
                    d_cur = *reinterpret_cast<const int2 *>(&desc_of(it)->n_valid);
                    d_nxt = *reinterpret_cast<const int2 *>(&desc_of(it + 1)->n_valid);
                } else if (I.pipelined) {
                    tile_pipelined(std::false_type{}, std::false_type{}, kNone, stage_of(it), stage_of(it + 1), nullptr, nullptr, 0u);
                    ++it;
                } else {
                    const PromptTile *d = desc_of(it), *d2 = desc_of(it + 1);
                    const Sees sees[2] = {sees_of(I.t_valid, word(d->t)), sees_of(word(d2->n_valid), word(d2->t))};
                    tile_pipelined(std::false_type{}, std::true_type{}, sees, stage_of(it), stage_of(it + 1), nullptr, nullptr, 0u);
                    ++it;
                }
                I = begin_iteration(it);    // (a whole tile that starts no segment: nothing else to prepare)
            }
            end_run();
            if (I.masked) {
                mask(1, sees_of(I.t_valid, word(desc_of(it)->t)));
            }
            weights_of_key_block(1);
            products(stage_of(it));
        }
        if (I.t_flags & kTileEnds) {
            const PromptTile *d = desc_of(it), *d2 = desc_of(it + 1);
            const int head = word(d2->head), row0 = word(d2->row0), p0 = word(d2->p0), nt = word(d2->nt), t0 = word(d2->t);
            if (wave_active) finish_segment(I.t_flags, word(d->t) + 1, word(d->b));
            if (!I.last_iter) {
                seg_head = head; seg_row0 = row0; seg_p0 = p0; seg_nt = nt; seg_t0 = t0;
                wave_active = wave_token < seg_nt;
                QueryRows q;
                fetch_q(q, head, row0, nt);
                reset_state();
                put_q(q);
            }
        }
    }
    if (p.status && bad) atomicOr(p.status, bad);
}

template <int D>
static hipError_t launch_prompt(const PromptParams &p, hipStream_t stream) {
    using G = Geometry<D, 4>;
    const size_t lds = (size_t)kPromptStages * G::kStageBytes + kPromptSlots * sizeof(PromptTile) + 64 * sizeof(float) +
                       (p.B <= kPromptSeqsInLds ? (2 * (size_t)p.B + 1) * sizeof(int) : 0);
    {
        static std::mutex guard;             // host threads may call in at the same time
        static size_t lds_allowed[kMaxDevices] = {};
        int device = 0;
        hipError_t e = hipGetDevice(&device);
        std::lock_guard<std::mutex> lock(guard);
        size_t *const allowed = e == hipSuccess && device < kMaxDevices ? &lds_allowed[device] : nullptr;
        if (!allowed || lds > *allowed) {
            e = hipFuncSetAttribute(reinterpret_cast<const void *>(&prompt_attn_kernel<D>), hipFuncAttributeMaxDynamicSharedMemorySize, (int)lds);
            if (e != hipSuccess) { (void)hipGetLastError(); return note_hip_error("hipFuncSetAttribute(prompt attention LDS size)", e); }
            if (allowed) *allowed = lds;
        }
    }
    hipLaunchKernelGGL((prompt_attn_kernel<D>), dim3(p.n_ranges), dim3(kPromptThreads), lds, stream, p, p.page_table);
    const hipError_t e = hipGetLastError();
    if (e != hipSuccess) return note_hip_error("launch prompt_attn_kernel", e);
    return launch_prompt_merge(p, kPromptRows, stream);
}

constexpr int kWideRanges = kNumCU;                  // workgroups of the launch: one a compute unit
static_assert(kWideRanges <= kMaxRanges, "the workspace has a note for each");

size_t prompt_wide_workspace_bytes(int D) { return ranges_workspace_bytes(kWideRanges, kPromptRows, D); }

hipError_t launch_prompt_wide(const PromptParams &params, hipStream_t stream) {
    PromptParams p = params;
    p.tokens_per_block = kPromptRows / p.G;
    p.n_ranges = kWideRanges;
    return p.D == 64 ? launch_prompt<64>(p, stream) : launch_prompt<128>(p, stream);
}

}  // namespace reader

// The attention weight that every cached key has drawn from the queries that count (a step's accepted path, or the last
// tokens of a prompt), per kv head:
//   weights[b, hkv, j] = decay * weights[b, hkv, j] + sum over rows (t, g) that see key j of exp(s <q[t, hkv G + g], k_j> - lse[t, hkv G + g])
// The log-sum-exp that the attention left turns a score into its softmax weight, so one product with the keys is all.  In powers of
// two it is rounded once more, to fp32: off by 2^-24 of it, as much as the attention's own rounding of it, 1.6e-7 of a weight on
// long contexts against 6.7e-8 where the scale is taken behind the difference, for one instruction less a weight.
//
// S = Q.K^T on the matrix cores in blocks of 16 rows x 16 keys (one page): a lane then holds four rows of one key, and the
// sum over rows is a sum over registers, with two exchanges between lanes at the end.  A wavefront holds up to 128 query rows
// as operands in registers and takes 64 keys a turn, whose pages travel to its own part of the LDS whole, 1 KB a copy
// instruction, four pages ahead.  (Loaded straight into the operand's layout, 64 bytes of 16 rows an instruction, they came at 4
// TB/s however many were asked for.)  Up to 128 rows a workgroup is one wavefront, which waits for nobody; beyond that two, four or
// eight of them share out the rows of the same keys and add up at the end of a turn (8 sequences of up to 2000 keys, 512 rows
// each, head dimension 64: 45 -> 20 us), and rows beyond those go through the keys once more.  Nobody else writes a key's weight: no
// atomics, the same bits every time.
// Bound by memory with few rows: 16 sequences of 1 to 4 K keys, 32 query and 8 kv heads, D 128, 6 tokens 19 us, 4.6 TB/s with the
// launch.  With 128 rows matrix instructions and exponentials take as long as the bytes, a SIMD's two wavefronts overlap them only
// in part: 4 sequences of 20 to 32 K keys, 32 tokens 53 us, 4.2 TB/s.
#include "prompt_common.h"
#include "tree_attn_common.h"

#include <type_traits>

namespace reader {

namespace {

typedef float f32x4 __attribute__((ext_vector_type(4)));
constexpr int kTurnPages = 4, kTurnKeys = kTurnPages * READER_PAGE_SIZE;
constexpr int kMaxTurns = 64 / kTurnPages;               // of a wavefront: a lane holds a page id

// positions of sequence `b` that may hold keys of it (0: none, or lengths that are no lengths)
__device__ inline int keys_of(const KeyWeightsParams &p, int b) {
    long long keys = p.seq_lens[b];
    bool ok = keys >= 0;
    if (!p.path) {
        const int lo = p.cu_tokens[b], hi = p.cu_tokens[b + 1];
        ok = ok && lo >= 0 && hi >= lo && hi <= p.N;
        keys += (long long)hi - lo;
    }
    return ok && keys <= min((long long)min(p.max_seq_len, p.max_positions), (long long)p.max_pages * READER_PAGE_SIZE) ? (int)keys : 0;
}

struct Share { int b, hkv, part, parts, turns; };

// A workgroup's share where all turns are more than the chip runs at a time: from the lengths themselves, which the host does not
// know, the fewest turns a workgroup with which all of them run at once (against an equal number of turns that the host takes from
// the longest length, rounded down: 16 sequences of 4000 keys, 128 rows, D 128 55 -> 43 us; rounded up that did as well, but ragged
// lengths then took 65 instead of 57).  A lane looks after up to kLaneSeqs sequences.
constexpr int kLaneSeqs = 4;
template <int kWaves>
__device__ inline Share share_of(const KeyWeightsParams &p, int lane) {
    const int per = (p.B + 63) / 64, slots = kNumCU * 8 / kWaves;
    int mine[kLaneSeqs], sum = 0;
#pragma unroll
    for (int i = 0; i < kLaneSeqs; ++i) {
        mine[i] = -1;                                    // no sequence
        if (i < per) {
            const int b = lane * per + i, keys = keys_of(p, min(b, p.B - 1));
            if (b < p.B) mine[i] = (keys + kTurnKeys - 1) / kTurnKeys;
        }
        sum += max(mine[i], 0);
    }
    auto over_lanes = [&](int x) {
#pragma unroll
        for (int d = 1; d < 64; d <<= 1) x += __shfl_xor(x, d);
        return __builtin_amdgcn_readfirstlane(x);
    };
    auto parts_of = [](int m, int t) { return m < 0 ? 0 : max((m + t - 1) / t, 1); };
    auto parts_here = [&](int t) {
        int n = 0;
#pragma unroll
        for (int i = 0; i < kLaneSeqs; ++i)
            if (i < per) n += parts_of(mine[i], t);
        return n;
    };
    const long long total = (long long)over_lanes(sum) * p.Hkv;
    int t = (int)min(max((total + slots - 1) / slots, 1LL), (long long)kMaxTurns);
    while (t < kMaxTurns && (long long)over_lanes(parts_here(t)) * p.Hkv > slots) ++t;
    const int here = parts_here(t);
    int upto = here;                                     // parts of this lane's sequences and those before
#pragma unroll
    for (int d = 1; d < 64; d <<= 1) {
        const int x = __shfl_up(upto, d);
        if (lane >= d) upto += x;
    }
    Share s = {};
    const int at = (int)blockIdx.x / p.Hkv;
    s.hkv = (int)blockIdx.x - at * p.Hkv;
    const unsigned long long behind = __ballot(upto > at);
    if (behind == 0) return s;                           // more workgroups than parts
    const int owner = __builtin_ctzll(behind);
    int left = at - (upto - here), b = 0, parts = 0;     // (of the owner's lane, the others' are dropped)
#pragma unroll
    for (int i = kLaneSeqs - 1, before = here; i >= 0; --i) {
        const int n = i < per ? parts_of(mine[i], t) : 0;
        before -= n;
        if (n > 0 && parts == 0 && left >= before) b = lane * per + i, parts = n, left -= before;
    }
    s.b = __shfl(b, owner), s.part = __shfl(left, owner), s.parts = __shfl(parts, owner), s.turns = t;
    s.b = __builtin_amdgcn_readfirstlane(s.b), s.part = __builtin_amdgcn_readfirstlane(s.part), s.parts = __builtin_amdgcn_readfirstlane(s.parts);
    return s;
}

// kBlocks: blocks of 16 query rows that a wavefront holds at a time.  turns: of a workgroup of the grid (parts, kv heads,
// sequences), or 0: shared out by the lengths
template <int D, int kBlocks, int kWaves>
__global__ __launch_bounds__(64 * kWaves, kBlocks * D <= 512 ? 3 : 2) void key_weights_kernel(KeyWeightsParams p, int turns) {
    constexpr int kSteps = D / 32;                       // 32-deep steps of the product
    constexpr int kRowBytes = D * 2, kChunks = D / 8, kPageBytes = READER_PAGE_SIZE * kRowBytes;
    constexpr int kCopies = kPageBytes / 1024, kRowsPerCopy = 64 / kChunks;
    __shared__ __attribute__((aligned(1024))) char s_ring[kWaves][kTurnPages * kPageBytes];   // of each wavefront: a turn's pages
    __shared__ float s_old[2][kTurnKeys];                                              // what the keys of a turn have so far
    __shared__ float s_sum[2][kWaves][kTurnKeys];                                      // what each wavefront's rows add
    const int lane = threadIdx.x & 63, wave = kWaves == 1 ? 0 : __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), i16 = lane & 15, quad = lane >> 4;
    // b, hkv: whose keys; turns from key0 on; this is part `part` of `parts` of them
    int hkv, b, key0, part, parts;
    if (turns > 0) {
        hkv = blockIdx.y, b = blockIdx.z, part = blockIdx.x, parts = gridDim.x, key0 = part * turns * kTurnKeys;
    } else {
        const Share s = share_of<kWaves>(p, lane);
        if (s.turns == 0) return;
        hkv = s.hkv, b = s.b, part = s.part, parts = s.parts, turns = s.turns, key0 = part * turns * kTurnKeys;
    }

    // (what does not depend on one another is asked for together: pages of this wavefront's keys, path, lengths)
    int page = p.page_table[(size_t)b * p.max_pages + min(key0 / READER_PAGE_SIZE + lane, p.max_pages - 1)];
    const int32_t *path = p.path + (p.path ? (size_t)b * p.max_path : 0);
    const int node = p.path ? path[min(lane, p.max_path - 1)] : 0, node2 = p.path ? path[min(lane + 64, p.max_path - 1)] : 0;
    const int len = p.seq_lens[b];

    // rows: `n` query tokens, the first of them at position `first`; row r is token r / G, head r % G of the group
    int n, bad = 0, token0 = 0;
    long long first_all;                                 // (lengths up to 2^31 - 1 add up to more)
    if (p.path) {
        n = p.accept_len[b] + 1;
        first_all = (long long)len - n;
        if (n < 1 || n > p.max_path || first_all < 0) bad = READER_STATUS_BAD_PATH;
        else if (__any((lane < n && (node < 0 || node >= p.T)) || (lane + 64 < n && (node2 < 0 || node2 >= p.T)))) bad = READER_STATUS_BAD_PATH;
    } else {
        const int lo = p.cu_tokens[b], hi = p.cu_tokens[b + 1], c0 = clamp_row(lo, p.N), c1 = clamp_row(hi, p.N);
        const int all = max(c1 - c0, 0);
        n = min(all, p.window);
        token0 = c1 - n;
        first_all = (long long)len + all - n;
        if (len < 0 || lo < 0 || hi < lo || hi > p.N) bad = READER_STATUS_BAD_LENGTH;
    }
    const long long keys_all = first_all + n;
    const long long most = min((long long)min(p.max_seq_len, p.max_positions), (long long)p.max_pages * READER_PAGE_SIZE);
    if (!bad && keys_all > most) bad = READER_STATUS_BAD_LENGTH;
    // (every wavefront of the sequence comes to the same verdict: it is left as it is)
    if (bad) {
        if (p.status && part == 0 && hkv == 0 && threadIdx.x == 0) atomicOr(p.status, bad);
        return;
    }
    const int first = (int)first_all, keys = (int)keys_all, rows = n * p.G;
    float *weights = p.weights + ((size_t)b * p.Hkv + hkv) * p.max_positions;
    if (p.decay == 0.f)                                  // a fresh start: nothing behind the last key
        for (long long j = keys + part * 64LL * kWaves + threadIdx.x; j < p.max_positions; j += parts * 64LL * kWaves) weights[j] = 0.f;
    if (key0 >= keys) return;
    if (rows == 0) {                                     // nobody to draw anything
        const int end = min(key0 + turns * kTurnKeys, keys);
        for (int j = key0 + (int)threadIdx.x; j < end; j += 64 * kWaves) weights[j] = p.decay == 0.f ? 0.f : p.decay * weights[j];
        return;
    }
    turns = min(turns, (keys - key0 + kTurnKeys - 1) / kTurnKeys);
    {
        const bool there = lane < turns * kTurnPages && key0 + lane * READER_PAGE_SIZE < keys, ok = page >= 0 && page < p.num_pages;
        if (__any(there && !ok) && p.status && threadIdx.x == 0) atomicOr(p.status, READER_STATUS_BAD_PAGE);
        page = there && ok ? page : -1;
    }

    // this lane's part of a copy: 16 bytes of row i * kRowsPerCopy + lane / kChunks, chunks swizzled by row
    unsigned copy_off[kCopies];
#pragma unroll
    for (int i = 0; i < kCopies; ++i) {
        const int r = i * kRowsPerCopy + lane / kChunks;
        copy_off[i] = r * kRowBytes + (((lane % kChunks) ^ swizzle_k<D>(r)) << 4);
    }
    char *const s_page = s_ring[wave];
    const unsigned page_lds = (unsigned)(size_t)(lds_char *)s_page;
    // Page `pg` of turn `turn` on its way to its place in the ring: kCopies instructions, whatever it is (a page that is not
    // there reads page 0, whose weights are dropped).
    auto copy_page = [&](int turn, int pg) {
        const int id = __builtin_amdgcn_readlane(page, turn * kTurnPages + pg);
        const char *base = reinterpret_cast<const char *>(p.k_cache) + ((size_t)max(id, 0) * p.Hkv + hkv) * kPageBytes;
#pragma unroll
        for (int i = 0; i < kCopies; ++i) copy16_uniform(base, copy_off[i], page_lds + pg * kPageBytes + i * 1024);
    };
    // what the keys of a turn have so far, by the same way: a load into a register would be waited for together with all copies
    auto copy_old = [&](int turn) {
        const float *src = weights + min(key0 + turn * kTurnKeys + lane, p.max_positions - 1);
        const unsigned dst = (unsigned)(size_t)(lds_char *)reinterpret_cast<char *>(s_old[turn & 1]);
        asm volatile("s_mov_b32 m0, %1\n\tglobal_load_lds_dword %0, off" :: "v"(src), "s"(dst) : "memory", "m0");
    };

    for (int r_all = 0; r_all < rows; r_all += kWaves * kBlocks * 16) {
        const int r_base = r_all + wave * kBlocks * 16;
        if constexpr (kWaves > 1) {
            if (r_base >= rows) {                        // a wavefront without rows adds nothing (rows do not come back either)
                for (int turn = 0; turn < turns; ++turn) {
                    s_sum[turn & 1][wave][lane] = 0.f;
                    __syncthreads();
                }
                __syncthreads();
                continue;
            }
        }
        const bool few = rows - r_base <= kBlocks * 4;   // a quarter of the blocks holds them
        if (wave == 0) copy_old(0);
#pragma unroll
        for (int pg = 0; pg < kTurnPages; ++pg) copy_page(0, pg);
        // the query rows as operands: block k, step s: row i16, values 32 s + 8 quad .. + 7; log-sum-exp (in
        // powers of two) of the four rows of this lane's results
        bf16x8 q[kBlocks][kSteps];
        float ref[kBlocks][4];
        auto place = [&](int r, int &t) {                // token and head of row r (half a row is far more than the product's rounding)
            t = (int)(((float)r + 0.5f) * p.g_rcp);
            return hkv * p.G + r - t * p.G;
        };
        const int top = rows - 1;
#pragma unroll
        for (int k = 0; k < kBlocks; ++k) {
            int t;
            const int head = place(min(r_base + k * 16 + i16, top), t);
            const size_t at = p.path ? (size_t)b * p.T + path[t] : (size_t)token0 + t;
#pragma unroll
            for (int s = 0; s < kSteps; ++s) q[k][s] = __builtin_bit_cast(bf16x8, ld16(p.q + (at * p.Hq + head) * D + s * 32 + quad * 8));
#pragma unroll
            for (int i = 0; i < 4; ++i) {
                const int r = r_base + k * 16 + quad * 4 + i;
                int ti;
                const int hi = place(min(r, top), ti);
                const float lse = p.path ? p.lse[((size_t)b * p.Hq + hi) * p.T + path[ti]] : p.lse[((size_t)token0 + ti) * p.Hq + hi];
                // (a row behind the last one, and one that saw no key at all, gives nothing)
                ref[k][i] = r < rows && lse != -INFINITY ? lse * 1.44269504088896340736f : INFINITY;
            }
        }
        for (int turn = 0; turn < turns; ++turn) {
            const int j0 = key0 + turn * kTurnKeys, j_mine = j0 + lane;
            const bool more = turn + 1 < turns;
            const bool causal = j0 + kTurnKeys > first + 1;      // some row does not see some of these keys
            float acc[kTurnPages];
#pragma unroll
            for (int pg = 0; pg < kTurnPages; ++pg) {
                // behind this page's copies stand those of three more pages (or nothing is on its way any more)
                if (more) wait_vmcnt<(kTurnPages - 1) * kCopies>();
                else wait_vmcnt<0>();
                asm volatile("" ::: "memory");
                bf16x8 key[kSteps];
#pragma unroll
                for (int s = 0; s < kSteps; ++s)
                    key[s] = *reinterpret_cast<const bf16x8 *>(s_page + pg * kPageBytes + i16 * kRowBytes + (((4 * s + quad) ^ swizzle_k<D>(i16)) << 4));
                // (the rows are in registers before the next turn's go to their place)
#pragma unroll
                for (int s = 0; s < kSteps; ++s) asm volatile("" : "+v"(key[s]) :: "memory");
                if (more) {
                    if (pg == 0 && wave == 0) copy_old(turn + 1);
                    copy_page(turn + 1, pg);
                }
                float sum = 0.f;
                auto add = [&](auto count, auto &&sees) {
#pragma unroll
                    for (int k = 0; k < decltype(count)::value; ++k) {
                        f32x4 x = {0.f, 0.f, 0.f, 0.f};
#pragma unroll
                        for (int s = 0; s < kSteps; ++s) x = __builtin_amdgcn_mfma_f32_16x16x32_bf16(q[k][s], key[s], x, 0, 0, 0);
#pragma unroll
                        for (int i = 0; i < 4; ++i) {
                            const float w = __builtin_amdgcn_exp2f(x[i] * p.scale_log2 - ref[k][i]);
                            sum += sees(k, i) ? w : 0.f;
                        }
                    }
                };
                auto seen = [&](int k, int i) {
                    int t;
                    place(r_base + k * 16 + quad * 4 + i, t);
                    return j0 + pg * 16 + i16 <= first + t;
                };
                auto all = [](int, int) { return true; };
                if (kBlocks >= 4 && few) {
                    if (causal) add(std::integral_constant<int, kBlocks / 4>(), seen);
                    else add(std::integral_constant<int, kBlocks / 4>(), all);
                } else if (causal) add(std::integral_constant<int, kBlocks>(), seen);
                else add(std::integral_constant<int, kBlocks>(), all);
                acc[pg] = sum;
            }
            // a key's four quarters of the rows sit 16 lanes apart; lane l then takes key l of the turn
            float sum = 0.f;
#pragma unroll
            for (int pg = 0; pg < kTurnPages; ++pg) {
                acc[pg] += __shfl_xor(acc[pg], 16);
                acc[pg] += __shfl_xor(acc[pg], 32);
                sum = quad == pg ? acc[pg] : sum;
            }
            if constexpr (kWaves > 1) {
                s_sum[turn & 1][wave][lane] = sum;
                __syncthreads();
                if (wave > 0) continue;
#pragma unroll
                for (int w = 1; w < kWaves; ++w) sum += s_sum[turn & 1][w][lane];
            }
            const float old = s_old[turn & 1][lane];
            const bool ok = __shfl(page, turn * kTurnPages + quad) >= 0;
            if (j_mine < keys) weights[j_mine] = (r_all > 0 ? old : p.decay == 0.f ? 0.f : p.decay * old) + (ok ? sum : 0.f);
        }
        wait_vmcnt<0>();                                 // (what has been written is read again for the next rows)
        asm volatile("" ::: "memory");
        if constexpr (kWaves > 1) __syncthreads();       // (the next rows' first sums take the place of sums that may still be read)
    }
}

template <int D, int kBlocks, int kWaves>
hipError_t launch_blocks(const KeyWeightsParams &p, int span, hipStream_t stream) {
    // turns of a workgroup: one, where all of them run at a time (8 wavefronts a compute unit).  Where they do not, up to 256
    // sequences are shared out by their lengths (every part of a sequence but its last is full, so there are at most `slots` of
    // full ones, or as many as the most turns leave); more sequences even out by themselves
    const long long all = (long long)((span + kTurnKeys - 1) / kTurnKeys) * p.Hkv * p.B, slots = kNumCU * 8 / kWaves;
    const long long most = max(slots, all / kMaxTurns) + (long long)p.B * p.Hkv;
    const bool shared = all > slots && p.B <= 64 * kLaneSeqs && most * 64 * kWaves < (1LL << 32);   // (a launch counts threads in 32 bits)
    int turns = shared ? 0 : (int)min(max(all / slots, 1LL), (long long)kMaxTurns);
    dim3 grid((unsigned)((span + turns * kTurnKeys - 1) / max(turns * kTurnKeys, 1)), (unsigned)p.Hkv, (unsigned)p.B);
    if (shared) grid = dim3((unsigned)most, 1, 1);
    hipLaunchKernelGGL((key_weights_kernel<D, kBlocks, kWaves>), grid, dim3(64 * kWaves), 0, stream, p, turns);
    return note_hip_error("launch key_weights_kernel", hipGetLastError());
}

template <int D>
hipError_t launch_rows(const KeyWeightsParams &p, int span, hipStream_t stream) {
    const long long rows = (long long)(p.path ? p.max_path : min(p.window, p.N)) * p.G;      // no sequence has more
    if (rows <= 16) return launch_blocks<D, 1, 1>(p, span, stream);
    if (rows <= 32) return launch_blocks<D, 2, 1>(p, span, stream);
    if (rows <= 64) return launch_blocks<D, 4, 1>(p, span, stream);
    if (rows <= 128) return launch_blocks<D, 8, 1>(p, span, stream);
    if (rows <= 256) return launch_blocks<D, 8, 2>(p, span, stream);
    if (rows <= 512 || (long long)((span + kTurnKeys - 1) / kTurnKeys) * p.Hkv * p.B > 2 * kNumCU) return launch_blocks<D, 8, 4>(p, span, stream);
    // (where a workgroup of eight is all that a compute unit gets.  2 sequences of 1000 keys, 984 rows: 32 -> 23 us; 64 of 3000, 800
    // rows: 94, and 125 with eight)
    return launch_blocks<D, 8, 8>(p, span, stream);
}

}  // namespace

hipError_t launch_key_weights(const KeyWeightsParams &p, hipStream_t stream) {
    // (a fresh start clears the whole row; where no position is allowed, lengths are still looked at)
    const int span = max(p.decay == 0.f ? p.max_positions : min(p.max_seq_len, p.max_positions), 1);
    return p.D == 64 ? launch_rows<64>(p, span, stream) : launch_rows<128>(p, span, stream);
}

}  // namespace reader

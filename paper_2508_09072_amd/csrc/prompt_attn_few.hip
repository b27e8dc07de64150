// Causal attention of packed prompts over the paged cache for few query rows a kv head: single tokens, short chunks.
//
// Bound by memory: every key and value feeds a handful of rows.  So a workgroup is one wavefront that waits for nobody: it takes a
// range of the (head, sequence, block, key) axis (prompt_ranges.h; a block is 16 or 32 rows here) and streams its keys 32 at a
// time, whole pages, 1 KB a copy instruction, through two stages of its own in LDS.  S^T = K.Q^T in blocks of 16 keys x 16 rows leaves a lane with eight scores of one row, which are, as they
// stand, the operand of O^T += V^T.P^T: the order of keys in that product is chosen to fit.  The running maximum moves only
// when a score is 2^16 above it (weights are then at most that: nothing to lose in fp32 sums and bf16 weights), so that the
// lanes of a row, which share its maximum, hardly ever have to agree on one.  Blocks that are cut leave fp32 records.
#include <mutex>

#include "prompt_attn_scalar.h"
#include "prompt_ranges.h"

namespace reader {

namespace {

typedef float f32x4 __attribute__((ext_vector_type(4)));
constexpr int kStep = 32, kStepPages = kStep / READER_PAGE_SIZE;
constexpr int kMinRange = 8 * kStep;
using Block = PromptBlock<kStep, 2 * kStep, 4 * kStep>;
constexpr float kNoReference = -1e30f, kMargin = 16.f;

// Wavefronts of a compute unit that run at once: as many as their stages fit the LDS.
constexpr int few_wavefronts(int D) { return D == 128 ? 4 : 8; }

__device__ __forceinline__ long long scan64(long long c, int lane) {
#pragma unroll
    for (int off = 1; off < 64; off <<= 1) {
        const long long v = __shfl_up(c, off);
        if (lane >= off) c += v;
    }
    return c;
}

// kBlocks: blocks of 16 query rows
template <int D, int kBlocks>
__global__ __launch_bounds__(64) void prompt_few_kernel(PromptParams p) {
    constexpr int kSteps = D / 32, kOut = D / 16;        // 32-deep steps of the first product, 16-wide blocks of the output
    constexpr int kRowBytes = D * 2, kChunks = D / 8, kPageBytes = READER_PAGE_SIZE * kRowBytes;
    constexpr int kCopies = kPageBytes / 1024, kRowsPerCopy = 64 / kChunks;
    constexpr int kStageCopies = 2 * kStepPages * kCopies, kRows = kBlocks * 16;
    __shared__ __attribute__((aligned(1024))) char s_stage[2][2 * kStepPages * kPageBytes];   // pages of K, then of V
    __shared__ int s_ids[2][64];                         // page ids of the segment, 64 at a time
    const int lane = threadIdx.x, i16 = lane & 15, quad = lane >> 4, tb = p.tokens_per_block;
    RangeNote *const notes = reinterpret_cast<RangeNote *>(p.workspace);
    const Sequences seqs{p.seq_lens, p.cu_tokens, p.N, p.max_seq_len};
    int bad = 0;

    // ---- this wavefront's range of the axis
    long long per_head = 0;
    for (int base = 0; base < p.B; base += 64) {
        const int b = base + lane;
        long long c = 0;
        if (b < p.B) {
            const int nn = seqs.tokens(b), len = p.seq_lens[b], lo = p.cu_tokens[b], hi = p.cu_tokens[b + 1];
            c = Block::sequence_cost(seqs.length(b), nn, tb);
            if (len < 0 || lo < 0 || hi < lo || hi > p.N || (long long)len + nn > p.max_seq_len) bad |= READER_STATUS_BAD_LENGTH;
        }
        per_head += __shfl(scan64(c, lane), 63);
    }
    if (bad && blockIdx.x == 0 && p.status) atomicOr(p.status, bad);
    bad = 0;
    const long long total = per_head * p.Hkv;
    long long n_ranges = total / kMinRange;
    n_ranges = n_ranges > (long long)gridDim.x ? gridDim.x : (n_ranges < 1 ? 1 : n_ranges);
    const int range = blockIdx.x;
    if (range >= n_ranges || total == 0) {
        if (lane == 0) notes[range] = RangeNote{};
        return;
    }
    auto locate = [&](long long x, Block &o) {
        if (x >= total) {
            o = Block{p.Hkv, 0, 0, 0, 0, 0};
            return 0;
        }
        o.head = (int)(x / per_head);
        const long long r = x - o.head * per_head;
        long long carry = 0;
        for (int base = 0;; base += 64) {
            const int b = base + lane;
            const long long upto = carry + scan64(b < p.B ? Block::sequence_cost(seqs.length(b), seqs.tokens(b), tb) : 0, lane);
            const long long all = __shfl(upto, 63);
            if (r < all) {                               // (the last of these 64 at the latest: r is below per_head)
                const int i = (int)__popcll(__ballot(upto <= r));
                o.b = base + i;
                carry = i > 0 ? __shfl(upto, i - 1) : carry;
                break;
            }
            carry = all;
        }
        o.load(seqs);
        return o.locate(r - carry, seqs, p.B, tb);
    };
    Block from, to;
    const int t_from = locate(range * total / n_ranges, from), t_to = locate((range + 1) * total / n_ranges, to);
    const PromptRange<Block> rg(from, t_from, to, t_to, p.Hkv);
    const RangeNote note = rg.note(seqs, p.B, tb);
    if (lane == 0) notes[range] = note;

    // this lane's part of a copy: 16 bytes of row i * kRowsPerCopy + lane / kChunks; chunks swizzled by row, so that the reads of an
    // operand touch every bank once (K: 16 rows, one chunk; V: 8 rows, two chunks side by side)
    auto swizzle_v16 = [](int row) { return D == 128 ? (row & 7) << 1 : ((row >> 1) & 3) << 1; };
    unsigned k_off[kCopies], v_off[kCopies];
#pragma unroll
    for (int i = 0; i < kCopies; ++i) {
        const int r = i * kRowsPerCopy + lane / kChunks;
        k_off[i] = r * kRowBytes + (((lane % kChunks) ^ swizzle_k<D>(r)) << 4);
        v_off[i] = r * kRowBytes + (((lane % kChunks) ^ swizzle_v16(r)) << 4);
    }
    const int v_row = quad * 4 + (i16 >> 2);
    const int v_rd = v_row * kRowBytes + (i16 & 1) * 8, v_chunk = (i16 & 3) >> 1;
    const unsigned stage_lds = (unsigned)(size_t)(lds_char *)&s_stage[0][0];
    const unsigned ids_lds = (unsigned)(size_t)(lds_char *)reinterpret_cast<char *>(&s_ids[0][0]);

    Block o = rg.at;
    for (bool first_block = true; !rg.behind(o); first_block = false) {
        int t0, t1;
        rg.share(o, first_block, tb, p.max_seq_len, t0, t1);
        const int keys = o.keys(tb, p.max_seq_len), nt = o.tokens(tb), row0 = o.c0 + o.k * tb, all = o.tiles(tb, p.max_seq_len);
        const long long p0 = (long long)o.L + o.k * tb;
        const bool last_block = rg.is_stop(o);
        if (t1 > t0) {
            const int32_t *table = p.page_table + (size_t)o.b * p.max_pages;
            const int steps = t1 - t0, page0 = t0 * kStepPages;
            auto load_ids = [&](int c) {
                const int32_t *src = table + min(page0 + c * 64 + lane, p.max_pages - 1);
                const unsigned dst = ids_lds + (c & 1) * 256;
                asm volatile("s_mov_b32 m0, %1\n\tglobal_load_lds_dword %0, off" :: "v"(src), "s"(dst) : "memory", "m0");
            };
            // page `pg` of step i: its id, or -1 where there is nothing to read
            auto id_of = [&](int i, int pg) {
                const int at = i * kStepPages + pg, id = __builtin_amdgcn_readfirstlane(s_ids[(at >> 6) & 1][at & 63]);
                return (page0 + at) * READER_PAGE_SIZE < keys && id >= 0 && id < p.num_pages ? id : -1;
            };
            // kStageCopies copy instructions, whatever the pages are; rows that nobody sees are copied from a block of zeros, so
            // that a weight of zero times them stays zero
            auto issue = [&](int i) {
                const unsigned stage = stage_lds + (i & 1) * (2 * kStepPages * kPageBytes);
#pragma unroll
                for (int pg = 0; pg < kStepPages; ++pg) {
                    const int id = id_of(i, pg), rows = keys - (page0 + i * kStepPages + pg) * READER_PAGE_SIZE;
                    const size_t at = ((size_t)max(id, 0) * p.Hkv + o.head) * kPageBytes;
                    const char *kb = reinterpret_cast<const char *>(p.k_cache) + at, *vb = reinterpret_cast<const char *>(p.v_cache) + at;
                    const bool whole = id >= 0 && rows >= READER_PAGE_SIZE;
                    const char *zeros = reinterpret_cast<const char *>(kZeroRow) + (lane & 15) * 16;
#pragma unroll
                    for (int j = 0; j < kCopies; ++j) {
                        const unsigned kd = stage + pg * kPageBytes + j * 1024, vd = kd + kStepPages * kPageBytes;
                        if (whole) {
                            copy16_uniform(kb, k_off[j], kd);
                            copy16_uniform(vb, v_off[j], vd);
                        } else {
                            const bool ok = id >= 0 && j * kRowsPerCopy + lane / kChunks < rows;
                            copy16_lane(ok ? kb + k_off[j] : zeros, kd);
                            copy16_lane(ok ? vb + v_off[j] : zeros, vd);
                        }
                    }
                }
            };
            load_ids(0);
            // the query rows as operands: block r, step s: row i16, values 32 s + 8 quad .. + 7
            bf16x8 q[kBlocks][kSteps];
            int lim[kBlocks];                            // keys that row i16 of block r sees
            size_t out_row[kBlocks];
            bool real[kBlocks];
#pragma unroll
            for (int r = 0; r < kBlocks; ++r) {
                const int row = r * 16 + i16, tok = (int)(((float)row + 0.5f) * p.g_rcp);    // row / G
                real[r] = tok < nt;
                lim[r] = real[r] ? (int)min(p0 + tok + 1, (long long)p.max_seq_len) : 0;
                out_row[r] = ((size_t)row0 + min(tok, nt - 1)) * p.Hq + (size_t)o.head * p.G + (row - tok * p.G);
#pragma unroll
                for (int s = 0; s < kSteps; ++s) q[r][s] = __builtin_bit_cast(bf16x8, keep_if(real[r], ld16(p.q + out_row[r] * D + s * 32 + quad * 8)));
            }
            f32x4 acc[kBlocks][kOut];
            float m[kBlocks], l[kBlocks];
#pragma unroll
            for (int r = 0; r < kBlocks; ++r) {
                m[r] = kNoReference;
                l[r] = 0.f;
#pragma unroll
                for (int db = 0; db < kOut; ++db) acc[r][db] = f32x4{0.f, 0.f, 0.f, 0.f};
            }
            wait_vmcnt<0>();                             // the first page ids are there (and the last segment's copies)
            asm volatile("" ::: "memory");
            issue(0);
            if (steps > 1) issue(1);
            for (int i = 0; i < steps; ++i) {
                if (i % 32 == 0 && i + 32 < steps) load_ids(i / 32 + 1);
                if (i + 1 < steps) wait_vmcnt<kStageCopies>();
                else wait_vmcnt<0>();
                asm volatile("" ::: "memory");
                const char *stage = s_stage[i & 1];
                const int j0 = (t0 + i) * kStep;
                const int id0 = id_of(i, 0), id1 = id_of(i, 1);
                const bool hole0 = id0 < 0 && j0 < keys, hole1 = id1 < 0 && j0 + READER_PAGE_SIZE < keys;
                if (hole0 || hole1) bad |= READER_STATUS_BAD_PAGE;
                const bool masked = j0 + kStep > p0 + 1 || j0 + kStep > p.max_seq_len || hole0 || hole1;
                u32x4 pk[kBlocks];
                {
                    bf16x8 key[kStepPages][kSteps];
#pragma unroll
                    for (int pg = 0; pg < kStepPages; ++pg)
#pragma unroll
                        for (int s = 0; s < kSteps; ++s)
                            key[pg][s] = *reinterpret_cast<const bf16x8 *>(stage + pg * kPageBytes + i16 * kRowBytes + (((4 * s + quad) ^ swizzle_k<D>(i16)) << 4));
#pragma unroll
                    for (int r = 0; r < kBlocks; ++r) {
                        f32x4 x[kStepPages];
#pragma unroll
                        for (int pg = 0; pg < kStepPages; ++pg) {
                            x[pg] = f32x4{0.f, 0.f, 0.f, 0.f};
#pragma unroll
                            for (int s = 0; s < kSteps; ++s) x[pg] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(key[pg][s], q[r][s], x[pg], 0, 0, 0);
                        }
                        if (masked) {
#pragma unroll
                            for (int pg = 0; pg < kStepPages; ++pg)
#pragma unroll
                                for (int e = 0; e < 4; ++e)
                                    if (j0 + pg * 16 + quad * 4 + e >= lim[r] || (pg == 0 ? hole0 : hole1)) x[pg][e] = -INFINITY;
                        }
                        float mx = fmaxf(fmaxf(x[0][0], x[0][1]), fmaxf(x[0][2], x[0][3]));
                        mx = fmaxf(mx, fmaxf(fmaxf(x[1][0], x[1][1]), fmaxf(x[1][2], x[1][3]))) * p.scale_log2;
                        if (__any(mx > m[r] + kMargin)) {
                            mx = fmaxf(mx, __shfl_xor(mx, 16));
                            mx = fmaxf(mx, __shfl_xor(mx, 32));
                            const float top = fmaxf(m[r], mx), f = __builtin_amdgcn_exp2f(m[r] - top);
                            m[r] = top;
                            l[r] *= f;
#pragma unroll
                            for (int db = 0; db < kOut; ++db) acc[r][db] *= f;
                        }
                        float w[8];
#pragma unroll
                        for (int e = 0; e < 8; ++e) {
                            w[e] = __builtin_amdgcn_exp2f(x[e / 4][e % 4] * p.scale_log2 - m[r]);
                            l[r] += w[e];
                        }
#pragma unroll
                        for (int e = 0; e < 4; ++e) pk[r][e] = pack_bf16x2(w[2 * e], w[2 * e + 1]);
                    }
                }
                // key 8 quad' + j of this product is key 4 quad + j % 4 of page j / 4, in both operands
                s16x4 vf[kOut][kStepPages];
#pragma unroll
                for (int db = 0; db < kOut; ++db)
#pragma unroll
                    for (int pg = 0; pg < kStepPages; ++pg)
                        vf[db][pg] = lds_read_tr16(stage + (kStepPages + pg) * kPageBytes + v_rd + (((db * 2 + v_chunk) ^ swizzle_v16(v_row)) << 4));
                // (the values are in registers before the step after next goes to their place)
#pragma unroll
                for (int db = 0; db < kOut; ++db) asm volatile("" : "+v"(vf[db][0]), "+v"(vf[db][1]) :: "memory");
                if (i + 2 < steps) issue(i + 2);
#pragma unroll
                for (int db = 0; db < kOut; ++db) {
                    const bf16x8 v8 = __builtin_bit_cast(bf16x8, __builtin_shufflevector(vf[db][0], vf[db][1], 0, 1, 2, 3, 4, 5, 6, 7));
#pragma unroll
                    for (int r = 0; r < kBlocks; ++r)
                        acc[r][db] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(v8, __builtin_bit_cast(bf16x8, pk[r]), acc[r][db], 0, 0, 0);
                }
            }
            // ---- end of the segment: the whole block is normalised and written out, a part of one leaves a record
            const bool whole = t0 == 0 && t1 == all;
            float *rec = reinterpret_cast<float *>(reinterpret_cast<char *>(p.workspace) + kNotesBytes) +
                         (size_t)(2 * range + (t0 == 0 ? 1 : 0)) * ((size_t)kRows * (D + 2));
            bool again = false;
#pragma unroll
            for (int r = 0; r < kBlocks; ++r) {
                l[r] += __shfl_xor(l[r], 16);
                l[r] += __shfl_xor(l[r], 32);
                const float inv = l[r] == 0.f ? 0.f : 1.f / l[r];         // (a row may see no key of a part)
                float check = l[r] * 0.f;                                 // (not a number once any value is none)
#pragma unroll
                for (int db = 0; db < kOut; ++db) {
                    const f32x4 v = acc[r][db] * inv;
                    check = check + v[0] * 0.f + v[1] * 0.f + v[2] * 0.f + v[3] * 0.f;
                    if (!whole) reinterpret_cast<f32x4 *>(rec)[(size_t)(db * 4 + quad) * kRows + r * 16 + i16] = v;
                    else if (real[r])
                        *reinterpret_cast<uint2 *>(p.out + out_row[r] * D + db * 16 + quad * 4) = make_uint2(pack_bf16x2(v[0], v[1]), pack_bf16x2(v[2], v[3]));
                }
                if (quad == 0) {
                    if (!whole) {
                        rec[(size_t)kRows * D + r * 16 + i16] = l[r] == 0.f ? -INFINITY : m[r];
                        rec[(size_t)kRows * (D + 1) + r * 16 + i16] = l[r];
                    } else if (real[r] && p.lse) {
                        p.lse[out_row[r]] = l[r] == 0.f ? -INFINITY : (m[r] + __builtin_amdgcn_logf(l[r])) * kLn2;
                    }
                }
                again = again || __any(real[r] && !(check == 0.f));
            }
            if (again) {
                // A value that is not a number, maybe behind a mask (times a weight of zero): the plain way, row after row; what has
                // just been written is written again, behind it.
                wait_vmcnt<0>();
                asm volatile("" ::: "memory");
                for (int row = 0; row < nt * p.G; ++row) {
                    const int tok = row / p.G;
                    const size_t at = ((size_t)row0 + tok) * p.Hq + (size_t)o.head * p.G + (row - tok * p.G);
                    const int j1 = (int)min(min(p0 + tok + 1, (long long)p.max_seq_len), (long long)t1 * kStep);
                    const ScalarRow<D> s = prompt_row_scalar<D>(p, p.q + at * D, table, o.head, t0 * kStep, j1, lane, bad);
                    const float inv = s.l == 0.f ? 0.f : 1.f / s.l;
#pragma unroll
                    for (int e = 0; e < D / 64; ++e) {
                        const int d = lane * (D / 64) + e;
                        if (whole) p.out[at * D + d] = (uint16_t)pack_bf16x2(s.o[e] * inv, 0.f);
                        else rec[((size_t)(d / 4) * kRows + row) * 4 + d % 4] = s.o[e] * inv;
                    }
                    if (lane == 0) {
                        if (!whole) {
                            rec[(size_t)kRows * D + row] = s.l == 0.f ? -INFINITY : s.m;
                            rec[(size_t)kRows * (D + 1) + row] = s.l;
                        } else if (p.lse) {
                            p.lse[at] = s.l == 0.f ? -INFINITY : (s.m + __builtin_amdgcn_logf(s.l)) * kLn2;
                        }
                    }
                }
            }
        }
        if (last_block) break;
        o.next(seqs, p.B, tb);
        o.make_uniform();
    }
    if (p.status && bad) atomicOr(p.status, bad);
}

template <int D, int kBlocks>
hipError_t launch_few(const PromptParams &p, hipStream_t stream) {
    hipLaunchKernelGGL((prompt_few_kernel<D, kBlocks>), dim3(p.n_ranges), dim3(64), 0, stream, p);
    const hipError_t e = hipGetLastError();
    if (e != hipSuccess) return note_hip_error("launch prompt_few_kernel", e);
    return launch_prompt_merge(p, kBlocks * 16, stream);
}

}  // namespace

hipError_t launch_prompt_few(const PromptParams &params, int rows, hipStream_t stream) {
    PromptParams p = params;
    p.tokens_per_block = rows / p.G;
    p.n_ranges = kNumCU * few_wavefronts(p.D);
    if (rows == 16) return p.D == 64 ? launch_few<64, 1>(p, stream) : launch_few<128, 1>(p, stream);
    return p.D == 64 ? launch_few<64, 2>(p, stream) : launch_few<128, 2>(p, stream);
}

size_t prompt_few_workspace_bytes(int D) { return kNotesBytes + (size_t)2 * kNumCU * few_wavefronts(D) * 32 * (D + 2) * sizeof(float); }

}  // namespace reader

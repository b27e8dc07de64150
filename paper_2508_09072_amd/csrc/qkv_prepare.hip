// Queries, keys and values of a pass's tokens from their projections (the "positions of tree nodes" that the attention
// takes for granted): a norm of every query and key head, the position rotation, and the way to where the attention reads
// them, in one pass over the data.
//   y = w * x / sqrt(mean(x^2) + eps)                       (heads of q and k; left out without norm weights)
//   (y_i, y_j) -> (y_i cos - y_j sin, y_j cos + y_i sin)    (pairs of the first `rot` values; the angle is the position's)
// v is copied.  Everything is computed in 32 bits and rounded once, at the end.
//
// Bound by memory: 4 (Hq + 2 Hkv) D bytes a token in and out, and a row of the rotation table for all heads of a token.  16 prompts
// of 301 to 2500 tokens with 48 heads of 128 (479 MB): 110 us, 4.4 TB/s, where a copy of 2 GB reaches 4.8.
#include "prompt_common.h"
#include "tree_attn_common.h"

namespace reader {

namespace {

constexpr int kQkvThreads = 256;

__device__ inline void unpack8(const u32x4 &w, float (&x)[8]) {
#pragma unroll
    for (int i = 0; i < 4; ++i) {
        x[2 * i] = __uint_as_float(w[i] << 16);
        x[2 * i + 1] = __uint_as_float(w[i] & 0xffff0000u);
    }
}

// A wavefront takes one token and every `parts`-th group of its head rows.  A row is D / 8 lanes of 8 values.
// kPacked: rows of packed prompts, else nodes of trees.  (80 registers at most, for six wavefronts a SIMD: five take 10 % longer.)
template <int D, bool kPacked>
__global__ __launch_bounds__(kQkvThreads, 6) void qkv_kernel(QkvParams p, int parts) {
    constexpr int kLanes = D / 8, kRows = 64 / kLanes;
    const int lane = threadIdx.x & 63;
    // (the first workgroup of packed rows looks the table over, whether or not anybody owns a row of what is wrong)
    if (kPacked && blockIdx.x == 0) {
        int wrong = 0;
#pragma unroll 4
        for (int b = threadIdx.x; b < p.B; b += kQkvThreads) wrong |= bad_sequence(p.cu_tokens, p.seq_lens, p.N, b);
        if (wrong && p.status) atomicOr(p.status, wrong);
        return;
    }
    const long long unit = (long long)(blockIdx.x - (kPacked ? 1 : 0)) * (kQkvThreads / 64) + __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    const int token = (int)(unit / parts), part = (int)(unit - (long long)token * parts);
    if (token >= p.N) return;

    // the token's sequence, its row there, how far behind the sequence's first new position it stands
    int b, row, ahead, bad = 0;
    bool skip = false;
    if constexpr (kPacked) {
        int first = 0;
        b = sequence_of_row(p.cu_tokens, p.B, token, lane, first);
        if (b >= p.B) return;                            // in front of the first or behind the last sequence: left as it is
        row = token - first;
        ahead = row;
    } else {
        b = token / p.T;
        row = token - b * p.T;
        // depth: the number of links up to the root (a bad link counts as one to the root, as in the attention)
        const int32_t *parents = p.parents + (size_t)b * p.T;
        const int lo = parents[min(lane, p.T - 1)], hi = parents[min(lane + 64, p.T - 1)];
        ahead = 0;
        for (int t = row; t > 0; ++ahead) {
            int up = t < 64 ? __builtin_amdgcn_readlane(lo, t) : __builtin_amdgcn_readlane(hi, t - 64);
            if (up < 0 || up >= t) { bad |= READER_STATUS_BAD_TREE; up = 0; }
            t = up;
        }
        if (row == 0 && __builtin_amdgcn_readlane(lo, 0) != -1) bad |= READER_STATUS_BAD_TREE;
    }
    const int L = p.seq_lens[b];
    const long long pos = (long long)(p.positions ? p.positions[b] : L) + ahead;
    if (p.rot > 0 && (pos < 0 || pos >= p.max_positions)) { bad |= READER_STATUS_BAD_LENGTH; skip = true; }
    // where the key and value rows go: [Hkv] rows `stride` apart from `at`
    size_t at = 0, stride = D;
    bool store_kv = !skip;
    if (!kPacked && p.k_tree) {
        at = (size_t)token * p.Hkv * D;
    } else {
        const long long j = (long long)L + row;
        if (L < 0 || j < 0 || j >= (long long)p.max_pages * READER_PAGE_SIZE) {
            bad |= READER_STATUS_BAD_LENGTH;
            store_kv = false;
        } else {
            const int page = p.page_table[(size_t)b * p.max_pages + (j >> 4)];
            if (page < 0 || page >= p.num_pages) { bad |= READER_STATUS_BAD_PAGE; store_kv = false; }
            else at = ((size_t)page * p.Hkv * READER_PAGE_SIZE + (j & 15)) * D;
            stride = READER_PAGE_SIZE * D;
        }
    }
    if (bad && p.status && lane == 0 && part == 0) atomicOr(p.status, bad);
    if (skip) return;
    uint16_t *const k_out = (!kPacked && p.k_tree ? p.k_tree : p.k_cache) + at, *const v_out = (!kPacked && p.k_tree ? p.v_tree : p.v_cache) + at;

    // this lane's values of a head row: 8 c .. 8 c + 7; the angles of its pairs and, of pairs half a rotation apart, the
    // lane that holds the other halves
    const int c = lane % kLanes, r0 = lane / kLanes;
    const int pair_lanes = p.rot / 16;                   // lanes that hold the first halves
    const bool rotates = c < 2 * pair_lanes, second = c >= pair_lanes;
    const int partner = lane + (rotates && !p.interleaved ? (second ? -pair_lanes : pair_lanes) : 0);
    float cs[8], sn[8];
#pragma unroll
    for (int i = 0; i < 8; ++i) { cs[i] = 1.f; sn[i] = 0.f; }
    if (rotates) {
        const float *cos_row = p.cos_sin + (size_t)pos * p.rot, *sin_row = cos_row + p.rot / 2;
        if (p.interleaved) {
            const float4 a = *reinterpret_cast<const float4 *>(cos_row + 4 * c), d = *reinterpret_cast<const float4 *>(sin_row + 4 * c);
            cs[0] = cs[1] = a.x; cs[2] = cs[3] = a.y; cs[4] = cs[5] = a.z; cs[6] = cs[7] = a.w;
            sn[0] = -d.x; sn[1] = d.x; sn[2] = -d.y; sn[3] = d.y; sn[4] = -d.z; sn[5] = d.z; sn[6] = -d.w; sn[7] = d.w;
        } else {
            const int i0 = 8 * (second ? c - pair_lanes : c);
            const float sign = second ? 1.f : -1.f;
#pragma unroll
            for (int i = 0; i < 8; i += 4) {
                const float4 a = *reinterpret_cast<const float4 *>(cos_row + i0 + i), d = *reinterpret_cast<const float4 *>(sin_row + i0 + i);
                cs[i] = a.x; cs[i + 1] = a.y; cs[i + 2] = a.z; cs[i + 3] = a.w;
                sn[i] = sign * d.x; sn[i + 1] = sign * d.y; sn[i + 2] = sign * d.z; sn[i + 3] = sign * d.w;
            }
        }
    }
    u32x4 w_mine[2] = {}, w_other[2] = {};               // norm weights of q and k: of this lane's values, of its partner's
    if (p.q_norm) {
        w_mine[0] = ld16(p.q_norm + 8 * c); w_other[0] = ld16(p.q_norm + 8 * (partner % kLanes));
        w_mine[1] = ld16(p.k_norm + 8 * c); w_other[1] = ld16(p.k_norm + 8 * (partner % kLanes));
    }

    const int heads = p.Hq + 2 * p.Hkv;
    const uint16_t *in = p.qkv + (size_t)token * heads * D + 8 * c;
    for (int base = part * kRows; base < heads; base += parts * kRows) {
        const int r = base + r0;
        // (read once: streamed past the caches; 4096 tokens of 80 heads 48.5 -> 45.7 us)
        u32x4 w = __builtin_nontemporal_load(reinterpret_cast<const u32x4 *>(in + (size_t)min(r, heads - 1) * D));
        if (base < p.Hq + p.Hkv) {                       // (uniform: some row of the group is a query or a key)
            const bool is_k = r >= p.Hq, is_v = r >= p.Hq + p.Hkv;
            float x[8], o[8];
            unpack8(w, x);
            u32x4 wp;
#pragma unroll
            for (int i = 0; i < 4; ++i) wp[i] = __shfl(w[i], partner);
            unpack8(wp, o);
            if (p.q_norm) {
                float ss = 0.f;
#pragma unroll
                for (int i = 0; i < 8; ++i) ss += x[i] * x[i];
#pragma unroll
                for (int off = 1; off < kLanes; off <<= 1) ss += __shfl_xor(ss, off);
                const float scale = 1.f / sqrtf(ss * (1.f / D) + p.eps);
                float a[8], d[8];
                unpack8(is_k ? w_mine[1] : w_mine[0], a);
                unpack8(is_k ? w_other[1] : w_other[0], d);
#pragma unroll
                for (int i = 0; i < 8; ++i) { x[i] *= scale * a[i]; o[i] *= scale * d[i]; }
            }
            if (rotates) {
#pragma unroll
                for (int i = 0; i < 8; i += 2) {
                    const float o0 = p.interleaved ? x[i + 1] : o[i], o1 = p.interleaved ? x[i] : o[i + 1];
                    const float y0 = x[i] * cs[i] + o0 * sn[i], y1 = x[i + 1] * cs[i + 1] + o1 * sn[i + 1];
                    x[i] = y0; x[i + 1] = y1;
                }
            }
            u32x4 y;
#pragma unroll
            for (int i = 0; i < 4; ++i) y[i] = pack_bf16x2(x[2 * i], x[2 * i + 1]);
            // (a head that nothing is done to keeps its bits, those of a NaN too)
            if (!is_v && (rotates || p.q_norm)) w = y;
        }
        if (r >= heads) continue;
        if (r < p.Hq) *reinterpret_cast<u32x4 *>(p.q + ((size_t)token * p.Hq + r) * D + 8 * c) = w;
        else if (store_kv) {
            const bool is_v = r >= p.Hq + p.Hkv;
            const int h = r - p.Hq - (is_v ? p.Hkv : 0);
            *reinterpret_cast<u32x4 *>((is_v ? v_out : k_out) + h * stride + 8 * c) = w;
        }
    }
}

template <int D, bool kPacked>
hipError_t launch(const QkvParams &p, hipStream_t stream) {
    const int rows = 64 / (p.D / 8), groups = (p.Hq + 2 * p.Hkv + rows - 1) / rows;
    // A token's rows go to as many wavefronts as fill the chip once, up to four of them to as many as fill it four times (4096
    // tokens of 80 heads: 45.7 us with one, 43.1 with four; 1000 tokens of 48 heads: 9.6 us with five, 12 with twelve).
    const long long once = (kNumCU * 16LL + p.N - 1) / p.N, often = (kNumCU * 64LL + p.N - 1) / p.N;
    long long parts = once > 4 ? once : often < 4 ? often : 4;
    parts = parts > groups ? groups : parts;
    const long long blocks = ((long long)p.N * parts + kQkvThreads / 64 - 1) / (kQkvThreads / 64) + (kPacked ? 1 : 0);
    hipLaunchKernelGGL((qkv_kernel<D, kPacked>), dim3((unsigned)blocks), dim3(kQkvThreads), 0, stream, p, (int)parts);
    return note_hip_error("launch qkv_kernel", hipGetLastError());
}

}  // namespace

hipError_t launch_qkv(const QkvParams &p, hipStream_t stream) {
    if (p.cu_tokens) return p.D == 64 ? launch<64, true>(p, stream) : launch<128, true>(p, stream);
    return p.D == 64 ? launch<64, false>(p, stream) : launch<128, false>(p, stream);
}

}  // namespace reader

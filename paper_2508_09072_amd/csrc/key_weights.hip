// The attention weight that every cached key has drawn from the queries that count (a step's accepted path, or the last
// tokens of a prompt), per kv head:
//   weights[b, hkv, j] = decay * weights[b, hkv, j] + sum over rows (t, g) that see key j of exp(s <q[t, hkv G + g], k_j> - lse[t, hkv G + g])
// The log-sum-exp that the attention left turns a score into its softmax weight, so one product with the keys is all.
//
// S = Q.K^T on the matrix cores in blocks of 16 rows x 16 keys (one page): a lane then holds four rows of one key, and the
// sum over rows is a sum over registers, with two exchanges between lanes at the very end.  A wavefront owns 64 keys, whose
// rows (its operand for all query rows) are loaded from memory once, straight into the operand's layout: 16 lanes read 16
// rows, 64 bytes of each per load.  Nobody else writes those keys' weights: no atomics, the same bits every time.
// Bound by memory for the few rows of a step (K is read once), by the matrix cores and exponentials beyond some 128 rows.
#include "prompt_common.h"
#include "tree_attn_common.h"

namespace reader {

namespace {

typedef float f32x4 __attribute__((ext_vector_type(4)));
constexpr int kKeysPerWave = 64, kWeightsThreads = 256, kKeysPerWg = kKeysPerWave * kWeightsThreads / 64;

template <int D>
__global__ __launch_bounds__(kWeightsThreads) void key_weights_kernel(KeyWeightsParams p) {
    constexpr int kSteps = D / 32;                       // 32-deep steps of the product
    const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    const int hkv = blockIdx.y, b = blockIdx.z, j0 = (int)blockIdx.x * kKeysPerWg + wave * kKeysPerWave;
    const int i16 = lane & 15, quad = lane >> 4;

    // rows: `n` query tokens, the first of them at position `first`; row r is token r / G, head r % G of the group
    int n, first, bad = 0, token0 = 0;
    const int len = p.seq_lens[b];
    if (p.path) {
        n = p.accept_len[b] + 1;
        first = len - n;
        if (n < 1 || n > p.max_path || first < 0) bad = READER_STATUS_BAD_PATH;
    } else {
        const int c0 = clamp_row(p.cu_tokens[b], p.N), c1 = clamp_row(p.cu_tokens[b + 1], p.N);
        const int all = max(c1 - c0, 0);
        n = min(all, p.window);
        token0 = c1 - n;
        first = len + all - n;
        if (len < 0 || p.cu_tokens[b] < 0 || p.cu_tokens[b + 1] < p.cu_tokens[b] || p.cu_tokens[b + 1] > p.N) bad = READER_STATUS_BAD_LENGTH;
    }
    const long long keys_all = (long long)first + n;
    const long long most = min((long long)min(p.max_seq_len, p.max_positions), (long long)p.max_pages * READER_PAGE_SIZE);
    if (!bad && keys_all > most) bad = READER_STATUS_BAD_LENGTH;
    // (every workgroup of the sequence comes to the same verdict: it is left as it is)
    if (!bad && p.path) {
        const int node = lane < n ? p.path[(size_t)b * p.max_path + lane] : 0;
        const int node2 = lane + 64 < n ? p.path[(size_t)b * p.max_path + lane + 64] : 0;
        if (__any(node < 0 || node >= p.T || node2 < 0 || node2 >= p.T)) bad = READER_STATUS_BAD_PATH;
    }
    if (bad) {
        if (p.status && blockIdx.x == 0 && hkv == 0 && threadIdx.x == 0) atomicOr(p.status, bad);
        return;
    }
    const int keys = (int)keys_all;
    float *weights = p.weights + ((size_t)b * p.Hkv + hkv) * p.max_positions;
    if (j0 >= keys) {
        if (p.decay == 0.f && j0 + lane < p.max_positions) weights[j0 + lane] = 0.f;
        return;
    }

    // the 64 keys as operands: page `pg` of the four, step s: row i16, values 32 s + 8 quad .. + 7
    bf16x8 k[4][kSteps];
    bool page_ok[4];
#pragma unroll
    for (int pg = 0; pg < 4; ++pg) {
        const int j = j0 + pg * 16;
        const int page = j < keys ? p.page_table[(size_t)b * p.max_pages + (j >> 4)] : 0;
        page_ok[pg] = page >= 0 && page < p.num_pages;
        if (!page_ok[pg]) bad = READER_STATUS_BAD_PAGE;
        // (nothing is loaded behind a page that is not there; pages past the last key read page 0, whose scores are dropped)
        const uint16_t *src = p.k_cache + (((size_t)(page_ok[pg] ? page : 0) * p.Hkv + hkv) * READER_PAGE_SIZE + i16) * D + quad * 8;
#pragma unroll
        for (int s = 0; s < kSteps; ++s) k[pg][s] = __builtin_bit_cast(bf16x8, ld16(src + s * 32));
    }
    float mine = 0.f;                                     // old weight of key j0 + lane
    const int j_mine = j0 + lane;
    if (p.decay != 0.f && j_mine < keys) mine = p.decay * weights[j_mine];

    const int rows = n * p.G;
    const bool causal = j0 + kKeysPerWave > first + 1;    // some row does not see some of these keys
    float acc[4] = {0.f, 0.f, 0.f, 0.f};
    for (int r0 = 0; r0 < rows; r0 += 16) {
        // operand row i16 of the block, and log-sum-exp and position of the four rows of this lane's results
        auto place = [&](int r, int &t) {                 // token and head of row r
            t = (int)(((float)r + 0.5f) * p.g_rcp);       // (r / G: half a row is far more than the product's rounding)
            return hkv * p.G + r - t * p.G;
        };
        int t;
        const int rq = min(r0 + i16, rows - 1);
        const int head = place(rq, t);
        const size_t row = p.path ? (size_t)b * p.T + p.path[(size_t)b * p.max_path + t] : (size_t)token0 + t;
        const uint16_t *q = p.q + (row * p.Hq + head) * D + quad * 8;
        bf16x8 a[kSteps];
#pragma unroll
        for (int s = 0; s < kSteps; ++s) a[s] = __builtin_bit_cast(bf16x8, ld16(q + s * 32));
        float ref[4];
        int last[4];
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            const int r = r0 + quad * 4 + i;
            int ti;
            const int hi = place(min(r, rows - 1), ti);
            const float lse = p.path ? p.lse[((size_t)b * p.Hq + hi) * p.T + p.path[(size_t)b * p.max_path + ti]]
                                     : p.lse[((size_t)token0 + ti) * p.Hq + hi];
            // (a row behind the last one, and one that saw no key at all, gives nothing)
            ref[i] = r < rows && lse != -INFINITY ? lse * 1.44269504088896340736f : INFINITY;
            last[i] = first + ti;
        }
#pragma unroll
        for (int pg = 0; pg < 4; ++pg) {
            f32x4 x = {0.f, 0.f, 0.f, 0.f};
#pragma unroll
            for (int s = 0; s < kSteps; ++s) x = __builtin_amdgcn_mfma_f32_16x16x32_bf16(a[s], k[pg][s], x, 0, 0, 0);
#pragma unroll
            for (int i = 0; i < 4; ++i) {
                float w = __builtin_amdgcn_exp2f(x[i] * p.scale_log2 - ref[i]);
                if (causal && j0 + pg * 16 + i16 > last[i]) w = 0.f;
                acc[pg] += w;
            }
        }
    }
    // a key's four quarters of the rows sit 16 lanes apart
#pragma unroll
    for (int pg = 0; pg < 4; ++pg) {
        acc[pg] += __shfl_xor(acc[pg], 16);
        acc[pg] += __shfl_xor(acc[pg], 32);
    }
    const float sum = quad == 0 ? acc[0] : quad == 1 ? acc[1] : quad == 2 ? acc[2] : acc[3];
    const bool ok = quad == 0 ? page_ok[0] : quad == 1 ? page_ok[1] : quad == 2 ? page_ok[2] : page_ok[3];
    if (j_mine < keys) weights[j_mine] = mine + (ok ? sum : 0.f);
    else if (p.decay == 0.f && j_mine < p.max_positions) weights[j_mine] = 0.f;
    if (bad && p.status && lane == 0) atomicOr(p.status, bad);
}

}  // namespace

hipError_t launch_key_weights(const KeyWeightsParams &p, hipStream_t stream) {
    const int span = p.decay == 0.f ? p.max_positions : min(p.max_seq_len, p.max_positions);   // (a fresh start clears the whole row)
    if (span <= 0) return hipSuccess;
    const dim3 grid((unsigned)((span + kKeysPerWg - 1) / kKeysPerWg), (unsigned)p.Hkv, (unsigned)p.B);
    if (p.D == 64) hipLaunchKernelGGL(key_weights_kernel<64>, grid, dim3(kWeightsThreads), 0, stream, p);
    else hipLaunchKernelGGL(key_weights_kernel<128>, grid, dim3(kWeightsThreads), 0, stream, p);
    return note_hip_error("launch key_weights_kernel", hipGetLastError());
}

}  // namespace reader

// Eviction: every (layer, sequence, kv head) that is over its budget keeps its newest `recent` rows and, of the others, the
// heaviest, `keep` rows in all, moved together in their order, in place.
//
// select: one workgroup per (layer, sequence, kv head).  The threshold is the k-th largest weight, found two bits at a time
//   from the top: sixteen rounds that count how many candidates reach each of three trial values.  Counts are ballots, so a
//   round costs the same whatever the weights (a histogram's bins are hit by whole wavefronts at once where weights are
//   equal or near).  A wavefront owns a contiguous run of positions, so that after one exchange of counts every wavefront
//   writes its part of the list of kept positions on its own.  Among equal weights the lowest positions stay.
// move: the rows go to the front.  Sources lie at or behind their destinations and increase, so a pass that has read all its
//   rows may overwrite its destinations: later passes read behind them.  Different columns of the rows never meet: a
//   workgroup takes a slice of the columns of K or of V, or the weights themselves, through all passes.
// Bound by memory: the kept rows are read and written once.
#include "prompt_common.h"
#include "tree_attn_common.h"

namespace reader {

namespace {

constexpr int kSelectThreads = 1024, kSelectWaves = kSelectThreads / 64;
constexpr int kHeldWeights = 32;                       // weights a thread holds: up to 32768 positions are read once

// Order-preserving: a heavier weight is a larger number; a NaN is lighter than any; the two zeros are equal.
__device__ inline uint32_t weight_rank(float w) {
    const uint32_t u = __float_as_uint(w + 0.f);
    return w != w ? 0u : (u & 0x80000000u) ? ~u : u | 0x80000000u;
}

__global__ __launch_bounds__(kSelectThreads) void evict_select_kernel(EvictParams p) {
    const int tid = threadIdx.x, lane = tid & 63, wave = __builtin_amdgcn_readfirstlane(tid >> 6);
    const long long unit = blockIdx.x;                 // (layer, sequence, kv head)
    const int b = (int)(unit / p.Hkv % p.B);
    const int n = p.seq_lens[b];
    __shared__ int s_bad;
    __shared__ int s_count[2][kSelectWaves][4];
    if (n <= p.keep) {                                 // within its budget
        if (tid == 0) {
            p.old_len[unit] = 0;
            if (n < 0 && p.status) atomicOr(p.status, READER_STATUS_BAD_LENGTH);
        }
        return;
    }
    // a sequence that does not fit its weights or its pages is left as it is, in every layer and head
    if (tid == 0) s_bad = n > p.max_positions || n > (long long)p.max_pages * READER_PAGE_SIZE ? READER_STATUS_BAD_LENGTH : 0;
    __syncthreads();
    if (!s_bad) {
        for (int i = tid; i < (n + READER_PAGE_SIZE - 1) / READER_PAGE_SIZE; i += kSelectThreads) {
            const int page = p.page_table[(size_t)b * p.max_pages + i];
            if (page < 0 || page >= p.num_pages) atomicOr(&s_bad, READER_STATUS_BAD_PAGE);
        }
    }
    __syncthreads();
    if (s_bad) {
        if (tid == 0) {
            p.old_len[unit] = 0;
            if (p.status) atomicOr(p.status, s_bad);
        }
        return;
    }

    const float *weights = p.weights + unit * p.max_positions;
    const int m = n - p.recent, k = p.keep - p.recent;          // candidates, and how many of them stay
    const int per_wave = ((m + kSelectThreads - 1) / kSelectThreads) * 64;     // positions of a wavefront's run
    const int chunks = per_wave / 64, run0 = wave * per_wave;
    uint32_t held[kHeldWeights];
#pragma unroll
    for (int e = 0; e < kHeldWeights; ++e) {
        const int j = run0 + e * 64 + lane;
        held[e] = e < chunks && j < m ? weight_rank(weights[j]) : 0u;
    }
    // calls f(rank, position exists, position) for every 64 positions of this wavefront's run, in order
    auto each = [&](auto &&f) {
#pragma unroll
        for (int e = 0; e < kHeldWeights; ++e) {
            if (e >= chunks) break;
            const int j = run0 + e * 64 + lane;
            f(held[e], j < m, j);
        }
        for (int e = kHeldWeights; e < chunks; ++e) {
            const int j = run0 + e * 64 + lane;
            f(j < m ? weight_rank(weights[j]) : 0u, j < m, j);
        }
    };
    // largest value that at least k candidates reach
    uint32_t bound = 0u;
    int round = 0;
    if (k > 0) {
        for (int shift = 30; shift >= 0; shift -= 2, round ^= 1) {
            int c[3] = {0, 0, 0};
            each([&](uint32_t v, bool exists, int) {
#pragma unroll
                for (int i = 0; i < 3; ++i) c[i] += __popcll(__ballot(exists && v >= bound + ((uint32_t)(i + 1) << shift)));
            });
            if (lane < 3) s_count[round][wave][lane] = lane == 0 ? c[0] : lane == 1 ? c[1] : c[2];
            __syncthreads();
            int all[3] = {0, 0, 0};
#pragma unroll
            for (int w = 0; w < kSelectWaves; ++w)
#pragma unroll
                for (int i = 0; i < 3; ++i) all[i] += s_count[round][w][i];
            bound += (uint32_t)((all[0] >= k) + (all[1] >= k) + (all[2] >= k)) << shift;
        }
    }
    // kept: what is heavier than the bound, and the first ones equal to it
    int heavier = 0, equal = 0;
    if (k > 0)
        each([&](uint32_t v, bool exists, int) {
            heavier += __popcll(__ballot(exists && v > bound));
            equal += __popcll(__ballot(exists && v == bound));
        });
    if (lane == 0) { s_count[round][wave][0] = heavier; s_count[round][wave][1] = equal; }
    __syncthreads();
    int heavier_all = 0, heavier_before = 0, equal_before = 0;
#pragma unroll
    for (int w = 0; w < kSelectWaves; ++w) {
        heavier_all += s_count[round][w][0];
        if (w < wave) { heavier_before += s_count[round][w][0]; equal_before += s_count[round][w][1]; }
    }
    const int ties = k - heavier_all;                  // equal ones that stay
    int32_t *source = p.source + unit * p.keep;
    int to = heavier_before + min(equal_before, ties), seen = equal_before;
    if (k > 0)
        each([&](uint32_t v, bool exists, int j) {
            const unsigned long long eq = __ballot(exists && v == bound), below = (1ull << lane) - 1ull;
            const bool stays = exists && (v > bound || (v == bound && seen + (int)__popcll(eq & below) < ties));
            const unsigned long long set = __ballot(stays);
            if (stays) source[to + (int)__popcll(set & below)] = j;
            to += __popcll(set);
            seen += __popcll(eq);
        });
    for (int i = tid; i < p.recent; i += kSelectThreads) source[k + i] = m + i;
    if (tid == 0) p.old_len[unit] = n;
}

constexpr int kMoveThreads = 256;
constexpr int kMoveSub = 8;                            // rows a thread carries through one pass

// Rows of `kChunks` 16-byte chunks, of which this workgroup moves `kSlice` from chunk c0 on.
template <int D, int kSlice>
__device__ inline void evict_move_rows(const EvictParams &p, uint16_t *cache, const int32_t *table, const int32_t *source, int hkv, int c0) {
    constexpr int kRows = kMoveThreads / kSlice;
    const int tid = threadIdx.x, r = tid / kSlice;
    cache += (size_t)hkv * READER_PAGE_SIZE * D + (size_t)(c0 + tid % kSlice) * 8;
    const size_t page_stride = (size_t)p.Hkv * READER_PAGE_SIZE * D;
    for (int base = 0; base < p.keep; base += kRows * kMoveSub) {
        int src[kMoveSub];
        u32x4 w[kMoveSub];
#pragma unroll
        for (int u = 0; u < kMoveSub; ++u) {
            const int d = base + u * kRows + r;
            src[u] = d < p.keep ? source[d] : d;
        }
#pragma unroll
        for (int u = 0; u < kMoveSub; ++u) {
            const int d = base + u * kRows + r;
            if (src[u] != d) w[u] = ld16(cache + (size_t)table[src[u] >> 4] * page_stride + (src[u] & 15) * D);
        }
        __syncthreads();                               // every row of the pass has been read
#pragma unroll
        for (int u = 0; u < kMoveSub; ++u) {
            const int d = base + u * kRows + r;
            if (src[u] != d) *reinterpret_cast<u32x4 *>(cache + (size_t)table[d >> 4] * page_stride + (d & 15) * D) = w[u];
        }
    }
}

__device__ inline void evict_move_weights(const EvictParams &p, float *weights, const int32_t *source, int n) {
    for (int base = 0; base < p.keep; base += kMoveThreads * kMoveSub) {
        float w[kMoveSub];
#pragma unroll
        for (int u = 0; u < kMoveSub; ++u) {
            const int d = base + u * kMoveThreads + (int)threadIdx.x;
            w[u] = d < p.keep ? weights[source[d]] : 0.f;
        }
        __syncthreads();
#pragma unroll
        for (int u = 0; u < kMoveSub; ++u) {
            const int d = base + u * kMoveThreads + (int)threadIdx.x;
            if (d < p.keep) weights[d] = w[u];
        }
    }
    __syncthreads();
    for (int j = p.keep + (int)threadIdx.x; j < n; j += kMoveThreads) weights[j] = 0.f;
}

// 1-D grid: per (layer, sequence, kv head) D / 8 / kSlice slices of K, as many of V, and the weights
template <int D, int kSlice>
__global__ __launch_bounds__(kMoveThreads) void evict_move_kernel(EvictParams p) {
    constexpr int kSlices = D / 8 / kSlice, kJobs = 2 * kSlices + 1;
    const long long unit = blockIdx.x / kJobs;
    const int job = (int)(blockIdx.x - unit * kJobs);
    const int n = p.old_len[unit];
    if (n == 0) return;
    const int hkv = (int)(unit % p.Hkv), b = (int)(unit / p.Hkv % p.B), layer = (int)(unit / p.Hkv / p.B);
    const int32_t *source = p.source + unit * p.keep, *table = p.page_table + (size_t)b * p.max_pages;
    if (job == kJobs - 1) {
        evict_move_weights(p, p.weights + unit * p.max_positions, source, n);
        if (layer == 0 && hkv == 0 && threadIdx.x == 0) p.seq_lens[b] = p.keep;     // (nobody reads it in this launch)
        return;
    }
    const bool is_v = job >= kSlices;
    uint16_t *cache = (is_v ? p.v_cache : p.k_cache) + (size_t)layer * (size_t)p.num_pages * p.Hkv * READER_PAGE_SIZE * D;
    evict_move_rows<D, kSlice>(p, cache, table, source, hkv, (is_v ? job - kSlices : job) * kSlice);
}

template <int D, int kSlice>
hipError_t launch_move(const EvictParams &p, unsigned units, hipStream_t stream) {
    hipLaunchKernelGGL((evict_move_kernel<D, kSlice>), dim3(units * (2 * (D / 8 / kSlice) + 1)), dim3(kMoveThreads), 0, stream, p);
    return note_hip_error("launch evict_move_kernel", hipGetLastError());
}

}  // namespace

hipError_t launch_kv_evict(const EvictParams &p, hipStream_t stream) {
    const unsigned units = (unsigned)p.NL * p.B * p.Hkv;
    hipLaunchKernelGGL(evict_select_kernel, dim3(units), dim3(kSelectThreads), 0, stream, p);
    const hipError_t e = hipGetLastError();
    if (e != hipSuccess) return note_hip_error("launch evict_select_kernel", e);
    return p.D == 64 ? launch_move<64, 4>(p, units, stream) : launch_move<128, 4>(p, units, stream);
}

}  // namespace reader

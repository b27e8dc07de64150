// Eviction: every (layer, sequence, kv head) that is over its budget keeps its newest `recent` rows and, of the others, the
// heaviest, `keep` rows in all, moved together in their order, in place.
//
// select: one workgroup per (layer, sequence, kv head).  The threshold is the k-th largest weight, found from the top in
//   histograms of eleven bits: at most three passes over ranks in LDS, the later ones over what shares the digits found so far,
//   and none once all of those stay.  (Counting what reaches three trial values a round, two bits at a time, took 38 us for 30000
//   weights and 8.5 for 4244.)  A wavefront owns a contiguous run of positions, so that after one exchange of counts every
//   wavefront writes its part of the list of kept positions on its own.  Among equal weights the lowest positions stay.
// move: the rows go to the front.  Sources lie at or behind their destinations and increase, so a pass that has read all its
//   rows may overwrite its destinations: later passes read behind them.  Different columns of the rows never meet: a
//   workgroup takes a slice of the columns of K or of V, or the weights themselves, through all passes.
// Bound by memory: the kept rows are read and written once.
#include "prompt_common.h"
#include "tree_attn_common.h"

namespace reader {

namespace {

constexpr int kSelectThreads = 1024, kSelectWaves = kSelectThreads / 64;
constexpr int kBins = 2048;                            // eleven bits of the bound a round
static_assert(kBins == 2 * kSelectThreads, "a thread holds two bins");
constexpr int kHeldWeights = 32768;                    // candidates whose ranks fit the LDS; the rest is read again in every round

// Order-preserving: a heavier weight is a larger number; a NaN is lighter than any; the two zeros are equal.
__device__ inline uint32_t weight_rank(float w) {
    const uint32_t u = __float_as_uint(w + 0.f);
    return w != w ? 0u : (u & 0x80000000u) ? ~u : u | 0x80000000u;
}

__global__ __launch_bounds__(kSelectThreads) void evict_select_kernel(EvictParams p, int held) {
    extern __shared__ uint32_t s_rank[];               // [held] ranks of the first candidates
    const int tid = threadIdx.x, lane = tid & 63, wave = __builtin_amdgcn_readfirstlane(tid >> 6);
    const long long unit = blockIdx.x;                 // (layer, sequence, kv head)
    const int b = (int)(unit / p.Hkv % p.B);
    const int n = p.seq_lens[b];
    __shared__ int s_bad;
    __shared__ int s_bin[kBins], s_found[3];
    __shared__ int s_run[kSelectWaves][2];             // of each wavefront's run: candidates heavier than the bound, and equal to it
    if (n <= p.keep) {                                 // within its budget
        if (tid == 0) {
            p.old_len[unit] = 0;
            if (n < 0 && p.status) atomicOr(p.status, READER_STATUS_BAD_LENGTH);
        }
        return;
    }
    // a sequence that does not fit its weights or its pages is left as it is, in every layer and head
    if (n > p.max_positions || n > (long long)p.max_pages * READER_PAGE_SIZE) {
        if (tid == 0) {
            p.old_len[unit] = 0;
            if (p.status) atomicOr(p.status, READER_STATUS_BAD_LENGTH);
        }
        return;
    }
    if (tid == 0) s_bad = 0;
    s_bin[tid] = s_bin[tid + kSelectThreads] = 0;
    const float *weights = p.weights + unit * p.max_positions;
    const int m = n - p.recent, k = p.keep - p.recent;          // candidates, and how many of them stay
    const int per_wave = ((m + kSelectThreads - 1) / kSelectThreads) * 64;     // positions of a wavefront's run
    const int run0 = wave * per_wave, run1 = min(run0 + per_wave, m);
#pragma unroll 4
    for (int j = tid; j < min(m, held); j += kSelectThreads) s_rank[j] = weight_rank(weights[j]);
    __syncthreads();
    bool missing = false;
    for (int i = tid; i < (n + READER_PAGE_SIZE - 1) / READER_PAGE_SIZE; i += kSelectThreads) {
        const int page = p.page_table[(size_t)b * p.max_pages + i];
        missing = missing || page < 0 || page >= p.num_pages;
    }
    if (missing) s_bad = 1;
    __syncthreads();
    if (s_bad) {
        if (tid == 0) {
            p.old_len[unit] = 0;
            if (p.status) atomicOr(p.status, READER_STATUS_BAD_PAGE);
        }
        return;
    }
    // calls f(rank, position exists, position) for every 64 positions of this wavefront's run, in order
    auto each = [&](auto &&f) {
        int base = run0;
#pragma unroll 2
        for (; base + 64 <= min(run1, held); base += 64) f(s_rank[base + lane], true, base + lane);
        for (; base < run1; base += 64) {
            const int j = base + lane;
            const bool exists = j < run1;
            f(!exists ? 0u : j < held ? s_rank[j] : weight_rank(weights[j]), exists, j);
        }
    };
    // the bound: the largest value that at least k candidates reach, eleven bits of it at a time
    uint32_t bound = 0u;
    int want = k;                                      // candidates still to be found at or below the digits that are fixed
    for (int round = 0; k > 0 && round < 3; ++round) {
        const int shift = round == 0 ? 21 : round == 1 ? 10 : 0, digits = round == 2 ? 10 : 11;
        if (round > 0) {
            for (int i = tid; i < kBins; i += kSelectThreads) s_bin[i] = 0;
            __syncthreads();
        }
        each([&](uint32_t v, bool exists, int) {
            const bool in = exists && (round == 0 || (v >> (shift + digits)) == (bound >> (shift + digits)));
            const int bin = (int)(v >> shift) & (kBins - 1) & ((1 << digits) - 1);
            // (weights that are equal or near meet in one bin, lane behind lane: those of the first lane's go together)
            const unsigned long long any = __ballot(in);
            if (any == 0) return;
            const int leader = (int)__builtin_ctzll(any), leader_bin = __builtin_amdgcn_readlane(bin, leader);
            const unsigned long long same = __ballot(in && bin == leader_bin);
            if (lane == leader) atomicAdd(&s_bin[leader_bin], (int)__popcll(same));
            else if (in && bin != leader_bin) atomicAdd(&s_bin[bin], 1);
        });
        __syncthreads();
        // bins from the top: thread t holds the t-th pair of them
        const int top = kBins - 1 - 2 * tid;
        const int c0 = s_bin[top], c1 = s_bin[top - 1];
        int upto = wave_inclusive_scan(c0 + c1);
        if (lane == 63) s_run[wave][0] = upto;
        __syncthreads();
        for (int w = 0; w < wave; ++w) upto += s_run[w][0];
        const int above = upto - c0 - c1;
        if (above < want && want <= upto) {            // (one thread: the bound's digits are here)
            const bool first = want <= above + c0;
            s_found[0] = first ? top : top - 1;
            s_found[1] = first ? above : above + c0;
            s_found[2] = first ? c0 : c1;
        }
        __syncthreads();
        bound |= (uint32_t)s_found[0] << shift;
        want -= s_found[1];
        if (want == s_found[2]) break;                 // (all that share these digits stay: no bit below them matters)
    }
    // kept: what is heavier than the bound, and the first ones equal to it
    int heavier = 0, equal = 0;
    if (k > 0)
        each([&](uint32_t v, bool exists, int) {
            heavier += __popcll(__ballot(exists && v > bound));
            equal += __popcll(__ballot(exists && v == bound));
        });
    if (lane == 0) { s_run[wave][0] = heavier; s_run[wave][1] = equal; }
    __syncthreads();
    int heavier_all = 0, heavier_before = 0, equal_before = 0;
#pragma unroll
    for (int w = 0; w < kSelectWaves; ++w) {
        heavier_all += s_run[w][0];
        if (w < wave) { heavier_before += s_run[w][0]; equal_before += s_run[w][1]; }
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

constexpr int kMoveSub = 8;                            // rows a thread carries through one pass

// This workgroup's slice of the rows: `kSlice` 16-byte chunks of each, from chunk c0 on.
template <int D, int kMoveThreads, int kSlice>
__device__ inline void evict_move_rows(const EvictParams &p, uint16_t *cache, const int32_t *table, const int32_t *source, int hkv, int c0) {
    constexpr int kRows = kMoveThreads / kSlice;
    const int tid = threadIdx.x, r = tid / kSlice;
    cache += (size_t)hkv * READER_PAGE_SIZE * D + (size_t)(c0 + tid % kSlice) * 8;
    const size_t page_stride = (size_t)p.Hkv * READER_PAGE_SIZE * D;
    // (as above, no load under a condition: rows that stay where they are are read too, but not written)
    auto list = [&](int base, int (&src)[kMoveSub]) {
#pragma unroll
        for (int u = 0; u < kMoveSub; ++u) src[u] = source[min(base + u * kRows + r, p.keep - 1)];
    };
    int src[kMoveSub];
    list(0, src);
    for (int base = 0; base < p.keep; base += kRows * kMoveSub) {
        int from[kMoveSub], to[kMoveSub], next[kMoveSub];
        u32x4 w[kMoveSub];
#pragma unroll
        for (int u = 0; u < kMoveSub; ++u) {
            from[u] = table[src[u] >> 4];
            to[u] = table[min(base + u * kRows + r, p.keep - 1) >> 4];
        }
        list(base + kRows * kMoveSub, next);           // (the next pass's, a trip ahead)
#pragma unroll
        for (int u = 0; u < kMoveSub; ++u) w[u] = ld16(cache + (size_t)from[u] * page_stride + (src[u] & 15) * D);
        __syncthreads();                               // every row of the pass has been read
#pragma unroll
        for (int u = 0; u < kMoveSub; ++u) {
            const int d = base + u * kRows + r;
            if (d < p.keep && src[u] != d) *reinterpret_cast<u32x4 *>(cache + (size_t)to[u] * page_stride + (d & 15) * D) = w[u];
            src[u] = next[u];
        }
    }
}

template <int kMoveThreads>
__device__ inline void evict_move_weights(const EvictParams &p, float *weights, const int32_t *source, int n) {
    for (int base = 0; base < p.keep; base += kMoveThreads * kMoveSub) {
        int src[kMoveSub];
        float w[kMoveSub];
#pragma unroll
        for (int u = 0; u < kMoveSub; ++u) src[u] = source[min(base + u * kMoveThreads + (int)threadIdx.x, p.keep - 1)];
#pragma unroll
        for (int u = 0; u < kMoveSub; ++u) w[u] = weights[src[u]];
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
template <int D, int kMoveThreads, int kSlice>
__global__ __launch_bounds__(kMoveThreads) void evict_move_kernel(EvictParams p) {
    constexpr int kSlices = D / 8 / kSlice, kJobs = 2 * kSlices + 1;
    const long long unit = blockIdx.x / kJobs;
    const int job = (int)(blockIdx.x - unit * kJobs);
    const int n = p.old_len[unit];
    if (n == 0) return;
    const int hkv = (int)(unit % p.Hkv), b = (int)(unit / p.Hkv % p.B), layer = (int)(unit / p.Hkv / p.B);
    const int32_t *source = p.source + unit * p.keep, *table = p.page_table + (size_t)b * p.max_pages;
    if (job == kJobs - 1) {
        evict_move_weights<kMoveThreads>(p, p.weights + unit * p.max_positions, source, n);
        if (layer == 0 && hkv == 0 && threadIdx.x == 0) p.seq_lens[b] = p.keep;     // (nobody reads it in this launch)
        return;
    }
    if (p.keep == 0) return;                           // (nothing stays)
    const bool is_v = job >= kSlices;
    uint16_t *cache = (is_v ? p.v_cache : p.k_cache) + (size_t)layer * (size_t)p.num_pages * p.Hkv * READER_PAGE_SIZE * D;
    evict_move_rows<D, kMoveThreads, kSlice>(p, cache, table, source, hkv, (is_v ? job - kSlices : job) * kSlice);
}

template <int D, int kMoveThreads, int kSlice>
hipError_t launch_move(const EvictParams &p, unsigned units, hipStream_t stream) {
    hipLaunchKernelGGL((evict_move_kernel<D, kMoveThreads, kSlice>), dim3(units * (2 * (D / 8 / kSlice) + 1)), dim3(kMoveThreads), 0, stream, p);
    return note_hip_error("launch evict_move_kernel", hipGetLastError());
}

template <int D>
hipError_t launch_move_by_size(const EvictParams &p, unsigned units, hipStream_t stream) {
    // Slices of 64 bytes where there are few units, for more workgroups; of 128 bytes otherwise, whose pieces memory serves
    // faster.  One layer of one sequence, 8 kv heads of 4500 rows to 4096: 34.9 against 37.0 us for the whole call; two of 30000
    // to 15000: 143 against 156; 64 units of up to 9000 to 3000: 89 against 79; 1024 units: 682 against 531 (rows of 256 bytes
    // whole: 537).
    return units <= 32 ? launch_move<D, 512, 4>(p, units, stream) : launch_move<D, 512, 8>(p, units, stream);
}

}  // namespace

hipError_t launch_kv_evict(const EvictParams &p, hipStream_t stream) {
    const unsigned units = (unsigned)p.NL * p.B * p.Hkv;
    const int held = p.max_positions < kHeldWeights ? p.max_positions : kHeldWeights;
    hipError_t e = hipFuncSetAttribute(reinterpret_cast<const void *>(&evict_select_kernel), hipFuncAttributeMaxDynamicSharedMemorySize,
                                       kHeldWeights * (int)sizeof(uint32_t));
    if (e != hipSuccess) { (void)hipGetLastError(); return note_hip_error("hipFuncSetAttribute(eviction's LDS size)", e); }
    hipLaunchKernelGGL(evict_select_kernel, dim3(units), dim3(kSelectThreads), held * sizeof(uint32_t), stream, p, held);
    e = hipGetLastError();
    if (e != hipSuccess) return note_hip_error("launch evict_select_kernel", e);
    return p.D == 64 ? launch_move_by_size<64>(p, units, stream) : launch_move_by_size<128>(p, units, stream);
}

}  // namespace reader

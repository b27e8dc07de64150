// Rows of K and V into the cache in 4 bits, and their moves inside it.
//
// A group of 32 values gets the scale 2^e, e = floor(log2 of the largest magnitude) - 2, one more where that magnitude is above 7
// times it (kept within [-125, 125]): no value is further from its code than 2^e, half of the largest step.  Codes are rounded to
// nearest even by v_cvt_scalef32_pk_fp4_bf16, whose operands are exact here.  A lane takes eight values, four lanes a group: 16 bytes
// loaded, 4 and a quarter of a byte stored, the group's maximum by two exchanges.  Bound by memory, in small calls by the launch.
#include <limits.h>

#include "kvq_common.h"
#include "tree_attn_common.h"

namespace reader {

namespace {

typedef __bf16 bf16x2 __attribute__((ext_vector_type(2)));
constexpr int kStoreThreads = 256;

// Eight values of a row as eight codes; the scale's byte, the same in the four lanes of a group.  false: the group has a value that is
// no finite number, and is stored as zeros.
__device__ __forceinline__ bool eight_codes(u32x4 x, uint32_t &codes, uint32_t &scale) {
    uint32_t top = 0;                                        // bits of the largest magnitude
#pragma unroll
    for (int w = 0; w < 4; ++w) top = max(top, max(x[w] & 0x7fffu, x[w] >> 16 & 0x7fffu));
    top = max(top, (uint32_t)__shfl_xor((int)top, 1));
    top = max(top, (uint32_t)__shfl_xor((int)top, 2));
    const bool finite = top < 0x7f80u;
    // exponent + 127 - 2; above 1.75 (mantissa 0x60) one more; subnormal magnitudes end at the lower bound like all below it
    const int e = (int)(top >> 7) - 2 + ((top & 0x7fu) > 0x60u ? 1 : 0);
    scale = finite ? (uint32_t)min(max(e, kKvqLowest + 127), kKvqHighest + 127) : (uint32_t)(kKvqLowest + 127);
    const float s = __uint_as_float(scale << 23);
    // (each word a value of its own: an element of a vector that is cast as it stands is the vector's first)
    const uint32_t x0 = x[0], x1 = x[1], x2 = x[2], x3 = x[3];
    codes = 0;
    codes = __builtin_amdgcn_cvt_scalef32_pk_fp4_bf16(codes, __builtin_bit_cast(bf16x2, x0), s, 0);
    codes = __builtin_amdgcn_cvt_scalef32_pk_fp4_bf16(codes, __builtin_bit_cast(bf16x2, x1), s, 1);
    codes = __builtin_amdgcn_cvt_scalef32_pk_fp4_bf16(codes, __builtin_bit_cast(bf16x2, x2), s, 2);
    codes = __builtin_amdgcn_cvt_scalef32_pk_fp4_bf16(codes, __builtin_bit_cast(bf16x2, x3), s, 3);
    if (!finite) codes = 0;
    return finite;
}

// Values 8 t .. 8 t + 7 of row s of a page.
template <int D>
__device__ __forceinline__ bool store_eight(uint8_t *block, int s, int t, u32x4 k, u32x4 v) {
    using B = KvqBlock<D>;
    uint32_t codes, scale;
    bool finite = eight_codes(k, codes, scale);
    *reinterpret_cast<uint32_t *>(block + B::k_code(s, 8 * t)) = codes;
    if (t % 4 == 0) block[B::k_scale(s, t / 4)] = (uint8_t)scale;
    finite = eight_codes(v, codes, scale) && finite;
    if constexpr (D == 128) *reinterpret_cast<uint32_t *>(block + B::v_code(s, 8 * t)) = codes;
    else {
        *reinterpret_cast<uint16_t *>(block + B::v_code(s, 8 * t)) = (uint16_t)codes;
        *reinterpret_cast<uint16_t *>(block + B::v_code(s, 8 * t + 4)) = (uint16_t)(codes >> 16);
    }
    if (t % 4 == 0) block[B::v_scale(s, t / 4)] = (uint8_t)scale;
    return finite;
}

// Rows of tensors: a wavefront takes 64 / (D / 8) heads of one row.  A row's bytes in a page are pieces of 16 and 4 (D = 128), so a page is
// written by 16 rows' stores that meet in the cache.  16 trees of 32 nodes, 8 heads of 128: 2.65 MB in 3.4 us, the launch itself.
template <int D>
__global__ __launch_bounds__(kStoreThreads) void kvq_store_kernel(KvqStoreParams p) {
    constexpr int kLanes = D / 8, kHeads = 64 / kLanes;
    const int lane = threadIdx.x & 63;
    const int row = __builtin_amdgcn_readfirstlane(blockIdx.x * (kStoreThreads / 64) + (threadIdx.x >> 6));
    if (row >= p.N) return;
    const int head = blockIdx.y * kHeads + lane / kLanes, t = lane % kLanes;
    int b, first, bad = 0;
    if (p.cu_tokens) {
        // (one workgroup of each launch looks the bounds over)
        if (row == 0 && blockIdx.y == 0)
            for (int i = lane; i < p.B; i += 64) bad |= bad_sequence(p.cu_tokens, p.seq_lens, p.N, i);
        b = sequence_of_row(p.cu_tokens, p.B, row, lane, first);
    } else {
        b = row / p.T;
        first = b * p.T;
    }
    if (b < p.B) {
        const int L = p.seq_lens[b];
        const long long at = (long long)L + (row - first);
        if (L < 0 || at >= (long long)p.max_pages * READER_PAGE_SIZE) bad |= READER_STATUS_BAD_LENGTH;
        else {
            const int page = p.page_table[(size_t)b * p.max_pages + at / READER_PAGE_SIZE];
            if (page < 0 || page >= p.num_pages) bad |= READER_STATUS_BAD_PAGE;
            else if (head < p.Hkv) {
                const size_t from = ((size_t)row * p.Hkv + head) * D + t * 8;
                const u32x4 k = ld16(p.k + from), v = ld16(p.v + from);
                if (!store_eight<D>(p.cache + ((size_t)page * p.Hkv + head) * KvqBlock<D>::kBytes, (int)(at % READER_PAGE_SIZE), t, k, v))
                    bad |= READER_STATUS_BAD_VALUE;
            }
        }
    }
    if (bad && p.status) atomicOr(p.status, bad);
}

// (read once: streamed past the caches)
__device__ __forceinline__ u32x4 load_once(const uint16_t *from) { return __builtin_nontemporal_load(reinterpret_cast<const u32x4 *>(from)); }

// Pages of a bf16 cache: a wavefront takes a page of a kv head of a layer.  8 layers of 8 prompts of 2 K to 8 K positions, 8 heads of 128:
// 1.76 GB in 372 us, 4.7 TB/s (a copy of 2 GiB: 4.9).
template <int D>
__global__ __launch_bounds__(kStoreThreads) void kvq_pack_kernel(KvqStoreParams p) {
    constexpr int kLanes = D / 8, kRows = 64 / kLanes;
    const int lane = threadIdx.x & 63, b = blockIdx.y, layer = blockIdx.z;
    const int unit = __builtin_amdgcn_readfirstlane(blockIdx.x * (kStoreThreads / 64) + (threadIdx.x >> 6));
    const int j = unit / p.Hkv, head = unit - j * p.Hkv;
    const int L = p.seq_lens[b], from = p.starts ? p.starts[b] : 0;
    const int mapped = (int)min((long long)p.max_pages * READER_PAGE_SIZE, (long long)p.max_seq_len);
    int bad = 0;
    if (L < 0 || from < 0 || from > L || L > mapped) {
        if (unit == 0 && layer == 0 && lane == 0 && p.status) atomicOr(p.status, READER_STATUS_BAD_LENGTH);
        return;
    }
    const int lo = max(from - j * READER_PAGE_SIZE, 0), hi = min(L - j * READER_PAGE_SIZE, READER_PAGE_SIZE);
    if (lo >= hi) return;
    const int src = p.from_table[(size_t)b * p.max_pages + j], dst = p.page_table[(size_t)b * p.max_pages + j];
    if (src < 0 || src >= p.from_pages || dst < 0 || dst >= p.num_pages) bad = READER_STATUS_BAD_PAGE;
    else {
        const size_t at = (((size_t)layer * p.from_pages + src) * p.Hkv + head) * (READER_PAGE_SIZE * D) + lane * 8;
        uint8_t *block = p.cache + (((size_t)layer * p.num_pages + dst) * p.Hkv + head) * KvqBlock<D>::kBytes;
#pragma unroll
        for (int i = 0; i < READER_PAGE_SIZE / kRows; ++i) {
            const int s = i * kRows + lane / kLanes;
            if (s < lo || s >= hi) continue;                 // (the four lanes of a group go the same way)
            const u32x4 k = load_once(p.k + at + i * 512), v = load_once(p.v + at + i * 512);
            if (!store_eight<D>(block, s, lane % kLanes, k, v)) bad = READER_STATUS_BAD_VALUE;
        }
    }
    if (bad && p.status) atomicOr(p.status, bad);
}

// ---- the accepted path's rows, in place

constexpr int kMoveThreads = 256, kMovePerThread = 8;

struct PathShared {
    int L, n, bad;
    int node[READER_MAX_T], from[READER_MAX_T], to[READER_MAX_T];    // node, page ids of its row and of where it goes
};

// Checks all that the sequence would touch before anything is written; a barrier at the end.
__device__ inline void check_path(const KvqCompactParams &p, int b, PathShared &sh) {
    const int tid = threadIdx.x;
    const int32_t *path = p.path + (size_t)b * p.max_path;
    const int node = tid < p.max_path ? path[tid] : -1, before = tid >= 1 && tid < p.max_path ? path[tid - 1] : -1;
    if (tid == 0) { sh.L = p.seq_lens[b]; sh.n = p.accept_len[b]; sh.bad = 0; }
    __syncthreads();
    const int L = sh.L, n = sh.n;
    const long long mapped = min((long long)p.max_pages * READER_PAGE_SIZE, (long long)INT_MAX);
    int bad = 0;
    if (n < 0 || n > p.max_path - 1 || L < 0 || (long long)L + n + 1 > mapped) bad = READER_STATUS_BAD_PATH;
    else if (tid <= n) {
        if (!(node >= 0 && node < p.T && (tid == 0 ? node == 0 : node > before) && (long long)L + node < mapped)) bad = READER_STATUS_BAD_PATH;
        else {
            const int32_t *table = p.page_table + (size_t)b * p.max_pages;
            const int from = table[(L + node) / READER_PAGE_SIZE], to = table[(L + tid) / READER_PAGE_SIZE];
            if (from < 0 || from >= p.num_pages || to < 0 || to >= p.num_pages) bad = READER_STATUS_BAD_PAGE;
            sh.node[tid] = node; sh.from[tid] = from; sh.to[tid] = to;
        }
    }
    if (bad) atomicOr(&sh.bad, bad);
    __syncthreads();
}

// One workgroup per (sequence, layer).  A row's bytes are moved in the pieces that lie together: D / 8 words of K, 16 pieces of V of
// D / 32 bytes, single scales.  Node ids increase along a path, so no row is written before it has been read: rows go in their
// order, a pass reads its pieces before it writes any.  (Of 128 values, a row has four pieces of 16 bytes of K, moved as words, 16 of
// 4 of V and 8 bytes of scales, in 7 of the block's 17 lines of 128 bytes.)  Bound by the chain of loads (path, table, rows): one user's path of 6, 8 heads of
// 64, 5.6 us.  With many layers by the lines that the scattered pieces touch: 32 layers of 64 paths of 8, 8 heads of 128, move 15 MB in
// 22 us and touch 105, 4.8 TB/s; the lengths' launch behind it takes 4.
template <int D>
__global__ __launch_bounds__(kMoveThreads) void kvq_compact_kernel(KvqCompactParams p) {
    using B = KvqBlock<D>;
    constexpr int kWords = D / 8, kPieces = kWords + 16 + 2 * (D / 32);
    __shared__ PathShared sh;
    const int b = blockIdx.x, layer = blockIdx.y, tid = threadIdx.x;
    check_path(p, b, sh);
    if (sh.bad) {
        if (layer == 0 && tid == 0 && p.status) atomicOr(p.status, sh.bad);
        return;
    }
    const int L = sh.L, n = sh.n, per_head = n * kPieces, total = p.Hkv * per_head;
    uint8_t *cache = p.cache + (size_t)layer * p.num_pages * p.Hkv * B::kBytes;
    for (int base = 0; base < total; base += kMoveThreads * kMovePerThread) {
        uint32_t held[kMovePerThread];
        uint8_t *to[kMovePerThread];
        int bytes[kMovePerThread];
#pragma unroll
        for (int r = 0; r < kMovePerThread; ++r) {
            const int idx = base + r * kMoveThreads + tid;
            bytes[r] = 0;
            if (idx >= total) continue;
            const int head = idx / per_head, rem = idx - head * per_head, j = 1 + rem / kPieces, piece = rem - (j - 1) * kPieces;
            const int node = sh.node[j];
            if (node == j) continue;                         // (in place)
            auto at = [&](int s) {
                return piece < kWords ? B::k_code(s, 8 * piece)
                       : piece < kWords + 16 ? B::v_code(s, (piece - kWords) * B::kChunk)
                       : piece < kWords + 16 + D / 32 ? B::k_scale(s, piece - kWords - 16) : B::v_scale(s, piece - kWords - 16 - D / 32);
            };
            const uint8_t *from = cache + ((size_t)sh.from[j] * p.Hkv + head) * B::kBytes + at((L + node) % READER_PAGE_SIZE);
            to[r] = cache + ((size_t)sh.to[j] * p.Hkv + head) * B::kBytes + at((L + j) % READER_PAGE_SIZE);
            bytes[r] = piece < kWords ? 4 : piece < kWords + 16 ? D / 32 : 1;
            held[r] = bytes[r] == 4 ? *reinterpret_cast<const uint32_t *>(from) : bytes[r] == 2 ? *reinterpret_cast<const uint16_t *>(from) : *from;
        }
        __syncthreads();                                     // every row of this pass has been read
#pragma unroll
        for (int r = 0; r < kMovePerThread; ++r) {
            if (bytes[r] == 4) *reinterpret_cast<uint32_t *>(to[r]) = held[r];
            else if (bytes[r] == 2) *reinterpret_cast<uint16_t *>(to[r]) = (uint16_t)held[r];
            else if (bytes[r] == 1) *to[r] = (uint8_t)held[r];
        }
    }
    // (with several layers another launch writes the lengths: all of them read the old one)
    if (p.NL == 1 && tid == 0) p.seq_lens[b] = L + n + 1;
}

__global__ __launch_bounds__(READER_MAX_T) void kvq_lengths_kernel(KvqCompactParams p) {
    __shared__ PathShared sh;
    check_path(p, blockIdx.x, sh);
    if (threadIdx.x != 0) return;
    if (!sh.bad) p.seq_lens[blockIdx.x] = sh.L + sh.n + 1;
    else if (p.status) atomicOr(p.status, sh.bad);
}

}  // namespace

hipError_t launch_kvq_store(const KvqStoreParams &p, hipStream_t stream) {
    constexpr int kRows = kStoreThreads / 64;
    const int heads = p.D == 64 ? 8 : 4;
    const dim3 grid((p.N + kRows - 1) / kRows, (p.Hkv + heads - 1) / heads);
    if (p.D == 64) hipLaunchKernelGGL(kvq_store_kernel<64>, grid, dim3(kStoreThreads), 0, stream, p);
    else hipLaunchKernelGGL(kvq_store_kernel<128>, grid, dim3(kStoreThreads), 0, stream, p);
    return note_hip_error("launch kvq_store_kernel", hipGetLastError());
}

hipError_t launch_kvq_pack(const KvqStoreParams &p, hipStream_t stream) {
    constexpr int kUnits = kStoreThreads / 64;
    const long long units = ((long long)p.max_seq_len + READER_PAGE_SIZE - 1) / READER_PAGE_SIZE * p.Hkv;
    const dim3 grid((unsigned)((units > 0 ? units + kUnits - 1 : kUnits) / kUnits), p.B, p.NL);
    if (p.D == 64) hipLaunchKernelGGL(kvq_pack_kernel<64>, grid, dim3(kStoreThreads), 0, stream, p);
    else hipLaunchKernelGGL(kvq_pack_kernel<128>, grid, dim3(kStoreThreads), 0, stream, p);
    return note_hip_error("launch kvq_pack_kernel", hipGetLastError());
}

hipError_t launch_kvq_compact_layers(const KvqCompactParams &p, hipStream_t stream) {
    if (p.NL > 0) {
        if (p.D == 64) hipLaunchKernelGGL(kvq_compact_kernel<64>, dim3(p.B, p.NL), dim3(kMoveThreads), 0, stream, p);
        else hipLaunchKernelGGL(kvq_compact_kernel<128>, dim3(p.B, p.NL), dim3(kMoveThreads), 0, stream, p);
        const hipError_t e = hipGetLastError();
        if (e != hipSuccess || p.NL == 1) return note_hip_error("launch kvq_compact_kernel", e);
    }
    hipLaunchKernelGGL(kvq_lengths_kernel, dim3(p.B), dim3(READER_MAX_T), 0, stream, p);
    return note_hip_error("launch kvq_lengths_kernel", hipGetLastError());
}

}  // namespace reader

// Pages of a cache that sequences share: sequences forked, permuted and dropped by their page tables, and pages made ready for what
// the next step writes (taken from the pool, given back, copied where others hold them too).
//
// page_refs counts the table entries that name a page; nothing else is kept of the pool, so a free page is found by looking the
// counts over: lowest ids first, which makes every result the same whatever the order in which wavefronts run.
#include "prompt_common.h"
#include "kvq_common.h"

namespace reader {

namespace {

constexpr int kPage = READER_PAGE_SIZE;
__device__ __forceinline__ bool in_pool(int id, int64_t num_pages) { return id >= 0 && id < num_pages; }
__device__ __forceinline__ int pages_of(int positions) { return positions / kPage + (positions % kPage != 0); }

// ---- reorder: two launches, a workgroup per sequence.  The first copies the tables and takes the old entries out of the counts, the
// second writes the new rows and counts theirs.  A row that stays itself keeps the pages of its positions and their counts.
constexpr int kRowThreads = 256;

// the row that row b becomes (-1: none), and what is wrong with it
__device__ __forceinline__ int source_of(const PagesParams &p, int b, int &bad) {
    const int s = p.sources[b];
    if (s >= -1 && s < p.B) return s;
    bad |= READER_STATUS_BAD_PATH;
    return b;
}
__device__ __forceinline__ int held_pages(const PagesParams &p, int length) { return min(pages_of(max(length, 0)), p.max_pages); }

__global__ __launch_bounds__(kRowThreads) void pages_leave_kernel(PagesParams p) {
    const int b = blockIdx.x, L = p.seq_lens[b], held = held_pages(p, L);
    int bad = 0;
    const bool stays = source_of(p, b, bad) == b;
    int32_t *row = p.page_table + (size_t)b * p.max_pages, *copy = p.work + (size_t)b * p.max_pages;
    if (threadIdx.x == 0) {
        p.work[(size_t)p.B * p.max_pages + b] = L;
        if (L < 0 || pages_of(max(L, 0)) > p.max_pages) bad |= READER_STATUS_BAD_LENGTH;
    }
    for (int j = threadIdx.x; j < p.max_pages; j += kRowThreads) {
        const int id = row[j];
        const bool real = in_pool(id, p.num_pages);
        if (j < held) copy[j] = id;
        if (j < held && !real) bad |= READER_STATUS_BAD_PAGE;
        if (real && !(stays && j < held)) atomicSub(&p.page_refs[id], 1);
    }
    if (bad && p.status) atomicOr(p.status, bad);
}

__global__ __launch_bounds__(kRowThreads) void pages_take_kernel(PagesParams p) {
    const int b = blockIdx.x;
    int bad = 0;
    const int s = source_of(p, b, bad);
    const int L = s < 0 ? 0 : p.work[(size_t)p.B * p.max_pages + s], held = held_pages(p, L);
    int32_t *row = p.page_table + (size_t)b * p.max_pages;
    const int32_t *from = p.work + (size_t)max(s, 0) * p.max_pages;
    if (s != b) {
        if (threadIdx.x == 0) p.seq_lens[b] = L;
        for (int j = threadIdx.x; j < held; j += kRowThreads) {
            const int id = from[j];
            row[j] = id;
            if (in_pool(id, p.num_pages)) atomicAdd(&p.page_refs[id], 1);
        }
    }
    for (int j = held + threadIdx.x; j < p.max_pages; j += kRowThreads) row[j] = -1;
}

// ---- reserve: one workgroup does the bookkeeping, a second launch copies pages.
constexpr int kBookThreads = 1024, kBookWaves = kBookThreads / 64;

struct Book {
    int32_t part[READER_MAX_B];        // page that the first new position falls into the middle of, or -1
    int32_t need[READER_MAX_B];        // pages to take; then: of all sequences in front
    uint8_t copies[READER_MAX_B];      // that page is copied
    int sums[kBookWaves], free_here[kBookWaves];
    int found, total, bad;
};

// Inclusive sums over the lanes.
__device__ __forceinline__ int scan_lanes(int v, int lane) {
#pragma unroll
    for (int d = 1; d < 64; d <<= 1) {
        const int u = __shfl_up(v, d);
        if (lane >= d) v += u;
    }
    return v;
}

// What a sequence asks for: positions [L, new) on pages of its own.
struct Wish {
    int used, want, first;             // pages that hold positions, pages in all, first position
    bool ok, writes;
    __device__ __forceinline__ Wish(const PagesParams &p, int b) {
        const int L = p.seq_lens[b], n = p.new_lens[b];
        ok = L >= 0 && n >= L && pages_of(max(n, 0)) <= p.max_pages;
        first = L;
        used = ok ? pages_of(L) : 0;
        want = ok ? pages_of(n) : 0;
        writes = ok && n > L;
    }
};

// A wavefront takes a row of the table at a time.  Entries in front of `used` are read at one place at most; behind it, an entry that
// is given back is marked -2 - id until all are known (whether others hold a page is asked of the counts as they were).
__global__ __launch_bounds__(kBookThreads) void pages_book_kernel(PagesParams p) {
    __shared__ Book s;
    const int tid = threadIdx.x, lane = tid & 63, wave = tid >> 6;
    int32_t *const list = p.work, *const pairs = p.work + p.num_pages;
    if (tid == 0) s.found = s.bad = 0;
    __syncthreads();
    int bad = 0;
    for (int b = wave; b < p.B; b += kBookWaves) {
        const Wish w(p, b);
        int32_t *row = p.page_table + (size_t)b * p.max_pages;
        int need = 0, part = -1;
        if (!w.ok) bad |= READER_STATUS_BAD_LENGTH;
        else {
            if (w.writes && w.first % kPage != 0) {
                part = row[w.first / kPage];
                if (!in_pool(part, p.num_pages)) { part = -1; bad |= READER_STATUS_BAD_PAGE; }
            }
            for (int j = w.used + lane; j < p.max_pages; j += 64) {
                const int id = row[j];
                const bool real = in_pool(id, p.num_pages), drop = real && (j >= w.want || p.page_refs[id] > 1);
                if (drop) row[j] = -2 - id;
                else if (!real && id != -1) row[j] = -1;
                need += j < w.want && (drop || !real);
            }
            need = __builtin_amdgcn_readlane(scan_lanes(need, lane), 63);
        }
        if (lane == 0) { s.part[b] = part; s.need[b] = need; }
    }
    __syncthreads();
    // of the sequences that write into one page, the last keeps it if nobody else holds it
    for (int b = tid; b < p.B; b += kBookThreads) {
        const int part = s.part[b], holders = part >= 0 ? p.page_refs[part] : 0;
        bool copies = false;
        if (holders > 1) {
            int writers = 0, last = b;
            for (int c = 0; c < p.B; ++c)
                if (s.part[c] == part) { ++writers; last = max(last, c); }
            copies = !(last == b && writers == holders);
        }
        s.copies[b] = copies;
    }
    __syncthreads();
    // pages to take in front of each sequence: four sequences a thread
    {
        int mine[4], sum = 0;
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            const int b = tid * 4 + i;
            mine[i] = sum;
            if (b < p.B) sum += s.need[b] + s.copies[b];
        }
        const int upto = scan_lanes(sum, lane);
        if (lane == 63) s.sums[wave] = upto;
        __syncthreads();
        int before = upto - sum;
        for (int w = 0; w < wave; ++w) before += s.sums[w];
#pragma unroll
        for (int i = 0; i < 4; ++i)
            if (tid * 4 + i < p.B) s.need[tid * 4 + i] = before + mine[i];
        if (tid == kBookThreads - 1) s.total = before + sum;
    }
    // what is given back leaves the counts
    for (int b = wave; b < p.B; b += kBookWaves) {
        const Wish w(p, b);
        if (!w.ok) continue;
        const int32_t *row = p.page_table + (size_t)b * p.max_pages;
        for (int j = w.used + lane; j < p.max_pages; j += 64)
            if (row[j] < -1) atomicSub(&p.page_refs[-2 - row[j]], 1);
        if (lane == 0 && s.copies[b]) atomicSub(&p.page_refs[s.part[b]], 1);
    }
    __syncthreads();
    __threadfence();                                         // (the counts have changed behind this compute unit's cache)
    // the lowest free pages, as many as are wanted
    const int total = s.total;
    for (int64_t base = 0; base < p.num_pages && s.found < total; base += kBookThreads * 4) {
        const int64_t at = base + tid * 4;
        unsigned free_bits = 0;
#pragma unroll
        for (int i = 0; i < 4; ++i)
            if (at + i < p.num_pages && p.page_refs[at + i] == 0) free_bits |= 1u << i;
        const int mine = __popc(free_bits), upto = scan_lanes(mine, lane);
        if (lane == 63) s.free_here[wave] = upto;
        __syncthreads();
        int before = s.found + upto - mine, all = 0;
        for (int w = 0; w < kBookWaves; ++w) {
            if (w < wave) before += s.free_here[w];
            all += s.free_here[w];
        }
#pragma unroll
        for (int i = 0; i < 4; ++i)
            if (free_bits >> i & 1) {
                if (before < total) list[before] = (int32_t)(at + i);
                ++before;
            }
        __syncthreads();
        if (tid == 0) s.found += all;
        __syncthreads();
    }
    const bool enough = s.found >= total;
    if (!enough) bad |= READER_STATUS_NO_PAGES;
    __threadfence_block();
    __syncthreads();
    for (int b = wave; b < p.B; b += kBookWaves) {
        const Wish w(p, b);
        int32_t *row = p.page_table + (size_t)b * p.max_pages;
        const bool copies = s.copies[b];
        int next = s.need[b], from = -1, to = -1;
        if (copies) {
            from = s.part[b];
            if (lane == 0) {
                if (!enough) atomicAdd(&p.page_refs[from], 1);
                else {
                    to = list[next];
                    row[w.first / kPage] = to;
                    p.page_refs[to] = 1;
                }
            }
            ++next;
        }
        if (lane == 0) {
            pairs[2 * b] = enough && copies ? from : -1;
            pairs[2 * b + 1] = to;
        }
        if (!w.ok) continue;
        for (int j0 = w.used; j0 < p.max_pages; j0 += 64) {
            const int j = j0 + lane;
            const int id = j < p.max_pages ? row[j] : -1;
            if (!enough) {                                   // everything as it was
                if (id < -1) { row[j] = -2 - id; atomicAdd(&p.page_refs[-2 - id], 1); }
                continue;
            }
            const bool take = j < w.want && id < 0;
            const unsigned long long takers = __ballot(take);
            if (take) {
                const int page = list[next + __popcll(takers & ((1ull << lane) - 1ull))];
                row[j] = page;
                p.page_refs[page] = 1;
            } else if (id < -1) row[j] = -1;
            next += (int)__popcll(takers);
        }
    }
    if (bad && p.status) atomicOr(p.status, bad);
}

// A workgroup copies one page of one layer's cache.
constexpr int kCopyThreads = 256;
__global__ __launch_bounds__(kCopyThreads) void pages_copy_kernel(PagesParams p) {
    const int32_t *pairs = p.work + p.num_pages;
    const int from = pairs[2 * blockIdx.x], to = pairs[2 * blockIdx.x + 1];
    if (from < 0) return;
    char *cache = (blockIdx.z == 0 ? p.k_cache : p.v_cache) + (size_t)blockIdx.y * p.num_pages * p.page_bytes;
    const uint4 *src = reinterpret_cast<const uint4 *>(cache + (size_t)from * p.page_bytes);
    uint4 *dst = reinterpret_cast<uint4 *>(cache + (size_t)to * p.page_bytes);
    const int64_t n = p.page_bytes / 16;
#pragma unroll 4
    for (int64_t i = threadIdx.x; i < n; i += kCopyThreads) dst[i] = src[i];
}

}  // namespace

hipError_t launch_pages_reorder(const PagesParams &p, hipStream_t stream) {
    hipLaunchKernelGGL(pages_leave_kernel, dim3(p.B), dim3(kRowThreads), 0, stream, p);
    const hipError_t e = hipGetLastError();
    if (e != hipSuccess) return note_hip_error("launch pages_leave_kernel", e);
    hipLaunchKernelGGL(pages_take_kernel, dim3(p.B), dim3(kRowThreads), 0, stream, p);
    return note_hip_error("launch pages_take_kernel", hipGetLastError());
}

hipError_t launch_pages_reserve(const PagesParams &p, hipStream_t stream) {
    hipLaunchKernelGGL(pages_book_kernel, dim3(1), dim3(kBookThreads), 0, stream, p);
    hipError_t e = hipGetLastError();
    if (e != hipSuccess) return note_hip_error("launch pages_book_kernel", e);
    if (p.NL == 0) return e;
    hipLaunchKernelGGL(pages_copy_kernel, dim3(p.B, p.NL, p.v_cache ? 2 : 1), dim3(kCopyThreads), 0, stream, p);
    return note_hip_error("launch pages_copy_kernel", hipGetLastError());
}

}  // namespace reader

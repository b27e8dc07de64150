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
// second writes the new rows and counts theirs.  A row that stays itself keeps the pages of its positions and their counts.  512 rows of
// 1100 entries: 6.9 and 5.6 us, most of it the launch and two dependent trips to memory (with 256 threads a row 0.8 us more each: another
// trip; 1024 are slower where rows are short, 4096 of 20 entries 22 us instead of 17, restoring copies included).
constexpr int kRowThreads = 512;

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
#pragma unroll 4
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
#pragma unroll 4
        for (int j = threadIdx.x; j < held; j += kRowThreads) {
            const int id = from[j];
            row[j] = id;
            if (in_pool(id, p.num_pages)) atomicAdd(&p.page_refs[id], 1);
        }
    }
    for (int j = held + threadIdx.x; j < p.max_pages; j += kRowThreads) row[j] = -1;
}

// The same for a small table, by one workgroup in one launch: 8 sequences of 300 entries 7 us instead of 11, 48 of them 15.
constexpr int kSmallTable = 4096, kSmallThreads = 1024;
__global__ __launch_bounds__(kSmallThreads) void pages_reorder_small_kernel(PagesParams p) {
    __shared__ int32_t s_table[kSmallTable];
    const int all = p.B * p.max_pages;                       // (lengths behind the entries)
    int bad = 0;
    for (int i = threadIdx.x; i < all; i += kSmallThreads) s_table[i] = p.page_table[i];
    for (int b = threadIdx.x; b < p.B; b += kSmallThreads) s_table[all + b] = p.seq_lens[b];
    __syncthreads();
    const int lane = threadIdx.x & 63;
    for (int b = threadIdx.x >> 6; b < p.B; b += kSmallThreads / 64) {
        const int s = source_of(p, b, bad), L = s_table[all + b], mine = held_pages(p, L);
        const int new_L = s < 0 ? 0 : s_table[all + s], held = held_pages(p, new_L);
        if (L < 0 || pages_of(max(L, 0)) > p.max_pages) bad |= READER_STATUS_BAD_LENGTH;
        if (lane == 0 && s != b) p.seq_lens[b] = new_L;
        for (int j = lane; j < p.max_pages; j += 64) {
            const int old = s_table[b * p.max_pages + j], id = j < held ? s_table[max(s, 0) * p.max_pages + j] : -1;
            if (j < mine && !in_pool(old, p.num_pages)) bad |= READER_STATUS_BAD_PAGE;
            if (old == id) continue;
            if (in_pool(old, p.num_pages)) atomicSub(&p.page_refs[old], 1);
            if (in_pool(id, p.num_pages)) atomicAdd(&p.page_refs[id], 1);
            p.page_table[(size_t)b * p.max_pages + j] = id;
        }
    }
    if (bad && p.status) atomicOr(p.status, bad);
}

// ---- reserve: four launches.  Rows are marked, settled and applied by a wavefront each; in between one workgroup adds up what they ask
// for and finds the lowest free pages.  (One workgroup for all of that but the copies, restoring copies included: 16 sequences 18 us
// instead of 20.5, 64 32 instead of 22, 256 98 instead of 41; there is no form of it for a few sequences.)  16 sequences: the launches take 4, 2.5, 6 and 4 us, latency; 256 of which 174 copy a page in each of 32
// layers: 4, 3.7, 6 and 24, the copies at 8 TB/s (read and written; the caches hold a part of what the call before left).  Counts change
// in the second and the fourth launch only, and nobody reads one there that another wavefront may be changing: what the first has read
// of them is kept in the workspace.
constexpr int kBookWaves = 16, kBookThreads = 64 * kBookWaves, kPerWave = 8;      // (words of 64 pages that a wavefront looks over at a time)
constexpr int kMarkRows = 4;                          // rows of a workgroup

// The workspace: pages to take, then of every sequence
struct Book {
    int32_t *list;             // [num_pages] the free pages that are taken, in the order in which they are
    int32_t *part;             // page that the first new position falls into the middle of, or -1
    int32_t *holders;          // its count
    int32_t *copies;           // it is copied
    int32_t *need;             // pages to take; then: of all sequences in front
    int32_t *enough;           // [1]
    __device__ __forceinline__ explicit Book(const PagesParams &p) {
        list = p.work;
        part = list + p.num_pages;
        holders = part + p.B; copies = holders + p.B; need = copies + p.B; enough = need + p.B;
    }
};

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

// Inclusive sums over the lanes.
__device__ __forceinline__ int scan_lanes(int v, int lane) {
#pragma unroll
    for (int d = 1; d < 64; d <<= 1) {
        const int u = __shfl_up(v, d);
        if (lane >= d) v += u;
    }
    return v;
}

// A wavefront marks a row: entries behind `used` that are given back become -2 - id.
__device__ __forceinline__ void mark(const PagesParams &p, const Book &s, int b, int lane) {
    const Wish w(p, b);
    int32_t *row = p.page_table + (size_t)b * p.max_pages;
    int need = 0, part = -1, holders = 0, bad = 0;
    if (!w.ok) bad = READER_STATUS_BAD_LENGTH;
    else {
        if (w.writes && w.first % kPage != 0) {
            part = row[w.first / kPage];
            if (in_pool(part, p.num_pages)) holders = p.page_refs[part];
            else { part = -1; bad = READER_STATUS_BAD_PAGE; }
        }
#pragma unroll 2
        for (int j = w.used + lane; j < p.max_pages; j += 64) {
            const int id = row[j];
            const bool real = in_pool(id, p.num_pages), drop = real && (j >= w.want || p.page_refs[id] > 1);
            if (drop) row[j] = -2 - id;
            else if (!real && id != -1) row[j] = -1;
            need += j < w.want && (drop || !real);
        }
        need = __builtin_amdgcn_readlane(scan_lanes(need, lane), 63);
    }
    if (lane == 0) {
        s.part[b] = part; s.holders[b] = holders; s.need[b] = need;
        if (bad && p.status) atomicOr(p.status, bad);
    }
}

// ... and settles it: what is given back leaves the counts.  Of the sequences that write into one page, the last keeps it if nobody
// else holds it.
__device__ __forceinline__ void settle(const PagesParams &p, const Book &s, int b, int lane) {
    const int part = s.part[b], holders = s.holders[b];
    bool copies = false;
    if (holders > 1) {
        int writers = 0, last = b;
        for (int base = 0; base < p.B; base += 64) {
            const unsigned long long same = __ballot(base + lane < p.B && s.part[min(base + lane, p.B - 1)] == part);
            writers += (int)__popcll(same);
            if (same) last = max(last, base + 63 - (int)__builtin_clzll(same));
        }
        copies = !(last == b && writers == holders);
    }
    const Wish w(p, b);
    if (w.ok) {
        const int32_t *row = p.page_table + (size_t)b * p.max_pages;
#pragma unroll 2
        for (int j = w.used + lane; j < p.max_pages; j += 64) {
            const int id = row[j];
            if (id < -1) atomicSub(&p.page_refs[-2 - id], 1);
        }
    }
    // (a page that is copied from leaves with the copy: it is in use till then, also where all others give it back here)
    if (lane == 0) s.copies[b] = copies;
}

// The sums in front of every sequence, and the lowest free pages: a workgroup of kBookThreads.
__device__ __forceinline__ void find(const PagesParams &p, const Book &s) {
    __shared__ int s_sums[kBookWaves], s_free[2][kBookWaves];
    const int tid = threadIdx.x, lane = tid & 63, wave = tid >> 6;
    int total = 0;
    {
        int mine[READER_MAX_B / kBookThreads], sum = 0;      // sequences of a thread
        const int first = tid * (READER_MAX_B / kBookThreads);
#pragma unroll
        for (int i = 0; i < READER_MAX_B / kBookThreads; ++i) {
            mine[i] = sum;
            if (first + i < p.B) sum += s.need[first + i] + s.copies[first + i];
        }
        const int upto = scan_lanes(sum, lane);
        if (lane == 63) s_sums[wave] = upto;
        __syncthreads();
        int before = upto - sum;
        for (int w = 0; w < kBookWaves; ++w) {
            if (w < wave) before += s_sums[w];
            total += s_sums[w];
        }
#pragma unroll
        for (int i = 0; i < READER_MAX_B / kBookThreads; ++i)
            if (first + i < p.B) s.need[first + i] = before + mine[i];
    }
    int found = 0;
    for (int64_t base = 0, turn = 0; base < p.num_pages && found < total; base += kBookThreads * kPerWave, turn ^= 1) {
        const int64_t from = base + wave * (64 * kPerWave);
        unsigned long long free_pages[kPerWave];
        int count = 0;
#pragma unroll
        for (int i = 0; i < kPerWave; ++i) {
            const int64_t at = from + i * 64 + lane;
            free_pages[i] = __ballot(at < p.num_pages && p.page_refs[min(at, p.num_pages - 1)] == 0);
            count += (int)__popcll(free_pages[i]);
        }
        if (lane == 0) s_free[turn][wave] = count;
        __syncthreads();                                     // (the next turn writes the other half)
        int before = found;
        for (int w = 0; w < kBookWaves; ++w) {
            if (w < wave) before += s_free[turn][w];
            found += s_free[turn][w];
        }
#pragma unroll
        for (int i = 0; i < kPerWave; ++i) {
            const int at = before + (int)__popcll(free_pages[i] & ((1ull << lane) - 1ull));
            if ((free_pages[i] >> lane & 1) && at < total) s.list[at] = (int32_t)(from + i * 64 + lane);
            before += (int)__popcll(free_pages[i]);
        }
    }
    if (tid == 0) {
        s.enough[0] = found >= total;
        if (found < total && p.status) atomicOr(p.status, READER_STATUS_NO_PAGES);
    }
}

__global__ __launch_bounds__(64 * kMarkRows) void pages_mark_kernel(PagesParams p) {
    const int b = blockIdx.x * kMarkRows + (threadIdx.x >> 6);
    if (b < p.B) mark(p, Book(p), b, threadIdx.x & 63);
}
__global__ __launch_bounds__(64 * kMarkRows) void pages_settle_kernel(PagesParams p) {
    const int b = blockIdx.x * kMarkRows + (threadIdx.x >> 6);
    if (b < p.B) settle(p, Book(p), b, threadIdx.x & 63);
}
__global__ __launch_bounds__(kBookThreads) void pages_find_kernel(PagesParams p) { find(p, Book(p)); }

// A workgroup copies one page of one layer's cache; the first of each sequence writes its row of the table.
constexpr int kCopyThreads = 256;
__global__ __launch_bounds__(kCopyThreads) void pages_apply_kernel(PagesParams p) {
    const int b = blockIdx.x, lane = threadIdx.x & 63;
    const Book s(p);
    const bool copies = s.copies[b] != 0, enough = s.enough[0] != 0;
    const int from = s.part[b], base = s.need[b], to = copies && enough ? s.list[base] : -1;
    if (blockIdx.y == 0 && blockIdx.z == 0 && threadIdx.x < 64) {
        const Wish w(p, b);
        int32_t *row = p.page_table + (size_t)b * p.max_pages;
        int next = base + copies;
        if (to >= 0 && lane == 0) {
            atomicSub(&p.page_refs[from], 1);
            row[w.first / kPage] = to;
            p.page_refs[to] = 1;
        }
        for (int j0 = w.used; w.ok && j0 < p.max_pages; j0 += 64) {
            const int j = j0 + lane;
            const int id = j < p.max_pages ? row[j] : -1;
            if (!enough) {                                   // everything as it was
                if (id < -1) { row[j] = -2 - id; atomicAdd(&p.page_refs[-2 - id], 1); }
                continue;
            }
            const bool take = j < w.want && id < 0;
            const unsigned long long takers = __ballot(take);
            if (take) {
                const int page = s.list[next + (int)__popcll(takers & ((1ull << lane) - 1ull))];
                row[j] = page;
                p.page_refs[page] = 1;
            } else if (id < -1) row[j] = -1;
            next += (int)__popcll(takers);
        }
    }
    if (to < 0 || p.NL == 0) return;
    char *cache = (blockIdx.z == 0 ? p.k_cache : p.v_cache) + (size_t)blockIdx.y * p.num_pages * p.page_bytes;
    const uint4 *src = reinterpret_cast<const uint4 *>(cache + (size_t)from * p.page_bytes);
    uint4 *dst = reinterpret_cast<uint4 *>(cache + (size_t)to * p.page_bytes);
    const int n = (int)(p.page_bytes / 16);
#pragma unroll 4
    for (int i = threadIdx.x; i < n; i += kCopyThreads) dst[i] = src[i];
}

}  // namespace

hipError_t launch_pages_reorder(const PagesParams &p, hipStream_t stream) {
    if ((long long)p.B * (p.max_pages + 1LL) <= kSmallTable) {
        hipLaunchKernelGGL(pages_reorder_small_kernel, dim3(1), dim3(kSmallThreads), 0, stream, p);
        return note_hip_error("launch pages_reorder_small_kernel", hipGetLastError());
    }
    hipLaunchKernelGGL(pages_leave_kernel, dim3(p.B), dim3(kRowThreads), 0, stream, p);
    const hipError_t e = hipGetLastError();
    if (e != hipSuccess) return note_hip_error("launch pages_leave_kernel", e);
    hipLaunchKernelGGL(pages_take_kernel, dim3(p.B), dim3(kRowThreads), 0, stream, p);
    return note_hip_error("launch pages_take_kernel", hipGetLastError());
}

hipError_t launch_pages_reserve(const PagesParams &p, hipStream_t stream) {
    const dim3 rows((p.B + kMarkRows - 1) / kMarkRows), row_threads(64 * kMarkRows);
    hipLaunchKernelGGL(pages_mark_kernel, rows, row_threads, 0, stream, p);
    hipLaunchKernelGGL(pages_settle_kernel, rows, row_threads, 0, stream, p);
    hipLaunchKernelGGL(pages_find_kernel, dim3(1), dim3(kBookThreads), 0, stream, p);
    hipLaunchKernelGGL(pages_apply_kernel, dim3(p.B, p.NL > 0 ? p.NL : 1, p.NL > 0 && p.v_cache ? 2 : 1), dim3(kCopyThreads), 0, stream, p);
    return note_hip_error("launch pages_apply_kernel", hipGetLastError());
}

}  // namespace reader

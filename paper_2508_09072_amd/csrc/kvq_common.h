// A cache in 4 bits: where a row's bytes are, and the parameters of the launches that write, move and read them.
//
// A page of a kv head is a block of 17 D bytes: the codes of K, the codes of V (4 bits a value: sign, then 0, 1/2, 1, 3/2, 2, 3, 4,
// 6; value 2 i in the low half of a byte), the scales of K, the scales of V (a byte for 32 values of a row, the exponent + 127).
// Inside, bytes lie as the attention's lanes read them, so that a wavefront's load of a page is one contiguous piece and nothing
// passes through LDS or between lanes on its way into the matrix instructions (kvq_attn.hip):
//   K  [quarter of the row 4][row 16][D / 8 bytes]           lane (quarter, row) holds D / 4 values of a row: the k-steps of the
//                                                            first product, in an order that the queries follow
//   V  [quad of rows 4][chunk of D / 16 values 16][row of the quad 4][D / 32 bytes]   lane (quad, chunk) holds D / 16 columns of four
//                                                            rows: the keys whose scores the first product leaves it with
//   K scales [group of 32 values][row 16], V scales [quad of rows 4][group][row of the quad 4]
// A byte belongs to one row: rows are written and moved without reading their neighbours.
#pragma once

#include "prompt_common.h"

namespace reader {

template <int D>
struct KvqBlock {
    static constexpr int kBytes = 17 * D, kV = 8 * D, kKScales = 16 * D, kVScales = 16 * D + D / 2;
    static constexpr int kGroups = D / 32, kQuarter = D / 4, kChunk = D / 16;
    // bytes of values d, d + 1 (d even) and of the scale of group g, of row s
    __host__ __device__ static constexpr int k_code(int s, int d) { return d / kQuarter * (8 * kQuarter) + s * (kQuarter / 2) + d % kQuarter / 2; }
    __host__ __device__ static constexpr int v_code(int s, int d) { return kV + s / 4 * (2 * D) + d / kChunk * (2 * kChunk) + s % 4 * (kChunk / 2) + d % kChunk / 2; }
    __host__ __device__ static constexpr int k_scale(int s, int g) { return kKScales + g * 16 + s; }
    __host__ __device__ static constexpr int v_scale(int s, int g) { return kVScales + s / 4 * (D / 8) + g * 4 + s % 4; }
};
// exponents of a scale: every value, 1/2 to 6 times it, is a finite bf16 number with a full mantissa
constexpr int kKvqLowest = -125, kKvqHighest = 125;

struct KvqStoreParams {
    const uint16_t *k, *v;         // rows [N, Hkv, D], or bf16 caches [NL, from_pages, Hkv, page_size, D]
    const int32_t *cu_tokens;      // packed rows, or null: T of every sequence
    const int32_t *from_table, *starts;    // (pages) where the positions are, and the first of them or null
    const int32_t *seq_lens, *page_table;
    uint8_t *cache;                // [NL, num_pages, Hkv, 17 D]
    int32_t *status;
    int32_t NL, B, T, N, Hkv, D, max_pages, max_seq_len;
    int64_t num_pages, from_pages;
};
hipError_t launch_kvq_store(const KvqStoreParams &p, hipStream_t stream);
hipError_t launch_kvq_pack(const KvqStoreParams &p, hipStream_t stream);

struct KvqCompactParams {
    uint8_t *cache;                // [NL, num_pages, Hkv, 17 D]
    const int32_t *path, *accept_len, *page_table;
    int32_t *seq_lens, *status;
    int32_t NL, B, T, Hkv, D, max_pages, max_path;
    int64_t num_pages;
};
hipError_t launch_kvq_compact_layers(const KvqCompactParams &p, hipStream_t stream);

struct KvqAttnParams : PromptParams {      // (k_cache and v_cache are not used; max_seq_len leaves room for a tree)
    const uint8_t *cache;                  // [num_pages, Hkv, 17 D]
    const int32_t *parents;                // draft trees [B, nodes], or null
};
constexpr int kKvqMaxPositions = 1 << 30;              // of a sequence
// of kvq_attn_rows: 16 and 64 rows a workgroup, blocks that are not cut (and kUncut32); 16 rows, ranges for few blocks
constexpr int kUncut16 = 17, kUncut64 = 65, kFew16 = 18;
size_t kvq_attn_workspace_bytes(int D);
int kvq_attn_rows(const KvqAttnParams &p);
hipError_t launch_kvq_attn(const KvqAttnParams &p, hipStream_t stream);
hipError_t launch_kvq_attn_wide(const KvqAttnParams &p, int rows, hipStream_t stream);    // 128 or 256 rows a workgroup

struct PagesParams {
    const int32_t *sources;        // (reorder) [B]
    const int32_t *new_lens;       // (reserve) [B]
    int32_t *page_table, *seq_lens, *page_refs, *status, *work;   // (reserve does not write seq_lens)
    char *k_cache, *v_cache;       // (reserve) [NL, num_pages, page_bytes], v may be null
    int32_t NL, B, max_pages;
    int64_t num_pages, page_bytes;
};
hipError_t launch_pages_reorder(const PagesParams &p, hipStream_t stream);
hipError_t launch_pages_reserve(const PagesParams &p, hipStream_t stream);

}  // namespace reader

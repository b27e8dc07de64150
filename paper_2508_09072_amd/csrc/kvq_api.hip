// C ABI entry points of the cache in 4 bits and of the pages that sequences share: argument validation on the host and dispatch.
// They are defined in include/reader.h.
#include <math.h>

#include "kvq_common.h"

namespace reader {

template <class... Pointers>
static bool aligned(const Pointers *...p) { return (((uintptr_t)p | ...) & 15) == 0; }

// The dimensions of a call on the cache in 4 bits (its kernels have no second variant; heads are a dimension of a grid).
static int kvq_dims(const reader_dims *dims) {
    int err = 0;
    if (!dims_ok(dims, &err)) return err;
    if (dims->variant != 0) return READER_EINVAL;
    return dims->Hkv > 65535 ? READER_EUNSUPPORTED : READER_OK;
}

static int kvq_rows(const reader_dims *dims, int32_t N) {
    if (N < 0) return READER_EINVAL;
    return N <= READER_MAX_TOKENS && (long long)N * dims->Hq <= 0x7fffffffLL ? READER_OK : READER_EUNSUPPORTED;
}

static bool kvq_cache(const reader_dims *dims, const void *kvq_cache, const int32_t *page_table) {
    return kvq_cache && page_table && dims->num_pages >= 1 && dims->max_pages_per_seq >= 1 && aligned(kvq_cache);
}

// What both forms of the attention check and fill; `room`: cache positions behind max_seq_len that rows of the call may see.
static int kvq_attn(const reader_dims *dims, int32_t N, const void *q, const void *cache, const int32_t *page_table,
                    const int32_t *seq_lens, void *out, float *lse, int32_t max_seq_len, int32_t room, void *workspace,
                    size_t workspace_bytes, int32_t *status, KvqAttnParams &p) {
    if (!q || !seq_lens || !out || !kvq_cache(dims, cache, page_table) || !aligned(q, out)) return READER_EINVAL;
    if ((long long)dims->max_pages_per_seq * dims->page_size < (long long)max_seq_len + room) return READER_EINVAL;
    if ((long long)max_seq_len + room > kKvqMaxPositions) return READER_EUNSUPPORTED;      // (steps ahead of the last one are counted too)
    if (!workspace || ((uintptr_t)workspace & 255) != 0 || workspace_bytes < reader_kvq_workspace_bytes(dims, N, max_seq_len)) return READER_EWORKSPACE;
    p.q = (const uint16_t *)q; p.cache = (const uint8_t *)cache;
    p.page_table = page_table; p.seq_lens = seq_lens;
    p.out = (uint16_t *)out; p.lse = lse; p.status = status; p.workspace = workspace;
    p.B = dims->B; p.N = N; p.Hq = dims->Hq; p.Hkv = dims->Hkv; p.G = dims->Hq / dims->Hkv; p.D = dims->D;
    p.max_pages = dims->max_pages_per_seq; p.max_seq_len = max_seq_len + room; p.num_pages = dims->num_pages;
    p.scale_log2 = (dims->sm_scale > 0.f ? dims->sm_scale : 1.0f / sqrtf((float)dims->D)) * 1.44269504088896340736f;
    p.g_rcp = 1.0f / (float)p.G;
    return READER_OK;
}

static size_t pages_workspace(const reader_dims *dims) {
    const size_t reserve = (size_t)dims->num_pages + 4 * (size_t)dims->B + 1, reorder = (size_t)dims->B * ((size_t)dims->max_pages_per_seq + 1);
    return ((reserve > reorder ? reserve : reorder) * sizeof(int32_t) + 255) & ~(size_t)255;
}

// What both operations on pages check and fill.
static int pages(const reader_dims *dims, int32_t *page_table, const int32_t *seq_lens, int32_t *page_refs, void *workspace, size_t workspace_bytes,
                 int32_t *status, PagesParams &p) {
    if (!page_table || !seq_lens || !page_refs || dims->num_pages < 1 || dims->max_pages_per_seq < 1) return READER_EINVAL;
    if (dims->num_pages > 0x7ffffff0LL) return READER_EUNSUPPORTED;          // (ids are marked with a sign on their way)
    if (!workspace || ((uintptr_t)workspace & 3) != 0 || workspace_bytes < pages_workspace(dims)) return READER_EWORKSPACE;
    p.page_table = page_table; p.page_refs = page_refs; p.status = status; p.work = (int32_t *)workspace;
    p.B = dims->B; p.max_pages = dims->max_pages_per_seq; p.num_pages = dims->num_pages;
    return READER_OK;
}

}  // namespace reader

using namespace reader;

extern "C" int reader_kvq_store(const reader_dims *dims, int32_t N, const void *k, const void *v, const int32_t *cu_tokens,
                                const int32_t *seq_lens, void *kvq_cache_, const int32_t *page_table, int32_t *status, void *stream) {
    int rc = kvq_dims(dims);
    if (rc != READER_OK) return rc;
    if (!cu_tokens && (long long)N != (long long)dims->B * dims->T) return READER_EINVAL;
    rc = kvq_rows(dims, N);
    if (rc != READER_OK) return rc;
    if (dims->B == 0 || N == 0) return READER_OK;
    if (!k || !v || !seq_lens || !kvq_cache(dims, kvq_cache_, page_table) || !aligned(k, v)) return READER_EINVAL;
    KvqStoreParams p = {};
    p.k = (const uint16_t *)k; p.v = (const uint16_t *)v; p.cu_tokens = cu_tokens; p.seq_lens = seq_lens; p.page_table = page_table;
    p.cache = (uint8_t *)kvq_cache_; p.status = status;
    p.NL = 1; p.B = dims->B; p.T = dims->T; p.N = N; p.Hkv = dims->Hkv; p.D = dims->D;
    p.max_pages = dims->max_pages_per_seq; p.num_pages = dims->num_pages;
    forget_stale_error();
    return launch_kvq_store(p, (hipStream_t)stream) == hipSuccess ? READER_OK : READER_EHIP;
}

extern "C" int reader_kvq_pack(const reader_dims *dims, int32_t num_layers, const void *k_cache, const void *v_cache, int64_t from_pages,
                               const int32_t *from_table, const int32_t *starts, const int32_t *seq_lens, int32_t max_seq_len,
                               void *kvq_cache_, const int32_t *page_table, int32_t *status, void *stream) {
    const int rc = kvq_dims(dims);
    if (rc != READER_OK) return rc;
    if (num_layers < 0 || max_seq_len < 0 || from_pages < 0) return READER_EINVAL;
    if (num_layers > 65535 || from_pages * dims->Hkv > 0x7fffffffLL || from_pages > 0x7fffffffLL) return READER_EUNSUPPORTED;
    if (dims->B == 0 || num_layers == 0) return READER_OK;
    if (!k_cache || !v_cache || !from_table || !seq_lens || from_pages < 1 || !kvq_cache(dims, kvq_cache_, page_table) || !aligned(k_cache, v_cache)) return READER_EINVAL;
    // (pages of heads are counted with the threads of a launch)
    if (((long long)max_seq_len / READER_PAGE_SIZE + 1) * dims->Hkv > (1 << 25)) return READER_EUNSUPPORTED;
    KvqStoreParams p = {};
    p.k = (const uint16_t *)k_cache; p.v = (const uint16_t *)v_cache; p.from_table = from_table; p.starts = starts;
    p.seq_lens = seq_lens; p.page_table = page_table; p.cache = (uint8_t *)kvq_cache_; p.status = status;
    p.NL = num_layers; p.B = dims->B; p.Hkv = dims->Hkv; p.D = dims->D;
    p.max_pages = dims->max_pages_per_seq; p.max_seq_len = max_seq_len; p.num_pages = dims->num_pages; p.from_pages = from_pages;
    forget_stale_error();
    return launch_kvq_pack(p, (hipStream_t)stream) == hipSuccess ? READER_OK : READER_EHIP;
}

extern "C" int reader_kvq_compact_layers(const reader_dims *dims, int32_t num_layers, const int32_t *path, const int32_t *accept_len,
                                         void *kvq_cache_, const int32_t *page_table, int32_t *seq_lens, int32_t *status, void *stream) {
    const int rc = kvq_dims(dims);
    if (rc != READER_OK) return rc;
    if (num_layers < 0) return READER_EINVAL;
    if (num_layers > 65535) return READER_EUNSUPPORTED;
    if (dims->B == 0) return READER_OK;
    if (!path || !accept_len || !seq_lens || !page_table) return READER_EINVAL;
    if (num_layers > 0 && !kvq_cache(dims, kvq_cache_, page_table)) return READER_EINVAL;
    KvqCompactParams p = {};
    p.cache = (uint8_t *)kvq_cache_; p.path = path; p.accept_len = accept_len; p.page_table = page_table;
    p.seq_lens = seq_lens; p.status = status;
    p.NL = num_layers; p.B = dims->B; p.T = dims->T; p.Hkv = dims->Hkv; p.D = dims->D;
    p.max_pages = dims->max_pages_per_seq; p.max_path = dims->max_path; p.num_pages = dims->num_pages;
    forget_stale_error();
    return launch_kvq_compact_layers(p, (hipStream_t)stream) == hipSuccess ? READER_OK : READER_EHIP;
}

extern "C" size_t reader_kvq_workspace_bytes(const reader_dims *dims, int32_t N, int32_t max_seq_len) {
    if (kvq_dims(dims) != READER_OK || kvq_rows(dims, N) != READER_OK || max_seq_len < 0) return 0;
    return (kvq_attn_workspace_bytes(dims->D) + 255) & ~(size_t)255;
}

extern "C" int reader_kvq_tree_attn(const reader_dims *dims, const void *q, const void *kvq_cache_, const int32_t *page_table,
                                    const int32_t *seq_lens, const int32_t *parents, void *out, float *lse, int32_t max_seq_len,
                                    void *workspace, size_t workspace_bytes, int32_t *status, void *stream) {
    int rc = kvq_dims(dims);
    if (rc != READER_OK) return rc;
    const int32_t N = dims->B * dims->T;
    rc = kvq_rows(dims, N);
    if (rc != READER_OK) return rc;
    if (max_seq_len < 0) return READER_EINVAL;
    if (dims->B == 0) return READER_OK;
    if (!parents) return READER_EINVAL;
    KvqAttnParams p = {};
    rc = kvq_attn(dims, N, q, kvq_cache_, page_table, seq_lens, out, lse, max_seq_len, dims->T, workspace, workspace_bytes, status, p);
    if (rc != READER_OK) return rc;
    p.parents = parents; p.nodes = dims->T;
    forget_stale_error();
    return launch_kvq_attn(p, (hipStream_t)stream) == hipSuccess ? READER_OK : READER_EHIP;
}

extern "C" int reader_kvq_prompt_attn(const reader_dims *dims, int32_t N, const void *q, const void *kvq_cache_, const int32_t *page_table,
                                      const int32_t *cu_tokens, const int32_t *seq_lens, void *out, float *lse, int32_t max_seq_len,
                                      void *workspace, size_t workspace_bytes, int32_t *status, void *stream) {
    int rc = kvq_dims(dims);
    if (rc != READER_OK) return rc;
    rc = kvq_rows(dims, N);
    if (rc != READER_OK) return rc;
    if (max_seq_len < 0) return READER_EINVAL;
    if (dims->B == 0 || N == 0) return READER_OK;
    if (!cu_tokens) return READER_EINVAL;
    KvqAttnParams p = {};
    rc = kvq_attn(dims, N, q, kvq_cache_, page_table, seq_lens, out, lse, max_seq_len, 0, workspace, workspace_bytes, status, p);
    if (rc != READER_OK) return rc;
    p.cu_tokens = cu_tokens;
    forget_stale_error();
    return launch_kvq_attn(p, (hipStream_t)stream) == hipSuccess ? READER_OK : READER_EHIP;
}

extern "C" size_t reader_pages_workspace_bytes(const reader_dims *dims) {
    int err = 0;
    return dims_ok(dims, &err) ? pages_workspace(dims) : 0;
}

extern "C" int reader_pages_reorder(const reader_dims *dims, const int32_t *sources, int32_t *page_table, int32_t *seq_lens, int32_t *page_refs,
                                    void *workspace, size_t workspace_bytes, int32_t *status, void *stream) {
    int err = 0;
    if (!dims_ok(dims, &err)) return err;
    if (dims->B == 0) return READER_OK;
    if (!sources) return READER_EINVAL;
    PagesParams p = {};
    const int rc = pages(dims, page_table, seq_lens, page_refs, workspace, workspace_bytes, status, p);
    if (rc != READER_OK) return rc;
    p.sources = sources; p.seq_lens = seq_lens;
    forget_stale_error();
    return launch_pages_reorder(p, (hipStream_t)stream) == hipSuccess ? READER_OK : READER_EHIP;
}

extern "C" int reader_pages_reserve(const reader_dims *dims, int32_t num_layers, int64_t page_bytes, const int32_t *seq_lens,
                                    const int32_t *new_lens, void *k_cache, void *v_cache, int32_t *page_table, int32_t *page_refs,
                                    void *workspace, size_t workspace_bytes, int32_t *status, void *stream) {
    int err = 0;
    if (!dims_ok(dims, &err)) return err;
    if (num_layers < 0 || page_bytes < 0) return READER_EINVAL;
    if (num_layers > 65535 || page_bytes > 0x7fffffffLL) return READER_EUNSUPPORTED;
    if (dims->B == 0) return READER_OK;
    if (!new_lens) return READER_EINVAL;
    if (num_layers > 0 && (!k_cache || page_bytes < 16 || page_bytes % 16 != 0 || !aligned(k_cache, v_cache))) return READER_EINVAL;
    PagesParams p = {};
    const int rc = pages(dims, page_table, seq_lens, page_refs, workspace, workspace_bytes, status, p);
    if (rc != READER_OK) return rc;
    p.seq_lens = const_cast<int32_t *>(seq_lens); p.new_lens = new_lens;
    p.k_cache = (char *)k_cache; p.v_cache = (char *)v_cache; p.NL = num_layers; p.page_bytes = page_bytes;
    forget_stale_error();
    return launch_pages_reserve(p, (hipStream_t)stream) == hipSuccess ? READER_OK : READER_EHIP;
}

// C ABI entry points of the operators around the verification step (prompts, per-head norms and rotation, accumulated key
// weights, eviction): argument validation on the host and dispatch.  They are defined in include/reader.h.
#include <math.h>

#include "prompt_common.h"

namespace reader {

static float softmax_scale_log2(const reader_dims &d) {
    return (d.sm_scale > 0.f ? d.sm_scale : 1.0f / sqrtf((float)d.D)) * 1.44269504088896340736f;
}

// What both forms of the projections' operator check and fill.
static int qkv_prepare(const reader_dims *dims, const void *qkv, const int32_t *seq_lens, const int32_t *positions,
                       const void *q_norm, const void *k_norm, float eps, const float *cos_sin, int32_t max_positions,
                       int32_t rot_dims, int32_t interleaved, void *q, int32_t *status, QkvParams &p) {
    if (rot_dims < 0 || rot_dims > dims->D || max_positions < 0 || (interleaved != 0 && interleaved != 1)) return READER_EINVAL;
    if (rot_dims % 16 != 0) return READER_EUNSUPPORTED;
    if ((q_norm == nullptr) != (k_norm == nullptr)) return READER_EINVAL;
    if (q_norm && !(eps >= 0.f && eps <= 1.f)) return READER_EINVAL;
    if (!qkv || !seq_lens || !q || (rot_dims > 0 && !cos_sin)) return READER_EINVAL;
    p.qkv = (const uint16_t *)qkv; p.q_norm = (const uint16_t *)q_norm; p.k_norm = (const uint16_t *)k_norm;
    p.cos_sin = cos_sin; p.seq_lens = seq_lens; p.positions = positions; p.q = (uint16_t *)q; p.status = status;
    p.B = dims->B; p.T = dims->T; p.Hq = dims->Hq; p.Hkv = dims->Hkv; p.D = dims->D;
    p.max_pages = dims->max_pages_per_seq; p.num_pages = dims->num_pages;
    p.max_positions = max_positions; p.rot = rot_dims; p.interleaved = interleaved; p.eps = eps;
    return READER_OK;
}

// Packed rows: their number, and that the (row, head) pairs of them can be counted in 31 bits.
static int rows_ok(const reader_dims *dims, int32_t N) {
    if (N < 0) return READER_EINVAL;
    return N <= READER_MAX_TOKENS && (long long)N * (dims->Hq + 2LL * dims->Hkv) <= 0x7fffffffLL ? READER_OK : READER_EUNSUPPORTED;
}

// The cache and page table of a call that reads or writes them.
static bool cache_ok(const reader_dims *dims, const void *k_cache, const void *v_cache, const int32_t *page_table) {
    return k_cache && v_cache && page_table && dims->num_pages >= 1 && dims->max_pages_per_seq >= 1;
}

// Query rows a workgroup takes (reader_prompt_rows).
//
// Up to 16 or 32 rows that a sequence has for each kv head, on average (the host knows no more): the kernel that streams keys for
// few rows.  Measured against the 256-row kernel: 16 single tokens on 1 to 16 K positions 99 to 122 us; 8 chunks of 8 tokens (32
// rows) on 2 to 9 K 45 to 55 and, with 64 rows, where it is not taken, 63 to 90.
//
// Beyond that the shortest of three estimates, for blocks that are never cut (64 or 128 rows) and for the 256-row kernel, which cuts
// the keys of all blocks evenly.  The first two last as long as the longest block's steps of 32 keys, one after the other, or as long
// as all blocks' steps take the compute units; the third 30 us of start, merge and imbalance, and per block what its tiles of 64
// keys and its ends take.  The constants are fitted to 100 shapes (5 head layouts; 1 to 64 sequences of 100 to 3000 tokens, chunks on
// up to 8 K positions): of the 98 with more than 32 rows the estimates pick the fastest of the three on 85
// and are 1 % behind it on average, 22 % at most.  Some
// of them, 256, 64 and 128 rows: one prompt of 100 tokens 19.5, 6.5 and 8.1 us; of 800 39.6, 24.0, 28.2; of 3000 106, 137, 106; 16
// of 300 48.9, 48.8, 42.3; 16 of 800 167, 198, 157; 256 tokens on 8 K positions 76, 189, 229 (32 query and 8 kv heads, D 128).
static int prompt_rows(const reader_dims &d, int32_t N, int32_t max_seq_len) {
    if (d.variant == 1) return 0;
    const int forced = tuning(READER_TUNE_PROMPT_ROWS), G = d.Hq / d.Hkv;
    if (forced == 16 || forced == 32 || forced == 64 || forced == 128 || forced == 256) return forced;
    if (d.B == 0 || (long long)N * G <= 16LL * d.B) return 16;
    if ((long long)N * G <= 32LL * d.B) return 32;
    const double tokens = (double)N / d.B;                        // of a sequence
    const double longest = max_seq_len > tokens ? max_seq_len : tokens, average = longest - 0.5 * tokens;   // keys of a block
    auto blocks = [&](int rows) { return (double)d.Hkv * d.B * ceil(tokens / (rows / G)); };
    auto uncut = [&](int rows, double step, double busy) {
        const double chain = step * (longest / 32 + 0.5), all = busy * blocks(rows) * (average / 32 + 0.5) / kNumCU;
        return 5.5 + (chain > all ? chain : all);
    };
    const bool wide_heads = d.D == 128;
    const double rows64 = wide_heads ? uncut(64, 0.76, 0.60) : uncut(64, 0.50, 0.32);
    const double rows128 = wide_heads ? uncut(128, 0.93, 0.87) : uncut(128, 0.64, 0.51);
    const double rows256 = 30.0 + blocks(256) / kNumCU * (wide_heads ? 11.0 + 1.65 * (average / 64 + 0.5) : 8.0 + 0.9 * (average / 64 + 0.5));
    // (block numbers of the uncut kernels are counted with the threads of a launch)
    const bool countable = ((long long)N / (64 / G) + d.B) * d.Hkv < (1 << 23);
    if (!countable || (rows256 <= rows64 && rows256 <= rows128)) return 256;
    return rows64 <= rows128 ? 64 : 128;
}

static hipError_t launch_prompt(const PromptParams &p, int rows, hipStream_t stream) {
    switch (rows) {
        case 0: return launch_prompt_attn_scalar(p, stream);
        case 16: case 32: return launch_prompt_few(p, rows, stream);
        case 64: case 128: return launch_prompt_mid(p, rows, stream);
        default: return launch_prompt_wide(p, stream);
    }
}

}  // namespace reader

using namespace reader;

extern "C" int reader_tree_qkv(const reader_dims *dims, const void *qkv, const int32_t *parents, const int32_t *seq_lens,
                               const int32_t *positions, const void *q_norm, const void *k_norm, float eps,
                               const float *cos_sin, int32_t max_positions, int32_t rot_dims, int32_t interleaved, void *q,
                               void *k_tree, void *v_tree, void *k_cache, void *v_cache, const int32_t *page_table,
                               int32_t *status, void *stream) {
    int err = 0;
    if (!dims_ok(dims, &err)) return err;
    if (dims->B == 0) return READER_OK;
    QkvParams p = {};
    int rc = qkv_prepare(dims, qkv, seq_lens, positions, q_norm, k_norm, eps, cos_sin, max_positions, rot_dims, interleaved, q, status, p);
    if (rc != READER_OK) return rc;
    if (!parents || (k_tree == nullptr) != (v_tree == nullptr)) return READER_EINVAL;
    if (!k_tree && !cache_ok(dims, k_cache, v_cache, page_table)) return READER_EINVAL;
    p.N = dims->B * dims->T;
    rc = rows_ok(dims, p.N);
    if (rc != READER_OK) return rc;
    p.parents = parents; p.page_table = page_table;
    p.k_tree = (uint16_t *)k_tree; p.v_tree = (uint16_t *)v_tree;
    p.k_cache = (uint16_t *)k_cache; p.v_cache = (uint16_t *)v_cache;
    forget_stale_error();
    return launch_qkv(p, (hipStream_t)stream) == hipSuccess ? READER_OK : READER_EHIP;
}

extern "C" int reader_prompt_qkv(const reader_dims *dims, int32_t N, const void *qkv, const int32_t *cu_tokens,
                                 const int32_t *seq_lens, const int32_t *positions, const void *q_norm, const void *k_norm,
                                 float eps, const float *cos_sin, int32_t max_positions, int32_t rot_dims,
                                 int32_t interleaved, void *q, void *k_cache, void *v_cache, const int32_t *page_table,
                                 int32_t *status, void *stream) {
    int err = 0;
    if (!dims_ok(dims, &err)) return err;
    int rc = rows_ok(dims, N);
    if (rc != READER_OK) return rc;
    if (dims->B == 0 || N == 0) return READER_OK;
    QkvParams p = {};
    rc = qkv_prepare(dims, qkv, seq_lens, positions, q_norm, k_norm, eps, cos_sin, max_positions, rot_dims, interleaved, q, status, p);
    if (rc != READER_OK) return rc;
    if (!cu_tokens || !cache_ok(dims, k_cache, v_cache, page_table)) return READER_EINVAL;
    p.N = N;
    p.cu_tokens = cu_tokens; p.page_table = page_table;
    p.k_cache = (uint16_t *)k_cache; p.v_cache = (uint16_t *)v_cache;
    forget_stale_error();
    return launch_qkv(p, (hipStream_t)stream) == hipSuccess ? READER_OK : READER_EHIP;
}

extern "C" size_t reader_prompt_workspace_bytes(const reader_dims *dims, int32_t N, int32_t max_seq_len) {
    int err = 0;
    if (!dims_ok(dims, &err) || rows_ok(dims, N) != READER_OK || max_seq_len < 0) return 0;
    const size_t wide = prompt_wide_workspace_bytes(dims->D), few = prompt_few_workspace_bytes(dims->D);
    return ((wide > few ? wide : few) + 255) & ~(size_t)255;
}

extern "C" int reader_prompt_rows(const reader_dims *dims, int32_t N, int32_t max_seq_len) {
    int err = 0;
    if (!dims_ok(dims, &err)) return err;
    const int rc = rows_ok(dims, N);
    if (rc != READER_OK) return rc;
    if (max_seq_len < 0 || (dims->variant != 0 && dims->variant != 1)) return READER_EINVAL;
    return prompt_rows(*dims, N, max_seq_len);
}

extern "C" int reader_prompt_attn(const reader_dims *dims, int32_t N, const void *q, const void *k_cache, const void *v_cache,
                                  const int32_t *page_table, const int32_t *cu_tokens, const int32_t *seq_lens, void *out,
                                  float *lse, int32_t max_seq_len, void *workspace, size_t workspace_bytes, int32_t *status,
                                  void *stream) {
    int err = 0;
    if (!dims_ok(dims, &err)) return err;
    const int rc = rows_ok(dims, N);
    if (rc != READER_OK) return rc;
    if (max_seq_len < 0 || (dims->variant != 0 && dims->variant != 1)) return READER_EINVAL;
    if (dims->B == 0 || N == 0) return READER_OK;
    if (!q || !cu_tokens || !seq_lens || !out || !cache_ok(dims, k_cache, v_cache, page_table)) return READER_EINVAL;
    if ((long long)dims->max_pages_per_seq * dims->page_size < max_seq_len) return READER_EINVAL;
    PromptParams p = {};
    p.q = (const uint16_t *)q; p.k_cache = (const uint16_t *)k_cache; p.v_cache = (const uint16_t *)v_cache;
    p.page_table = page_table; p.cu_tokens = cu_tokens; p.seq_lens = seq_lens;
    p.out = (uint16_t *)out; p.lse = lse; p.status = status; p.workspace = workspace;
    p.B = dims->B; p.N = N; p.Hq = dims->Hq; p.Hkv = dims->Hkv; p.G = dims->Hq / dims->Hkv; p.D = dims->D;
    p.max_pages = dims->max_pages_per_seq; p.max_seq_len = max_seq_len; p.num_pages = dims->num_pages;
    p.scale_log2 = softmax_scale_log2(*dims);
    if (dims->variant == 1) {
        if ((long long)N * dims->Hq > READER_MAX_TOKENS) return READER_EUNSUPPORTED;   // (threads of a launch)
    } else {
        if (!workspace || ((uintptr_t)workspace & 255) != 0) return READER_EWORKSPACE;
        if (workspace_bytes < reader_prompt_workspace_bytes(dims, N, max_seq_len)) return READER_EWORKSPACE;
    }
    p.g_rcp = 1.0f / (float)p.G;
    forget_stale_error();
    return launch_prompt(p, prompt_rows(*dims, N, max_seq_len), (hipStream_t)stream) == hipSuccess ? READER_OK : READER_EHIP;
}

static int key_weights_prepare(const reader_dims *dims, int32_t rows, const void *q, const float *lse, const void *k_cache,
                               const int32_t *page_table, const int32_t *seq_lens, float decay, float *weights,
                               int32_t max_positions, int32_t max_seq_len, int32_t *status, KeyWeightsParams &p) {
    if (max_positions < 0 || max_seq_len < 0 || !(decay >= 0.f && decay <= 1.f)) return READER_EINVAL;
    if (dims->Hkv > 65535) return READER_EUNSUPPORTED;                    // (a dimension of the grid)
    if ((rows > 0 && (!q || !lse)) || !seq_lens || !weights || !cache_ok(dims, k_cache, k_cache, page_table)) return READER_EINVAL;
    p.q = (const uint16_t *)q; p.lse = lse; p.k_cache = (const uint16_t *)k_cache;
    p.page_table = page_table; p.seq_lens = seq_lens; p.weights = weights; p.status = status;
    p.B = dims->B; p.T = dims->T; p.Hq = dims->Hq; p.Hkv = dims->Hkv; p.G = dims->Hq / dims->Hkv; p.D = dims->D;
    p.max_pages = dims->max_pages_per_seq; p.max_path = dims->max_path; p.num_pages = dims->num_pages;
    p.max_positions = max_positions; p.max_seq_len = max_seq_len;
    p.scale_log2 = softmax_scale_log2(*dims); p.decay = decay; p.g_rcp = 1.0f / (float)p.G;
    return READER_OK;
}

extern "C" int reader_key_weights(const reader_dims *dims, const void *q, const float *lse, const int32_t *path,
                                  const int32_t *accept_len, const void *k_cache, const int32_t *page_table,
                                  const int32_t *seq_lens, float decay, float *weights, int32_t max_positions,
                                  int32_t max_seq_len, int32_t *status, void *stream) {
    int err = 0;
    if (!dims_ok(dims, &err)) return err;
    if (dims->B == 0) return READER_OK;
    KeyWeightsParams p = {};
    const int rc = key_weights_prepare(dims, dims->B, q, lse, k_cache, page_table, seq_lens, decay, weights, max_positions, max_seq_len, status, p);
    if (rc != READER_OK) return rc;
    if (!path || !accept_len) return READER_EINVAL;
    p.path = path; p.accept_len = accept_len;
    forget_stale_error();
    return launch_key_weights(p, (hipStream_t)stream) == hipSuccess ? READER_OK : READER_EHIP;
}

extern "C" int reader_prompt_key_weights(const reader_dims *dims, int32_t N, const void *q, const float *lse,
                                         const int32_t *cu_tokens, int32_t window, const void *k_cache,
                                         const int32_t *page_table, const int32_t *seq_lens, float decay, float *weights,
                                         int32_t max_positions, int32_t max_seq_len, int32_t *status, void *stream) {
    int err = 0;
    if (!dims_ok(dims, &err)) return err;
    int rc = rows_ok(dims, N);
    if (rc != READER_OK) return rc;
    if (window < 0) return READER_EINVAL;
    if (window > READER_MAX_WINDOW) return READER_EUNSUPPORTED;
    if (dims->B == 0) return READER_OK;
    KeyWeightsParams p = {};
    rc = key_weights_prepare(dims, N, q, lse, k_cache, page_table, seq_lens, decay, weights, max_positions, max_seq_len, status, p);
    if (rc != READER_OK) return rc;
    if (!cu_tokens) return READER_EINVAL;
    p.cu_tokens = cu_tokens; p.N = N; p.window = window;
    forget_stale_error();
    return launch_key_weights(p, (hipStream_t)stream) == hipSuccess ? READER_OK : READER_EHIP;
}

// (layer, sequence, kv head) triples; each has `keep` list entries and a word in the workspace
static long long evict_units(const reader_dims *dims, int32_t num_layers) { return (long long)num_layers * dims->B * dims->Hkv; }

extern "C" size_t reader_kv_evict_workspace_bytes(const reader_dims *dims, int32_t num_layers, int32_t keep) {
    int err = 0;
    if (!dims_ok(dims, &err) || num_layers < 0 || keep < 0) return 0;
    return ((size_t)evict_units(dims, num_layers) * ((size_t)keep + 1) * sizeof(int32_t) + 255) & ~(size_t)255;
}

extern "C" int reader_kv_evict(const reader_dims *dims, int32_t num_layers, int32_t keep, int32_t recent, void *k_cache,
                               void *v_cache, const int32_t *page_table, int32_t *seq_lens, float *weights,
                               int32_t max_positions, void *workspace, size_t workspace_bytes, int32_t *status,
                               void *stream) {
    int err = 0;
    if (!dims_ok(dims, &err)) return err;
    if (num_layers < 1 || keep < 0 || recent < 0 || recent > keep || max_positions < 0) return READER_EINVAL;
    if (evict_units(dims, num_layers) > READER_MAX_EVICT_UNITS) return READER_EUNSUPPORTED;
    if (dims->B == 0) return READER_OK;
    if (!seq_lens || !weights || !cache_ok(dims, k_cache, v_cache, page_table)) return READER_EINVAL;
    if (!workspace || ((uintptr_t)workspace & 3) != 0 || workspace_bytes < reader_kv_evict_workspace_bytes(dims, num_layers, keep))
        return READER_EWORKSPACE;
    EvictParams p = {};
    p.k_cache = (uint16_t *)k_cache; p.v_cache = (uint16_t *)v_cache; p.page_table = page_table;
    p.seq_lens = seq_lens; p.weights = weights; p.status = status;
    p.old_len = (int32_t *)workspace;
    p.source = p.old_len + evict_units(dims, num_layers);
    p.NL = num_layers; p.B = dims->B; p.Hkv = dims->Hkv; p.D = dims->D;
    p.max_pages = dims->max_pages_per_seq; p.max_positions = max_positions; p.keep = keep; p.recent = recent;
    p.num_pages = dims->num_pages;
    forget_stale_error();
    return launch_kv_evict(p, (hipStream_t)stream) == hipSuccess ? READER_OK : READER_EHIP;
}

// C ABI entry points of the operators around the verification step (prompts, per-head norms and rotation, accumulated key
// weights, eviction): argument validation on the host and dispatch.  They are defined in include/reader.h.
#include <math.h>

#include "prompt_common.h"

namespace reader {

static float softmax_scale_log2(const reader_dims &d) {
    return (d.sm_scale > 0.f ? d.sm_scale : 1.0f / sqrtf((float)d.D)) * 1.44269504088896340736f;
}

// Wide loads and copies into LDS take 16 bytes: tensors start at a multiple of them.
template <class... Pointers>
static bool aligned(const Pointers *...p) { return (((uintptr_t)p | ...) & 15) == 0; }

// What both forms of the projections' operator check and fill.
static int qkv_prepare(const reader_dims *dims, const void *qkv, const int32_t *seq_lens, const int32_t *positions,
                       const void *q_norm, const void *k_norm, float eps, const float *cos_sin, int32_t max_positions,
                       int32_t rot_dims, int32_t interleaved, void *q, int32_t *status, QkvParams &p) {
    if (rot_dims < 0 || rot_dims > dims->D || max_positions < 0 || (interleaved != 0 && interleaved != 1)) return READER_EINVAL;
    if (rot_dims % 16 != 0) return READER_EUNSUPPORTED;
    if ((q_norm == nullptr) != (k_norm == nullptr)) return READER_EINVAL;
    if (q_norm && !(eps >= 0.f && eps <= 1.f)) return READER_EINVAL;
    if (!qkv || !seq_lens || !q || (rot_dims > 0 && !cos_sin)) return READER_EINVAL;
    if (!aligned(qkv, q_norm, k_norm, q) || (rot_dims > 0 && !aligned(cos_sin))) return READER_EINVAL;
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
    return k_cache && v_cache && page_table && dims->num_pages >= 1 && dims->max_pages_per_seq >= 1 && aligned(k_cache, v_cache);
}

// Query rows a workgroup takes (reader_prompt_rows): the shortest of six estimates, in us, of what the host knows (sequences of one
// length, the longest one's last tokens):
//   16, 32 rows: start and merge, and steps of 32 keys, which all blocks share out evenly (four wavefronts a compute unit); keys of
//     a call that do not stay in the caches come from memory for every block;
//   32, 64, 128 rows, blocks never cut: the longest block's steps, one after the other (with 32 rows two at a time; slower where every
//     compute unit has one of full length), or what all blocks' steps take the compute units;
//   256 rows: start, merge and imbalance, and per block what its tiles of 64 keys and its ends take, shared out evenly.
// The constants are fitted to 252 shapes (7 head layouts; 1 to 64 sequences of 1 to 3000 tokens on up to 30 K positions).  Some of them,
// 16, 32, 32 uncut, 64, 128 and 256 rows (32 query and 8 kv heads, D 128):
// one prompt of 100 tokens 16.2, 19.5, 6.2, 6.6, 8.4, 19.0; of 1500 220, 149, 58.6, 45.9, 51.4, 51.1; of 3000 696, 441, 194, 144,
// 100, 99.0; 16 of 300 214, 150, 75.9, 52.4, 43.7, 42.0; 256 tokens on 1000 positions 48.4, 37.5, 26.0, 35.4, 41.4, 31.4; 64 on 8
// K 58.6, 40.9, 136, 200, 230, 74.6; 32 sequences of 12 on 8 K 474, 324, 213, 239, 283, 173; 16 single tokens on 500 16.2, 18.8,
// 14.4, 16.8, 20.0, 25.4; on 2000 30.7, 32.5, 41.9, 52.4, 62.1, 39.9.  The estimates pick the fastest of the six on 223 of the 252
// and are 0.7 % behind it on average, 27 % at most (all of them: profiles/prompt_rows_sweep.txt).  They take max_seq_len for the
// longest sequence: where it is only a bound, one prompt of 100 tokens takes 18 us instead of 6, of 777 39 instead of 22, single
// tokens on 500 positions 14 to 16 instead of 10 to 13; 3000 tokens, batches of prompts and long contexts the same.
static int prompt_rows(const reader_dims &d, int32_t N, int32_t max_seq_len) {
    if (d.variant == 1) return 0;
    const int forced = tuning(READER_TUNE_PROMPT_ROWS), G = d.Hq / d.Hkv;
    if (forced == 16 || forced == 32 || forced == kUncut32 || forced == 64 || forced == 128 || forced == 256) return forced;
    if (d.B == 0 || N == 0) return 16;
    const double tokens = (double)N / d.B;                        // of a sequence
    const double longest = max_seq_len > tokens ? max_seq_len : tokens, average = longest - 0.5 * tokens;   // keys of a block
    const bool large = d.D == 128;
    auto blocks = [&](int rows) { return (double)d.Hkv * d.B * ceil(tokens / (rows / G)); };
    auto few = [&](int rows, double start, double step) {
        const bool far = (double)d.Hkv * d.B * longest * d.D * 4 > 64e6;
        const double from_memory = large ? 0.59 : 0.29;
        return start + (far && step < from_memory ? from_memory : step) * blocks(rows) * (average / 32 + 14) / kNumCU;
    };
    auto uncut = [&](int rows, double step, double step_busy, double all_steps) {
        const bool busy = blocks(rows) * average >= 0.8 * kNumCU * longest;
        const double chain = (busy ? step_busy : step) * (longest / (rows == 32 ? 64 : 32) + 0.5);
        const double all = all_steps * blocks(rows) * (average / 32 + (rows == 32 ? 6 : 4)) / kNumCU;
        return 5.5 + (chain > all ? chain : all);
    };
    const double parts = blocks(256) < kNumCU / 4 ? (large ? 20.0 : 12.0) : 0.0;     // (every range leaves records, nothing else)
    double best = (large ? 26.0 : 25.0) + parts + blocks(256) / kNumCU * (large ? 7.0 + 1.6 * (average / 64 + 0.5) : 4.0 + 0.763 * (average / 64 + 0.5));
    int rows = 256;
    auto offer = [&](int r, double us) {
        if (us < best) { best = us; rows = r; }
    };
    offer(16, large ? few(16, 13.7, 0.303) : few(16, 13.6, 0.156));
    offer(32, large ? few(32, 16.3, 0.457) : few(32, 15.3, 0.22));
    // (block numbers of the uncut kernels are counted with the threads of a launch)
    if (((long long)N / (32 / G) + d.B) * d.Hkv < (1 << 23)) {
        offer(kUncut32, large ? uncut(32, 0.98, 1.09, 0.33) : uncut(32, 0.70, 0.91, 0.22));
        offer(128, large ? uncut(128, 0.93, 1.2, 0.57) : uncut(128, 0.64, 0.8, 0.43));
        offer(64, large ? uncut(64, 0.85, 0.83, 0.45) : uncut(64, 0.56, 0.64, 0.29));
    }
    return rows;
}

static hipError_t launch_prompt(const PromptParams &p, int rows, hipStream_t stream) {
    switch (rows) {
        case 0: return launch_prompt_attn_scalar(p, stream);
        case 16: case 32: return launch_prompt_few(p, rows, stream);
        case kUncut32: case 64: case 128: return launch_prompt_mid(p, rows, stream);
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
    if (!aligned(k_tree, v_tree)) return READER_EINVAL;
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
    if (!q || !cu_tokens || !seq_lens || !out || !cache_ok(dims, k_cache, v_cache, page_table) || !aligned(q, out)) return READER_EINVAL;
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
    if ((rows > 0 && (!q || !lse)) || !seq_lens || !weights || !cache_ok(dims, k_cache, k_cache, page_table) || !aligned(q)) return READER_EINVAL;
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

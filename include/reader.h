/*
 * reader.h - C ABI of the MI355X (gfx950) draft-tree verification library for
 * READER (arXiv 2508.09072), the lossless retrieval-drafted speculative decoder.
 *
 * One verification step of the base model over a draft tree (Algorithm 1, "Verify
 * and accept"; Algorithm 5) is, per transformer layer, a tree-masked attention
 * (Section 3.2) and, once per step, a greedy acceptance of the longest draft path
 * that agrees with the base model (Algorithm 5, Appendix C) followed by the
 * append of that path's K/V rows to each sample's cache so that it stays tight
 * (Section 4.3, Algorithm 4).  This library is those three operations, the steps
 * right next to them (the base model's tokens from its logits, greedy or sampled
 * with coupled uniforms; the paper's periodic rearrangement of a padded cache;
 * compaction when the tree rows already sit in every layer's cache), and the
 * host-side retrieval drafter that makes draft trees from the short-term context.
 *
 * Conventions
 *  - Every pointer is a DEVICE pointer unless its name ends in `_host` or the
 *    comment of the entry point says otherwise (the drafter works on host memory).  All
 *    device buffers are borrowed: the caller allocates, owns and frees them.  On the
 *    device side the library
 *    allocates nothing, frees nothing and never synchronises; each call enqueues
 *    its kernels on `stream` (a hipStream_t passed as void*, NULL = default
 *    stream) and returns.  Results are valid once the stream reaches that point.
 *  - bf16 tensors are passed as `void*`; element (i,j,k,l) of a tensor of shape
 *    [A,B,C,D] sits at ((i*B + j)*C + k)*D + l (C order, no padding).
 *  - Return value: READER_OK (0) or a negative READER_E* code.  Argument checks
 *    happen on the host before anything is enqueued, so a failed call has no
 *    effect.  Nothing is printed, no exception crosses the boundary.
 *  - Data-dependent problems that only the device can see (a malformed tree, a
 *    page id outside the pool, an accepted length that does not fit) never fault:
 *    the kernel skips the offending item and ORs a READER_STATUS_* bit into the
 *    optional device word `status`.  In the attention a bad link of a tree counts as
 *    a root link and the cached keys behind a bad page id are left out of the sums;
 *    tree rows that live in the cache (in-cache layout) behind a bad page id leave
 *    the outputs of their sequence unspecified (finite or NaN, never a fault).
 *  - Tree convention: node 0 is the root = the last committed token (it comes
 *    from the base model, acceptance rate 1, Section 3.3); parents[b][0] = -1 and
 *    0 <= parents[b][i] < i.  Trees may differ between sequences; the paper's
 *    fixed per-batch shape is the case where all rows of `parents` are equal.
 *  - Grouped-query attention: query head hq reads kv head hq / (Hq / Hkv).
 *  - Paged cache: position j of sequence b lives in physical page
 *    page_table[b][j / page_size], slot j % page_size.
 *  - Threads: the compute entry points keep nothing between calls but a count of fused steps
 *    (each of them marks its workspace with a number of its own) and may be called
 *    from several host threads, each on its own stream and with its own workspace,
 *    outputs and status word; calls that share a workspace or write the same cache
 *    pages or lengths must be ordered by the caller (one stream, or events).
 *    reader_last_error_detail and the reader_profile_* hooks share one process-wide
 *    buffer and are meant for one thread.  The library reads no environment variable.
 *  - Size limits (a call beyond them returns READER_EUNSUPPORTED, nothing is enqueued):
 *    T <= READER_MAX_T, D in {64, 128}, page_size == READER_PAGE_SIZE, Hq / Hkv <= 16,
 *    B <= READER_MAX_B, num_pages * Hkv < 2^31, B * max_pages_per_seq < 2^31.
 */
#ifndef READER_H
#define READER_H

#include <stddef.h>
#include <stdint.h>

#ifdef __cplusplus
extern "C" {
#endif

enum {
    READER_OK = 0,
    READER_EINVAL = -1,       /* null pointer, non-positive size, inconsistent dims, malformed host tree */
    READER_EUNSUPPORTED = -2, /* a size outside what the kernels are built for */
    READER_EWORKSPACE = -3,   /* workspace pointer missing or too small */
    READER_EHIP = -4          /* the HIP runtime refused a launch */
};

enum {
    READER_STATUS_BAD_TREE = 1, /* parents[b][0] != -1 or parents[b][i] not in [0, i) */
    READER_STATUS_BAD_PAGE = 2, /* a page id outside [0, num_pages) was met */
    READER_STATUS_BAD_PATH = 4, /* accept_len/path entry out of range, or path longer than max_path */
    READER_STATUS_BAD_LENGTH = 8, /* a length, packed bound or position that the tensors, the page table or a table of positions do not hold */
    READER_STATUS_BAD_VALUE = 16, /* a value that the cache in 4 bits cannot hold: a NaN or an infinity */
    READER_STATUS_NO_PAGES = 32   /* the pool has fewer free pages than were asked for */
};

enum {
    READER_MAX_T = 128,  /* draft-tree nodes per sequence */
    READER_PAGE_SIZE = 16,
    READER_MAX_B = 4096, /* sequences per call (what the in-kernel prefix scan over the lengths is sized for) */
    READER_MAX_WINDOW = 65536,          /* query tokens per sequence of reader_prompt_key_weights */
    READER_MAX_EVICT_UNITS = 1 << 20,   /* (layer, sequence, kv head) triples of reader_kv_evict */
    READER_MAX_TOKENS = 1 << 25         /* rows of a packed batch */
};

/* Problem sizes; plain data, passed by const pointer (host memory). */
typedef struct reader_dims {
    int32_t B;                 /* sequences in the batch, 0..READER_MAX_B (0 = nothing to do) */
    int32_t T;                 /* draft-tree nodes per sequence, 1..READER_MAX_T */
    int32_t Hq;                /* query heads */
    int32_t Hkv;               /* kv heads, Hq % Hkv == 0, Hq / Hkv <= 16 */
    int32_t D;                 /* head dimension, 64 or 128 */
    int32_t page_size;         /* tokens per cache page, must be READER_PAGE_SIZE */
    int32_t max_pages_per_seq; /* row stride of page_table */
    int32_t max_path;          /* row stride of `path`: >= deepest node's depth + 1, <= T */
    int64_t num_pages;         /* pages in the pool (first dim of k_cache / v_cache) */
    float sm_scale;            /* softmax scale; <= 0 selects 1/sqrt(D) */
    int32_t variant;           /* 0 = default kernel selection.  1 = force the scalar reference
                                  kernel of reader_tree_attn (slow; for cross-checks only) */
} reader_dims;

/* Library version string (static storage). */
const char *reader_version(void);

/* Text for a READER_E* code (static storage). */
const char *reader_strerror(int code);

/* Which HIP call failed last and how, after a READER_EHIP return ("" if none so far; static storage). */
const char *reader_last_error_detail(void);

/*
 * Host-side check of the tree convention above on HOST arrays parents_host[B][T].
 * Pure function, no GPU needed.  READER_OK or READER_EINVAL.
 */
int reader_validate_tree(const int32_t *parents_host, int32_t B, int32_t T);

/*
 * Bytes of device workspace reader_tree_attn needs for these dims when no
 * sequence is longer than max_seq_len.  Pure host function.  Returns 0 when the
 * dims are invalid.  The workspace holds the partial (bf16 output normalised by its
 * own sum, running max, running sum) records of key ranges that were split across workgroups; its
 * contents are meaningless between calls and it may be shared by calls that are
 * ordered on one stream.
 */
size_t reader_workspace_bytes(const reader_dims *dims, int32_t max_seq_len);

/*
 * How reader_tree_attn would run these dims when no sequence is longer than max_seq_len: which of its
 * kernels, how many query rows a workgroup carries, into how many chunks the rows of a (sequence, kv head)
 * pair are cut, and how many ranges of key tiles the launch has (workgroups = key_ranges * row_chunks).
 * For benchmarks and profiles that name the kernel they time; the choice follows Section 3.2's
 * memory-bound / compute-bound distinction (few query rows: stream K/V with dedicated copy wavefronts;
 * many: all wavefronts on the matrix cores).  Pure host function; honours reader_tuning_override.
 * READER_OK, or the error reader_tree_attn would return for the dims.
 */
enum reader_attn_kernel {
    READER_ATTN_KERNEL_SCALAR = 0,          /* dims->variant = 1: the scalar reference kernel */
    READER_ATTN_KERNEL_ROWS128 = 1,         /* tree_attn_mfma_kernel<D, 4>: 128 rows, 4 computing + 4 copying wavefronts */
    READER_ATTN_KERNEL_ROWS256_WAVES8 = 2,  /* tree_attn_mfma_kernel<D, 8>: 256 rows, 8 wavefronts of 32 rows */
    READER_ATTN_KERNEL_ROWS256_WAVES4 = 3,  /* tree_attn_wide_kernel<D>: 256 rows, 4 wavefronts of 64 rows */
    READER_ATTN_KERNEL_SHORT = 4            /* tree_attn_short_kernel<D>: short problems, 128 rows, static grid */
};
typedef struct reader_attn_plan_t {
    int32_t kernel;                /* enum reader_attn_kernel */
    int32_t rows_per_workgroup;    /* 128 or 256 (short kernel: 128; 0 for the scalar kernel) */
    int32_t row_chunks;
    int32_t key_ranges;
} reader_attn_plan_t;
int reader_attn_plan(const reader_dims *dims, int32_t max_seq_len, reader_attn_plan_t *plan);

/*
 * Whether reader_verify_step of these dims is one launch (verify_short_join_kernel<D>) on a stream that is not being
 * captured: 1 or 0, or the error reader_attn_plan would return.  Pure host function; honours reader_tuning_override.
 */
int reader_step_is_one_launch(const reader_dims *dims, int32_t max_seq_len);

/*
 * Tree-masked attention (Section 3.2; Appendix C invariant 2).
 * For every sequence b, query head hq and tree node i:
 *     out[b,i,hq,:] = sum_j softmax_j( sm_scale * <q[b,i,hq,:], k_j> ) * v_j
 * where j runs over the seq_lens[b] cached positions of b (kv head hq/(Hq/Hkv))
 * and over the tree nodes that are i itself or an ancestor of i.
 *
 *   q            bf16 [B, T, Hq, D]                     in
 *   k_tree,v_tree bf16 [B, T, Hkv, D]                   in   K/V rows of the tree nodes; or both NULL:
 *                the in-cache layout (Section 4.3), where the forward pass wrote the row of node n
 *                of sequence b at cache position seq_lens[b] + n; page_table must then map pages
 *                for [0, seq_lens[b] + T) and max_pages_per_seq * page_size >= max_seq_len + T
 *   k_cache,v_cache bf16 [num_pages, Hkv, page_size, D] in   paged prefix cache
 *   page_table   i32 [B, max_pages_per_seq]             in   must map pages for [0, seq_lens[b])
 *   seq_lens     i32 [B]                                in   prefix length L_b, tree rows excluded
 *   parents      i32 [B, T]                             in
 *   out          bf16 [B, T, Hq, D]                     out  fp32 accumulation, rounded to nearest even
 *   lse          f32 [B, Hq, T] or NULL                 out  natural-log sum of exp of the scaled scores
 *   max_seq_len  upper bound of seq_lens[b] (host value) used to size the launch; a sequence
 *                longer than this is truncated to it and nothing faults
 *   workspace    >= reader_workspace_bytes(dims, max_seq_len) bytes, 256-byte aligned
 *   status       i32 [1] or NULL                        in/out  READER_STATUS_* bits are ORed in
 *
 * Arithmetic: bf16 products accumulated in fp32 on the matrix cores; softmax
 * weights are rounded to bf16 before they multiply V.  Rows of a malformed tree
 * are computed as if the bad node were a root.
 */
int reader_tree_attn(const reader_dims *dims,
                     const void *q, const void *k_tree, const void *v_tree,
                     const void *k_cache, const void *v_cache,
                     const int32_t *page_table, const int32_t *seq_lens, const int32_t *parents,
                     void *out, float *lse,
                     int32_t max_seq_len, void *workspace, size_t workspace_bytes,
                     int32_t *status, void *stream);

/*
 * reader_tree_attn for callers that cannot allocate device memory or hand in a workspace: code
 * under HIP graph capture, tight serving loops, harnesses that forbid hipMalloc.  Same arguments
 * (without workspace and workspace_bytes), same kernels and the same results as reader_tree_attn
 * with dims->variant = 0; the partial records go to a workspace of READER_NOALLOC_WORKSPACE_BYTES
 * that is part of the library's device code (every GPU the library is used on holds its own copy
 * until the process ends).  The call allocates and frees nothing, on the host or the device.
 *
 *  - Dims whose reader_workspace_bytes(dims, max_seq_len) exceeds READER_NOALLOC_WORKSPACE_BYTES
 *    are refused with READER_EWORKSPACE (reader_last_error_detail says by how much).  The planner
 *    keeps key ranges x row chunks within the number of compute units, so the records never need
 *    more than 34.7 MB and the limit covers every shape with B * Hkv up to about 600,000 (the
 *    header holds 8 bytes per (sequence, kv head)); more ranges forced with
 *    reader_tuning_override can exceed it.
 *  - All calls on one GPU share that GPU's workspace: calls that may overlap in time (different
 *    streams, or host threads without ordering) race on it and must be ordered by the caller.
 *  - The first call on a device looks up the workspace's device address (this may load the
 *    library's device code).  A call with dims->B == 0 does only that and is the way to set a
 *    device up ahead of time, outside any graph capture.
 * dims->variant must be 0.  Returns as reader_tree_attn, READER_EUNSUPPORTED for a device index
 * above 63.
 */
#define READER_NOALLOC_WORKSPACE_BYTES (40u << 20)
int reader_tree_attn_noalloc(const reader_dims *dims,
                             const void *q, const void *k_tree, const void *v_tree,
                             const void *k_cache, const void *v_cache,
                             const int32_t *page_table, const int32_t *seq_lens, const int32_t *parents,
                             void *out, float *lse,
                             int32_t max_seq_len, int32_t *status, void *stream);

/*
 * Greedy lossless acceptance (Algorithm 5; Appendix C invariants 2 and 3).
 * target_tokens[b][i] is the base model's own next token after the prefix that
 * ends at node i.  A non-root node is accepted iff its parent is accepted and
 * draft_tokens[b][i] == target_tokens[b][parents[b][i]]; draft_tokens[b][0] is
 * ignored.  Among accepted nodes the deepest wins, the lowest node id among
 * equally deep ones (siblings may carry equal tokens, Section 4.2 "deepening").
 *
 *   draft_tokens, target_tokens, parents   i32 [B, T]       in
 *   accept_len   i32 [B]            out  number of accepted non-root nodes, 0..max_path-1
 *   path         i32 [B, max_path]  out  node ids root..terminal, then -1
 *   bonus_token  i32 [B]            out  target token at the terminal node (always committed)
 *   status       i32 [1] or NULL    in/out
 *
 * A path deeper than max_path-1 is cut at max_path-1 and READER_STATUS_BAD_PATH is set.
 * Integer work; results are exact.
 */
int reader_accept_path(const reader_dims *dims,
                       const int32_t *draft_tokens, const int32_t *target_tokens,
                       const int32_t *parents,
                       int32_t *accept_len, int32_t *path, int32_t *bonus_token,
                       int32_t *status, void *stream);

/*
 * Compaction of the accepted path into the cache (Section 4.3; Algorithm 4, done
 * every step so that no padding ever enters a sample's cache).  For every b and
 * j = 0..accept_len[b]: the K and V rows (all kv heads) of tree node path[b][j]
 * are copied to cache position seq_lens[b] + j, then seq_lens[b] += accept_len[b] + 1.
 * The root row (j = 0) is included: its K/V were first computed in this step.
 *
 *   k_tree, v_tree   bf16 [B, T, Hkv, D]                    in
 *   path             i32 [B, max_path], accept_len i32 [B]  in
 *   k_cache, v_cache bf16 [num_pages, Hkv, page_size, D]    in/out
 *   page_table       i32 [B, max_pages_per_seq]             in   must map pages for
 *                                                                [0, seq_lens[b] + accept_len[b] + 1)
 *   seq_lens         i32 [B]                                in/out
 *   status           i32 [1] or NULL                        in/out
 *
 * A sequence whose accept_len, path entry, target position or page id is out of
 * range is left untouched (cache and seq_lens) and a status bit is set.  Bit-exact copy.
 */
int reader_kv_compact(const reader_dims *dims,
                      const void *k_tree, const void *v_tree,
                      const int32_t *path, const int32_t *accept_len,
                      void *k_cache, void *v_cache, const int32_t *page_table,
                      int32_t *seq_lens, int32_t *status, void *stream);

/*
 * Compaction in the in-cache layout, all layers of the model in one call (Section 4.3;
 * Algorithm 4 applied every step).  The step's forward pass wrote the draft tree's K/V rows
 * behind each sequence in every layer's cache: node n of sequence b at position
 * seq_lens[b] + n.  For every b, layer, kv head and j = 1..accept_len[b], position
 * seq_lens[b] + j receives the row that position seq_lens[b] + path[b][j] held before the
 * call (the root, j = 0, is in place); then seq_lens[b] += accept_len[b] + 1.  Rows behind the
 * new length keep what they held.  The move is done in place: node ids increase along a path
 * (a parent precedes its children), so path[b][j] >= j and no row is overwritten before it
 * has been read.
 *
 *   num_layers       >= 0 (0: only the lengths are updated)
 *   path             i32 [B, max_path], accept_len i32 [B]               in
 *   k_cache, v_cache bf16 [num_layers, num_pages, Hkv, page_size, D]     in/out
 *   page_table       i32 [B, max_pages_per_seq]   in   must map pages for every position
 *                                                      the call touches
 *   seq_lens         i32 [B]                      in/out
 *   status           i32 [1] or NULL              in/out
 *
 * A sequence whose accept_len is out of range, whose path does not start at node 0 or does
 * not increase strictly, or that would touch a position outside the page table or a page id
 * out of range is left untouched (cache and seq_lens) and READER_STATUS_BAD_PATH /
 * READER_STATUS_BAD_PAGE is set.  Bit-exact copy.  dims->Hq and dims->sm_scale are not used.
 * One kernel launch: the workgroup of a sequence that finishes last writes its new length, found through
 * per-sequence counters that are device memory of the library (zero between calls).  Two calls that run on
 * one GPU at the same time (different streams) would share those counters: order them.
 * Returns READER_OK, READER_EINVAL (bad dims, num_layers outside 0..65535, null pointer).
 */
int reader_kv_compact_layers(const reader_dims *dims, int32_t num_layers,
                             const int32_t *path, const int32_t *accept_len,
                             void *k_cache, void *v_cache, const int32_t *page_table,
                             int32_t *seq_lens, int32_t *status, void *stream);

/*
 * One whole verification step (Algorithm 5: base-model pass over the draft tree, longest
 * accepted path; Section 4.3 / Algorithm 4: the accepted rows join the cache), with the
 * arguments, layouts, results and status bits of
 *     reader_tree_attn -> reader_accept_path -> reader_kv_compact
 * called in that order on one stream, but in two kernel launches instead of four (three
 * where the four-wavefront kernel runs): the last launch merges the attention partials, accepts
 * a path per sequence and compacts it.  Most short problems are one launch (reader_step_is_one_launch),
 * whose workgroups wait for one another (never without bound: whoever arrives last does what others
 * have left), except on a stream that is being captured: two there, with the same results.  target_tokens are an input here too
 * (the base model's tokens come from outside this library), so the attention output is not
 * consulted by the acceptance.
 * k_cache, v_cache and seq_lens are read by the attention and then updated by the
 * compaction: nothing is appended before the attention of every sequence has been computed, so
 * sequences may share pages as the three calls let them, a partly filled one among forks of
 * unequal length too.  dims->variant must be 0.  Errors as for the three calls.
 *
 * k_tree and v_tree both NULL: the in-cache layout of reader_tree_attn, one layer.  The step
 * is then reader_tree_attn -> reader_accept_path -> reader_kv_compact_layers(num_layers = 1)
 * on k_cache, v_cache [num_pages, Hkv, page_size, D]: the accepted rows move in place (one
 * more small launch, except where the step is one).  A model with several layers runs the attention of each layer, and
 * after the last one reader_accept_path and one reader_kv_compact_layers over all of them.
 */
int reader_verify_step(const reader_dims *dims,
                       const void *q, const void *k_tree, const void *v_tree,
                       void *k_cache, void *v_cache,
                       const int32_t *page_table, int32_t *seq_lens,
                       const int32_t *parents,
                       const int32_t *draft_tokens, const int32_t *target_tokens,
                       void *out, float *lse,
                       int32_t *accept_len, int32_t *path, int32_t *bonus_token,
                       int32_t max_seq_len, void *workspace, size_t workspace_bytes,
                       int32_t *status, void *stream);

/*
 * Periodic rearrangement of a padded cache (Section 4.3; Algorithm 4, KVCacheRearrange).
 * The padded layout is the one the paper starts from: every sample owns S slots, all
 * samples append at one common position, and a sample that accepted fewer tokens than
 * the longest acceptance of a step is padded.  Which slots hold a token is bookkeeping
 * (`valid`), never read off the values.  In place, for every sample b and layer l:
 *     the rows of the valid positions move to the front, in their order;
 *     every later row up to the old extent (last valid position + 1) becomes zero;
 *     rows past the old extent, and rows in front of the first hole, are not touched.
 * valid[b] becomes ones-then-zeros and new_len[b] the number of valid positions.
 *
 *   k_pad, v_pad  bf16 [NL, B, S, Hkv, D]   in/out   NL layers share one validity map
 *   valid         u8   [B, S]               in/out   nonzero = the slot holds a token
 *   new_len       i32  [B]                  out
 *   scratch       >= reader_kv_rearrange_scratch_bytes(B, S) bytes of device memory,
 *                 4-byte aligned; contents meaningless between calls
 * D must be 64 or 128 and NL * B * (Hkv + 1) below 2^31 (READER_EUNSUPPORTED otherwise).
 * Two launches (scan of the flags; the moves and the clearing).  Returns READER_OK or a READER_E* code
 * (nothing is enqueued then).
 */
size_t reader_kv_rearrange_scratch_bytes(int32_t B, int32_t S);
int reader_kv_rearrange(int32_t NL, int32_t B, int32_t S, int32_t Hkv, int32_t D,
                        void *k_pad, void *v_pad, uint8_t *valid, int32_t *new_len,
                        void *scratch, size_t scratch_bytes, void *stream);

/*
 * The base model's greedy tokens from its logits (Algorithm 5, "compare base logits with
 * drafted tokens"): target_tokens[r] = argmax over v of logits[r][v], for the B*T rows of
 * a verification step; the result is the target_tokens input of reader_accept_path.
 *
 *   logits         bf16 [rows, V]   in    compared exactly as bf16 values
 *   target_tokens  i32  [rows]      out   lowest index among equal maxima; a NaN is never
 *                                         the maximum (a row of NaNs gives 0)
 * Returns READER_OK or READER_EINVAL (rows < 0, V < 1, null pointer).
 */
int reader_target_argmax(int32_t rows, int32_t V, const void *logits, int32_t *target_tokens, void *stream);

/*
 * The base model's tokens under a sampling policy (Appendix C, randomized decoding).  The
 * policy is a map F(distribution, u) fed with one uniform per decoding position, and the
 * speculative run draws with the same uniforms as the plain run, which makes the two runs
 * emit the same tokens.  F is inverse-CDF sampling of softmax(logits / temperature):
 *   target_tokens[b][n] = lowest k with  sum_{v <= k} w_v  >  u * sum_v w_v,
 *   w_v = exp((logits[b][n][v] - max_v logits[b][n][v]) / temperature),
 *   u = uniforms[b][depth(n)]   (the root has depth 0; every node of one depth stands for the
 *                                same position and therefore draws with the same uniform).
 * The result is the target_tokens input of reader_accept_path, whose bonus token is then the
 * policy's own draw at the first position the draft does not cover.  Top-k / top-p filtering
 * is not applied.
 *
 *   logits         bf16 [B, T, V]  in    a NaN carries no probability; a +inf logit takes all of
 *                                        it (shared equally among the +inf tokens of the row)
 *   parents        i32  [B, T]     in    as for reader_tree_attn; a pointer that does not lead
 *                                        towards the root ends the depth walk there
 *   uniforms       f32  [B, T]     in    values in [0, 1); entry d serves depth d
 *   temperature    in [READER_MIN_TEMPERATURE, READER_MAX_TEMPERATURE] (below the lower end the
 *                  policy is the arg max in all but name: use reader_target_argmax)
 *   target_tokens  i32  [B, T]     out   a token of zero weight is never returned; a row
 *                                        without any weight gives 0
 * Sums are formed in fp32 (blocks of 512 tokens, then over the blocks): where u * total lies
 * within rounding (about 1e-5 of the total) of a boundary between two tokens' cumulative
 * weights, either of them may be returned.
 * Returns READER_OK or READER_EINVAL (B < 0, T outside 1..READER_MAX_T, V outside
 * 1..READER_MAX_SAMPLE_V, temperature outside its range or not a number, null pointer).
 */
#define READER_MAX_SAMPLE_V 4194304
#define READER_MIN_TEMPERATURE 1e-6f
#define READER_MAX_TEMPERATURE 1e6f
int reader_target_sample(int32_t B, int32_t T, int32_t V, const void *logits, const int32_t *parents,
                         const float *uniforms, float temperature, int32_t *target_tokens, void *stream);

/*
 * Host-side retrieval drafter over the short-term context (Section 4.2; Algorithm 2 with the
 * trie as its only structure).  Everything below runs on the CPU with HOST pointers; it makes
 * the token and parent arrays a verification step takes.  Not thread-safe per trie.
 *
 * The trie holds every n-gram of up to max_depth tokens of the sequences inserted so far, with
 * the number of times each was seen; inserting n tokens costs O(n * max_depth).
 * Looking up a context: the longest tail of the context (at most max_depth - 1 tokens, at least
 * one) that is in the trie and has a continuation; a tail that is not there loses its first
 * token and is tried again.  Continuations are ranked by descending count, equal counts in the
 * order they were first seen.
 */
typedef struct reader_trie reader_trie;
/* max_depth in 2..4096; NULL on a bad argument or when memory runs out */
reader_trie *reader_trie_create(int32_t max_depth);
void reader_trie_destroy(reader_trie *trie);   /* NULL is allowed */
/* number of nodes including the root, -1 for NULL */
int64_t reader_trie_nodes(const reader_trie *trie);
/* READER_OK, READER_EINVAL (NULL trie, n < 0, NULL tokens), READER_EUNSUPPORTED (out of memory) */
int reader_trie_insert(reader_trie *trie, const int32_t *tokens, int64_t n);
/*
 * SearchPath (Algorithm 2): starting from the context `suffix`, up to `depth` times take the
 * best-ranked continuation of the current context and append it to the context.  Writes the k
 * tokens found to path_tokens[0..k) and returns k (0 <= k <= depth), or -1 on a bad argument.
 */
int32_t reader_trie_search_path(const reader_trie *trie, const int32_t *suffix, int32_t n_suffix, int32_t depth,
                                int32_t *path_tokens);
/*
 * Draft tree by depth-first extraction (Section 4.2): the root (node 0) is the last token of
 * `suffix`; below it the continuations of the context, most frequent first, depth-first, at
 * most max_depth levels and `budget` nodes in all.  Nodes are numbered in the order they are
 * visited, so a parent precedes its children.  tokens, parents: i32 [budget] out.
 * Returns the number of nodes (>= 1), or -1 on a bad argument (n_suffix < 1, budget < 1, ...).
 */
int32_t reader_trie_extract_tree(const reader_trie *trie, const int32_t *suffix, int32_t n_suffix,
                                 int32_t max_depth, int32_t budget, int32_t *tokens, int32_t *parents);
/*
 * Attaches a path as one chain below node at_node of a tree of n_nodes nodes stored in arrays
 * of `capacity` entries (the widening and deepening of Section 4.2 attach one retrieved
 * path at the root, or at a drafted node); tokens that do not fit are dropped.  Returns the
 * new number of nodes, or -1 on a bad argument.
 */
int32_t reader_tree_attach_path(int32_t *tokens, int32_t *parents, int32_t n_nodes, int32_t capacity,
                                int32_t at_node, const int32_t *path_tokens, int32_t k);
/*
 * Self-repetition metric (Section 4.1): a pointer walks the response; at each stop the longest
 * run of tokens starting at the pointer that also occurs in the prompt or in the part of the
 * response already walked (entirely inside it) is skipped, or one token if there is none.
 * Returns response tokens / number of stops (0 for an empty response, -1 on a bad argument).
 */
double reader_self_repetition(const int32_t *prompt, int64_t n_prompt, const int32_t *response, int64_t n_response);

/*
 * Tree-shape selection (Appendix E; objective of Theorem 1, Section 3.3).  Host pointers, no GPU.
 * A seed tree (parents as everywhere: parents[0] = -1, 0 <= parents[i] < i) carries per node an
 * acceptance frequency alpha[i] (alpha[0] = 1 for the root; a child's is at most its parent's) and
 * an effective drafting time t_draft[i] (Lemma 2; t_draft[0] is ignored).  T_n is the seed tree after
 * n removals, each of the leaf with the lowest alpha (equal alphas: the highest node id), so
 * every T_n is a prefix subtree of the seed tree.  Its modelled throughput is
 *     ( sum of alpha_i over its nodes ) / ( sum of t_draft_i over its non-root nodes + tv[|T_n| - 1] ),
 * tv[k - 1] = measured verification time of a tree of k nodes (same unit as t_draft), k = 1..T.
 *
 * reader_tree_prune_order writes the removal order (T - 1 node ids) and returns T - 1.
 * reader_tree_select returns the pruning level n* with the best throughput and marks the nodes of
 * T_n* in keep[T] (1 = stays).  exhaustive != 0 scores every n; otherwise a golden-section search
 * is run, which assumes that the curve rises and then falls (Appendix E: close to unimodal) and
 * scores O(log T) trees: the way to go when a score is a benchmark run.  *throughput and
 * *evaluations (both optional) receive the best score and the number of trees scored.
 * Both return -1 on a bad argument (malformed tree, null pointer, negative or undefined value,
 * tv not positive) or when memory runs out.
 */
int32_t reader_tree_prune_order(const int32_t *parents, const float *alpha, int32_t T, int32_t *order);
int32_t reader_tree_select(const int32_t *parents, const float *alpha, const float *t_draft, const float *tv,
                           int32_t T, int32_t exhaustive, int32_t *keep, double *throughput, int32_t *evaluations);

/*
 * Measurement hooks for benchmarks (not operations of the method).  While enabled,
 * every reader_tree_attn / reader_verify_step call launches its main streaming kernel
 * with a HIP event pair that takes the kernel's own start and end time stamps (the
 * later launches of the call are outside the pair; in a fused step whose first launch
 * does more than attend, the pair spans that too).
 * reader_profile_collect waits for the recorded events (it synchronises the host with
 * them), adds up the elapsed times of all pairs recorded since the last collect into
 * *kernel_ms_sum, stores their count in *launches, and forgets them.  The event
 * objects are host-side handles owned by the library; at most 65536 pairs are kept
 * between collects (further launches are simply not timed).  Not thread-safe.
 * reader_profile_collect_each does the same but hands out every pair's time: ms_each
 * (host, float [capacity]) receives the first min(count, capacity) times in launch
 * order, *launches the count; READER_EINVAL for a null pointer or capacity < 0.
 */
int reader_profile_enable(int32_t on);
int reader_profile_collect(double *kernel_ms_sum, int32_t *launches);
int reader_profile_collect_each(float *ms_each, int32_t capacity, int32_t *launches);

/*
 * What this GPU gives the two things the attention kernels are made of, for the roofline discussion
 * (not an operation of the method).  Runs two bare loops on `stream` and waits for them:
 *   - every compute unit copies 32 KB tiles of `src` into a ring of LDS buffers with the instruction
 *     and the ring depth of the attention kernel and does nothing else: *hbm_read_gbs (src should be
 *     larger than the last-level cache, 256 MB, for the figure to be an HBM figure; the first
 *     src_bytes rounded down to a multiple of 8 MB are read);
 *   - one wavefront per SIMD issues the matrix instruction (v_mfma_f32_32x32x16_bf16) back to back on
 *     register operands: *mfma_bf16_tflops, and the shader clock the part runs at under that load in
 *     *mfma_clock_mhz (it lowers its clock under matrix load).
 *   src      device, src_bytes >= 32 MB, read only;  scratch  device, >= 262160 bytes, overwritten
 *   the three results are HOST doubles.
 * Creates and destroys two events; synchronises the host with the stream.  READER_OK, READER_EINVAL
 * (null pointer, sizes too small), READER_EHIP.
 */
int reader_measure_peaks(const void *src, size_t src_bytes, void *scratch, size_t scratch_bytes,
                         double *hbm_read_gbs, double *mfma_bf16_tflops, double *mfma_clock_mhz, void *stream);

/*
 * Launch-planner overrides for tests and experiments (not operations of the method; a caller
 * never needs them).  The planner of reader_tree_attn / reader_verify_step picks the number of
 * query rows per workgroup, the number of key ranges, the cost it books for the start of a
 * (sequence, kv head) pair when it cuts the ranges, and 32- or 64-bit arithmetic for the cut,
 * all from the dims alone.  An override replaces one of these choices for every later call of
 * the process (reader_workspace_bytes included, so sizes stay consistent) until it is cleared
 * with a negative value.  Every choice gives the same results up to rounding; only the speed
 * and the code path differ.  Stored atomically: a call sees the old or the new value.
 *   READER_TUNE_ATTN_ROWS       128 or 256 query rows per workgroup (other values: planner decides)
 *   READER_TUNE_ATTN_RANGES     >= 1 key ranges asked for (capped at the number of compute units)
 *   READER_TUNE_ATTN_PAIR_COST  0..64 tile times booked per pair beyond its tiles
 *   READER_TUNE_ATTN_PAIR_FRONT how many of them are booked to the workgroup that starts the pair (the rest to
 *                               the one that finishes it); capped at the pair cost
 *   READER_TUNE_ATTN_AXIS64     1 = cut the ranges in 64-bit arithmetic even where 32 bits suffice
 *   READER_TUNE_ATTN_WIDE       which kernel 256-row workgroups run: 1 = four wavefronts with 64 rows each (one per
 *                               SIMD, the accumulation registers managed by hand), 0 = eight with 32 rows each;
 *                               the planner takes the first at head dimension 128 and the second at 64
 *   READER_TUNE_ATTN_SHORT      0 = never the kernel for short problems, n >= 1 = always, with n shares per pair (n up
 *                               to 1024, and at most 240 tiles per share); any other override above keeps it out
 *   READER_TUNE_JOIN            0 = reader_verify_step of a short problem never waits inside a launch, n >= 1 = its workgroups
 *                               wait for (n - 1) / 100 us at most (1: whoever finds another one missing leaves at once; never more
 *                               than 10 ms), the one that appends four times as long
 *   READER_TUNE_JOIN_SPREAD     1 = the shares of a pair run on different XCDs there (0 or cleared: on one)
 *   READER_TUNE_PROMPT_ROWS     one of the values of reader_prompt_rows: 16, 32, READER_PROMPT_ROWS_32_UNCUT, 64, 128 or 256 (other
 *                               values: planner decides); of the attention over the cache in 4 bits 16, 128, 256 (cut into ranges;
 *                               18: 16 rows, half as many ranges), 17, READER_PROMPT_ROWS_32_UNCUT, 65 (16, 32, 64 rows, not cut)
 * Returns READER_OK, or READER_EINVAL for an unknown `which`.
 */
enum {
    READER_TUNE_ATTN_ROWS = 0,
    READER_TUNE_ATTN_RANGES = 1,
    READER_TUNE_ATTN_PAIR_COST = 2,
    READER_TUNE_ATTN_AXIS64 = 3,
    READER_TUNE_ATTN_WIDE = 4,
    READER_TUNE_ATTN_PAIR_FRONT = 5,
    READER_TUNE_ATTN_SHORT = 6,
    READER_TUNE_JOIN = 7,
    READER_TUNE_JOIN_SPREAD = 8,
    READER_TUNE_PROMPT_ROWS = 9,
    READER_TUNE_COUNT_ = 10
};
int reader_tuning_override(int32_t which, int32_t value);

/*
 * ------------------------------------------------------------------ around the verification step
 * A program fills the paged cache from its prompts, decodes over it, and may keep it within a budget.
 *
 * Packed prompts: the new tokens of all sequences are rows of one tensor, sequence b's are rows
 * cu_tokens[b] .. cu_tokens[b + 1] - 1 (i32 [B + 1], not decreasing, cu_tokens[0] >= 0, cu_tokens[B] <= N); rows
 * in front of the first and behind the last sequence are padding and stay as they were.  A sequence may have no new
 * tokens.  New keys and values go behind the seq_lens[b] positions that the cache holds (as a draft tree's do in the
 * in-cache layout); every layer's calls see the same seq_lens, and the caller adds the new tokens to it after the last
 * layer.
 *
 * Bounds out of order or of range, and negative lengths, set READER_STATUS_BAD_LENGTH, whoever they are of.  A bound out
 * of range counts as the nearest of 0 and N.  A sequence whose bounds go back has no tokens, and in such a batch a row
 * may be taken for that of either of two sequences that claim it, or be left as it was; nothing but rows of the batch
 * and of its sequences is written.  (The key weights leave a sequence whose bounds are wrong as it is.)
 *
 * bf16 tensors and the rotation table start at a multiple of 16 bytes (READER_EINVAL otherwise).  No output overlaps an
 * input, but for what is named in/out.
 *
 * Rotation table: f32 [max_positions, rot_dims], row `pos` holds rot_dims / 2 cosines and then as many sines of that
 * position's angles (made by the caller, in 64 bits for far positions).  The first rot_dims values of a head are
 * turned (rot_dims a multiple of 16, 0: none), pair i by angle i: values i and i + rot_dims / 2, or with
 * `interleaved` values 2 i and 2 i + 1:  (a, b) -> (a cos - b sin, b cos + a sin).
 *
 * Norm weights: bf16 [D], or both NULL: no norm.  y = w * x / sqrt(mean(x^2) + eps) over the D values of each head, in
 * front of the rotation.  eps in [0, 1].  fp32 throughout, one rounding to nearest even at the end; values of heads
 * that nothing is done to, and v, keep their bits.
 */

/*
 * Queries, keys and values of a draft tree's nodes from their projections, as reader_tree_attn and reader_verify_step
 * take them.  The position of a node is the root's plus the node's depth.
 *
 *   qkv          bf16 [B, T, Hq + 2 Hkv, D]   in   query heads, key heads, value heads
 *   parents      i32 [B, T]                   in
 *   seq_lens     i32 [B]                      in   cached positions: the root's position, unless `positions` is given
 *   positions    i32 [B] or NULL              in   position of the root (a cache that rows were evicted from is shorter
 *                                                  than the text)
 *   q_norm, k_norm  bf16 [D], both or neither in
 *   cos_sin      f32 [max_positions, rot_dims] in  (may be NULL if rot_dims is 0)
 *   q            bf16 [B, T, Hq, D]           out
 *   k_tree, v_tree  bf16 [B, T, Hkv, D]       out  or both NULL: the in-cache layout, node n at cache position
 *                                                  seq_lens[b] + n of
 *   k_cache, v_cache  bf16 [num_pages, Hkv, page_size, D]  out, page_table i32 [B, max_pages_per_seq] in (else unused)
 *   status       i32 [1] or NULL              in/out
 *
 * A bad link counts as a link to the root (READER_STATUS_BAD_TREE).  A node whose position the rotation table does not
 * hold is left out (READER_STATUS_BAD_LENGTH); one that the page table does not hold (BAD_LENGTH) or whose page id is out of
 * range (BAD_PAGE) gets its q but no K/V rows.  dims->sm_scale and max_path are not used.  One launch.
 */
int reader_tree_qkv(const reader_dims *dims, const void *qkv, const int32_t *parents, const int32_t *seq_lens,
                    const int32_t *positions, const void *q_norm, const void *k_norm, float eps,
                    const float *cos_sin, int32_t max_positions, int32_t rot_dims, int32_t interleaved,
                    void *q, void *k_tree, void *v_tree, void *k_cache, void *v_cache,
                    const int32_t *page_table, int32_t *status, void *stream);

/*
 * The same for packed prompts: row t of sequence b, its i-th new token, has position seq_lens[b] + i (positions[b] + i if
 * `positions` is given) and its K/V rows go to cache position seq_lens[b] + i.
 *
 *   qkv          bf16 [N, Hq + 2 Hkv, D]      in
 *   cu_tokens    i32 [B + 1]                  in
 *   q            bf16 [N, Hq, D]              out
 *   k_cache, v_cache  bf16 [num_pages, Hkv, page_size, D]  out
 * The rest as above; dims->T and max_path have to be valid and are not used.  One launch.
 */
int reader_prompt_qkv(const reader_dims *dims, int32_t N, const void *qkv, const int32_t *cu_tokens,
                      const int32_t *seq_lens, const int32_t *positions, const void *q_norm, const void *k_norm,
                      float eps, const float *cos_sin, int32_t max_positions, int32_t rot_dims, int32_t interleaved,
                      void *q, void *k_cache, void *v_cache, const int32_t *page_table, int32_t *status, void *stream);

/*
 * Causal attention of packed prompts over the paged cache: whole prompts (seq_lens[b] = 0), the next chunk of longer
 * ones, single tokens, or all of them in one call.  The i-th new token of sequence b attends to cache positions
 * 0 .. seq_lens[b] + i, its own among them (the keys and values of the new tokens are in the cache already):
 *     out[t, hq, :] = sum_j softmax_j( sm_scale * <q[t, hq, :], k_j> ) * v_j
 *
 *   q            bf16 [N, Hq, D]                            in
 *   k_cache, v_cache  bf16 [num_pages, Hkv, page_size, D]   in
 *   page_table   i32 [B, max_pages_per_seq]                 in   must map pages for [0, seq_lens[b] + new tokens)
 *   cu_tokens    i32 [B + 1], seq_lens i32 [B]              in
 *   out          bf16 [N, Hq, D]                            out  fp32 accumulation, rounded to nearest even
 *   lse          f32 [N, Hq] or NULL                        out  natural-log sum of exp of the scaled scores
 *   max_seq_len  upper bound of seq_lens[b] + new tokens; keys at or behind it are left out and
 *                READER_STATUS_BAD_LENGTH is set.  max_pages_per_seq * page_size >= max_seq_len.  The kernel is chosen as
 *                if the longest sequence had that length: a loose bound costs short calls up to three times their time
 *   workspace    >= reader_prompt_workspace_bytes(dims, N, max_seq_len) bytes, 256-byte aligned; its contents are
 *                meaningless between calls, calls that are ordered on one stream may share it
 *   status       i32 [1] or NULL                            in/out
 *
 * Keys behind a page id out of range are left out (READER_STATUS_BAD_PAGE); a row that sees no key at all gives
 * zeros and a log-sum-exp of -inf.  What a masked position holds, a NaN or an infinity too, does not reach the row.
 * Softmax weights are rounded to bf16 before they multiply V.  dims->variant = 1 is the plain kernel (one wavefront per
 * row, no workspace).  dims->T and max_path have to be valid and are not used.
 */
size_t reader_prompt_workspace_bytes(const reader_dims *dims, int32_t N, int32_t max_seq_len);
/* Query rows of a kv head that a workgroup of reader_prompt_attn takes for these sizes, by an estimate of the kernels' times: 16 or
 * 32 (few rows; keys cut into ranges), READER_PROMPT_ROWS_32_UNCUT, 64 or 128 (blocks of rows that are never cut), 256 (keys cut into
 * ranges); 0 for dims->variant = 1; or the error that reader_prompt_attn would return for the sizes.  Pure host function;
 * honours reader_tuning_override. */
enum { READER_PROMPT_ROWS_32_UNCUT = 33 };
int reader_prompt_rows(const reader_dims *dims, int32_t N, int32_t max_seq_len);
int reader_prompt_attn(const reader_dims *dims, int32_t N, const void *q, const void *k_cache, const void *v_cache,
                       const int32_t *page_table, const int32_t *cu_tokens, const int32_t *seq_lens,
                       void *out, float *lse, int32_t max_seq_len, void *workspace, size_t workspace_bytes,
                       int32_t *status, void *stream);

/*
 * Attention weight that every cached key has drawn, accumulated per kv head over the queries of committed tokens:
 *     weights[b, hkv, j] = decay * weights[b, hkv, j] + sum_{t, g} exp(sm_scale * <q[t, hkv G + g, :], k_j> - lse[t, hkv G + g])
 * over the query tokens t that see key j.  decay = 0 starts afresh: the old contents are not read, and positions behind
 * the last key get zero up to max_positions.  Otherwise those stay as they are: they have to be zero, as eviction and a
 * fresh start leave them, for the keys that come to live there.
 *
 * After a verification step: the query tokens are the accepted path, whose rows reader_kv_compact (or
 * reader_verify_step) has appended: seq_lens is the new length, and node path[b][j] sits at position
 * seq_lens[b] - (accept_len[b] + 1) + j and sees what lies in front of it and itself.
 *
 *   q            bf16 [B, T, Hq, D]                 in   as given to the attention
 *   lse          f32 [B, Hq, T]                     in   as the attention left it
 *   path         i32 [B, max_path], accept_len i32 [B]   in
 *   k_cache      bf16 [num_pages, Hkv, page_size, D]     in
 *   page_table   i32 [B, max_pages_per_seq], seq_lens i32 [B]   in
 *   weights      f32 [B, Hkv, max_positions]        in/out
 *   max_seq_len  upper bound of seq_lens[b]
 *   status       i32 [1] or NULL                    in/out
 *
 * A sequence with an accept_len or path entry out of range (READER_STATUS_BAD_PATH), or longer than max_seq_len,
 * max_positions or its pages (BAD_LENGTH), is left as it is.  A key behind a page id out of range draws nothing
 * (BAD_PAGE).  No atomics: the same inputs give the same bits.  One launch.
 */
int reader_key_weights(const reader_dims *dims, const void *q, const float *lse, const int32_t *path,
                       const int32_t *accept_len, const void *k_cache, const int32_t *page_table,
                       const int32_t *seq_lens, float decay, float *weights, int32_t max_positions,
                       int32_t max_seq_len, int32_t *status, void *stream);

/*
 * The same behind a prompt: the query tokens are the last `window` (0..READER_MAX_WINDOW) new tokens of every sequence, all
 * of them where there are fewer.  q bf16 [N, Hq, D], lse f32 [N, Hq] and seq_lens (in front of the new tokens) as for
 * reader_prompt_attn; max_seq_len bounds seq_lens[b] + new tokens.  A sequence whose packed bounds are out of order or of
 * range is left as it is (READER_STATUS_BAD_LENGTH).
 */
int reader_prompt_key_weights(const reader_dims *dims, int32_t N, const void *q, const float *lse,
                              const int32_t *cu_tokens, int32_t window, const void *k_cache,
                              const int32_t *page_table, const int32_t *seq_lens, float decay, float *weights,
                              int32_t max_positions, int32_t max_seq_len, int32_t *status, void *stream);

/*
 * Eviction from the cache by accumulated attention weight, all layers in one call.  In every sequence longer than `keep`,
 * each (layer, kv head) keeps `keep` rows: the newest `recent` positions, and of the others the heaviest, the lowest
 * position first among equal weights (a NaN is lighter than any number).  The kept rows of K and V, and their weights,
 * move to positions 0 .. keep - 1 in their order, in place; weights of the freed positions become zero; seq_lens[b] =
 * keep.  Rows at and behind the new length hold what is left there.  Other sequences are not touched.  What a head keeps
 * is its own affair: rows carry their rotation with them, and the positions of later tokens are the caller's to count on
 * (`positions` of reader_tree_qkv and reader_prompt_qkv).  Pages of an evicted sequence must not be shared with another.
 *
 *   num_layers   >= 1
 *   keep, recent  0 <= recent <= keep
 *   k_cache, v_cache  bf16 [num_layers, num_pages, Hkv, page_size, D]   in/out
 *   page_table   i32 [B, max_pages_per_seq], seq_lens i32 [B] (in/out)
 *   weights      f32 [num_layers, B, Hkv, max_positions]                in/out
 *   workspace    >= reader_kv_evict_workspace_bytes(dims, num_layers, keep) bytes, 4-byte aligned
 *   status       i32 [1] or NULL                                        in/out
 *
 * A sequence that is longer than max_positions or its pages (READER_STATUS_BAD_LENGTH), or has a page id out of range
 * (BAD_PAGE), is left as it is.  Bit-exact copy.  At most READER_MAX_EVICT_UNITS (layer, sequence, kv head) triples.
 * dims->Hq, T, max_path and sm_scale are not used.
 */
size_t reader_kv_evict_workspace_bytes(const reader_dims *dims, int32_t num_layers, int32_t keep);
int reader_kv_evict(const reader_dims *dims, int32_t num_layers, int32_t keep, int32_t recent,
                    void *k_cache, void *v_cache, const int32_t *page_table, int32_t *seq_lens,
                    float *weights, int32_t max_positions, void *workspace, size_t workspace_bytes,
                    int32_t *status, void *stream);

/*
 * ------------------------------------------------------------------ a cache in 4 bits
 * The paged cache at 17 / 64 of the bytes: K and V of a position in 4 bits a value.  Values 32 g .. 32 g + 31 of a row share a
 * scale 2^e, -125 <= e <= 125, and each is one of 0, 1/2, 1, 3/2, 2, 3, 4, 6 times it, with a sign: exact in bf16.  With a the
 * largest magnitude of the group, e = floor(log2(a)) - 2, and one more where a > 7 * 2^e, so that no value moves by more than 2^e (but
 * where the upper bound on e holds it back, a > 7 * 2^125); values are rounded to nearest even.  A group with a NaN or an infinity
 * is stored as zeros and READER_STATUS_BAD_VALUE is set.
 *
 *   kvq_cache   u8 [num_pages, Hkv, READER_KVQ_BLOCK_BYTES(D)], 16-byte aligned.  A block holds, for the 16 rows s of a page, d even:
 *     codes of values d, d + 1 of K (the low half of a byte is the even value's; bit 3 of a code is its sign, the others number
 *       the values above)       at  d / (D/4) * 2 D + s * (D/8) + d % (D/4) / 2
 *     ... of V                  at  8 D + s / 4 * 2 D + d / (D/16) * (D/8) + s % 4 * (D/32) + d % (D/16) / 2
 *     the scale of K's group g  at  16 D + 16 g + s            (a byte, e + 127)
 *     ... of V's                at  16 D + D / 2 + s / 4 * (D/8) + 4 g + s % 4
 *   (whole-number divisions).  Scale bytes above 252 are of no value: the rows that read them are unspecified.
 *
 * The rows of new tokens and of draft trees are stored behind the seq_lens[b] positions that the cache holds before the attention is
 * called, as in the in-cache layout of reader_tree_attn: plain decoding and the verification of a tree then read the same
 * values.  dims->variant must be 0; the bf16 tensors start at a multiple of 16 bytes.  A page that rows are stored in
 * belongs to one sequence (reader_pages_reserve).
 * The attention takes up to 2^30 positions a sequence.  Scores are held in 32 bits: a row whose scores times log2(e) reach 2^30 in
 * magnitude, or whose query holds a NaN or an infinity, is unspecified; other rows are not.  Where there are many query rows, values
 * 32 g .. 32 g + 31 of a query are held to 2^-15 of the largest of them (exactly above 1/128 of it), or to 2^-130 where that is more.
 */
#define READER_KVQ_BLOCK_BYTES(D) (17 * (D))

/*
 * K/V rows into the cache: row t of sequence b, its i-th new one, goes to position seq_lens[b] + i.
 *
 *   N            rows
 *   k, v         bf16 [N, Hkv, D]                           in   (k_tree, v_tree of reader_tree_qkv, for one)
 *   cu_tokens    i32 [B + 1] or NULL                        in   packed rows as above; NULL: draft trees, N = B * T
 *   seq_lens     i32 [B]                                    in
 *   kvq_cache    u8 [num_pages, Hkv, 17 D]                  out
 *   page_table   i32 [B, max_pages_per_seq]                 in
 *   status       i32 [1] or NULL                            in/out
 *
 * A row that the page table does not hold (READER_STATUS_BAD_LENGTH) or whose page id is out of range (BAD_PAGE) is left out.
 * One launch.
 */
int reader_kvq_store(const reader_dims *dims, int32_t N, const void *k, const void *v, const int32_t *cu_tokens,
                     const int32_t *seq_lens, void *kvq_cache, const int32_t *page_table, int32_t *status, void *stream);

/*
 * Positions [starts[b], seq_lens[b]) of a bf16 cache into the same positions of the cache in 4 bits, all layers in one call: a
 * prompt is worked on in bf16 (reader_prompt_qkv, reader_prompt_attn) and kept in 4 bits.
 *
 *   k_cache, v_cache  bf16 [num_layers, from_pages, Hkv, page_size, D]   in
 *   from_table   i32 [B, max_pages_per_seq]                 in   pages of k_cache and v_cache
 *   starts       i32 [B] or NULL                            in   NULL: zeros
 *   seq_lens     i32 [B]                                    in   ends, at most max_seq_len
 *   kvq_cache    u8 [num_layers, num_pages, Hkv, 17 D]      out
 *   page_table   i32 [B, max_pages_per_seq]                 in   pages of kvq_cache
 *   status       i32 [1] or NULL                            in/out
 *
 * A sequence whose bounds are out of order, or behind max_seq_len or the page table, is left out (READER_STATUS_BAD_LENGTH), as are
 * the positions of a page whose id is out of range in either table (BAD_PAGE).  One launch.
 */
int reader_kvq_pack(const reader_dims *dims, int32_t num_layers, const void *k_cache, const void *v_cache, int64_t from_pages,
                    const int32_t *from_table, const int32_t *starts, const int32_t *seq_lens, int32_t max_seq_len, void *kvq_cache,
                    const int32_t *page_table, int32_t *status, void *stream);

/*
 * reader_kv_compact_layers on the cache in 4 bits: for every b, layer, kv head and j = 1..accept_len[b], position seq_lens[b] + j
 * receives the row that position seq_lens[b] + path[b][j] held; then seq_lens[b] += accept_len[b] + 1.  The same checks, status
 * bits and results; num_layers 0: only the lengths.  Calls on several streams do not meet (nothing is kept between calls).
 *
 *   kvq_cache    u8 [num_layers, num_pages, Hkv, 17 D]      in/out
 */
int reader_kvq_compact_layers(const reader_dims *dims, int32_t num_layers, const int32_t *path, const int32_t *accept_len,
                              void *kvq_cache, const int32_t *page_table, int32_t *seq_lens, int32_t *status, void *stream);

/*
 * Tree-masked attention over the cache in 4 bits: reader_tree_attn in its in-cache layout, the row of node n of sequence b at
 * position seq_lens[b] + n.
 *
 *   q            bf16 [B, T, Hq, D]                         in
 *   kvq_cache    u8 [num_pages, Hkv, 17 D]                  in
 *   page_table   i32 [B, max_pages_per_seq]                 in   must map pages for [0, seq_lens[b] + T)
 *   seq_lens     i32 [B]                                    in   tree rows excluded
 *   parents      i32 [B, T]                                 in
 *   out          bf16 [B, T, Hq, D]                         out  fp32 accumulation, rounded to nearest even
 *   lse          f32 [B, Hq, T] or NULL                     out
 *   max_seq_len  upper bound of seq_lens[b]; max_pages_per_seq * page_size >= max_seq_len + T.  A longer sequence counts as this
 *                long (READER_STATUS_BAD_LENGTH)
 *   workspace    >= reader_kvq_workspace_bytes(dims, B * T, max_seq_len) bytes, 256-byte aligned; its contents are meaningless
 *                between calls, calls that are ordered on one stream may share it
 *   status       i32 [1] or NULL                            in/out
 *
 * A node whose link is wrong counts as a root (BAD_TREE): it sees the prefix and itself.  Keys behind a page id out of range are left
 * out (BAD_PAGE); a row that sees no key gives zeros and a log-sum-exp of -inf.  What the pages hold behind the last row does
 * not reach the outputs.  Softmax weights are rounded to bf16 before they multiply V.  dims->max_path is not used.  One launch, or two
 * where the keys of a block of rows are shared out.
 */
size_t reader_kvq_workspace_bytes(const reader_dims *dims, int32_t N, int32_t max_seq_len);
int reader_kvq_tree_attn(const reader_dims *dims, const void *q, const void *kvq_cache, const int32_t *page_table,
                         const int32_t *seq_lens, const int32_t *parents, void *out, float *lse, int32_t max_seq_len,
                         void *workspace, size_t workspace_bytes, int32_t *status, void *stream);

/*
 * Causal attention of packed prompts, chunks and single tokens over the cache in 4 bits: arguments, masks, padding and status bits
 * of reader_prompt_attn, the new tokens' rows stored already.
 *
 *   q            bf16 [N, Hq, D]                            in
 *   out          bf16 [N, Hq, D]                            out
 *   lse          f32 [N, Hq] or NULL                        out
 *   max_seq_len  upper bound of seq_lens[b] + new tokens; keys at or behind it are left out (READER_STATUS_BAD_LENGTH)
 *   workspace    >= reader_kvq_workspace_bytes(dims, N, max_seq_len) bytes, 256-byte aligned
 */
int reader_kvq_prompt_attn(const reader_dims *dims, int32_t N, const void *q, const void *kvq_cache, const int32_t *page_table,
                           const int32_t *cu_tokens, const int32_t *seq_lens, void *out, float *lse, int32_t max_seq_len,
                           void *workspace, size_t workspace_bytes, int32_t *status, void *stream);

/*
 * ------------------------------------------------------------------ pages that sequences share
 * A pool of num_pages pages, of whichever cache: page_refs[p] is the number of entries of page tables that name page p, and a page
 * nobody names is free.  Sequences may hold pages together (the prefix that they share, a beam and its forks); entries that
 * hold no page are -1.  The two calls below keep the counts; a page that is held elsewhere too has a count of its own there (the
 * entries of the table at hand are added and taken away, never counted anew).  Counts that do not match the tables give pages away
 * that are in use: nothing checks them.
 *
 *   page_table   i32 [B, max_pages_per_seq]                 in/out
 *   page_refs    i32 [num_pages]                            in/out
 *   workspace    >= reader_pages_workspace_bytes(dims) bytes, 4-byte aligned; its contents are meaningless between calls
 * Of dims only B, max_pages_per_seq and num_pages are used; the rest has to be valid.  No atomics but of whole numbers: the same
 * inputs give the same results.
 */
size_t reader_pages_workspace_bytes(const reader_dims *dims);

/*
 * Row b of the batch becomes what row sources[b] was before the call: forks (a source that is named twice), permutations, and
 * sequences dropped (a row that nobody names).  The new row holds the pages of its positions, all of them shared with the
 * row's other forks, and nothing behind (pages that were reserved there are given back); seq_lens follows.
 *
 *   sources      i32 [B]                                    in   -1: the row becomes empty, of length 0
 *   seq_lens     i32 [B]                                    in/out
 *   status       i32 [1] or NULL                            in/out
 *
 * A source outside [-1, B) counts as b (READER_STATUS_BAD_PATH).  An entry in front of a sequence's length that names no page
 * is handed on as it is (BAD_PAGE); a length that the table does not hold takes the whole row (BAD_LENGTH).  One launch up to
 * B * (max_pages_per_seq + 1) = 4096, else two.
 */
int reader_pages_reorder(const reader_dims *dims, const int32_t *sources, int32_t *page_table, int32_t *seq_lens, int32_t *page_refs,
                         void *workspace, size_t workspace_bytes, int32_t *status, void *stream);

/*
 * Makes positions [seq_lens[b], new_lens[b]) of every sequence ready to be written: on pages that nobody else holds.
 *   - the page that seq_lens[b] falls into the middle of, if others hold it too: a free page takes its place and its contents, in
 *     all layers; of the sequences of the call that write into one page and hold it alone together, the last keeps it
 *   - pages that lie wholly behind seq_lens[b]: entries that hold none, or one that others hold too, get a free page
 *   - pages behind new_lens[b] are given back; entries there that name no page become -1
 * Free pages are taken in ascending order, for the sequences in their order and the pages of each from the first; what the call
 * gives back can be taken by it, but for pages that it copies from.  If there are not as many as are wanted, none is taken or given
 * back and READER_STATUS_NO_PAGES is set.  seq_lens is not changed.
 *
 *   num_layers   >= 0 (0: no contents to copy, the caches are not used)
 *   page_bytes   bytes of a page of one layer, a multiple of 16
 *   seq_lens, new_lens  i32 [B]                             in   new_lens[b] >= seq_lens[b] (else the sequence is left as it is,
 *                                                                READER_STATUS_BAD_LENGTH, as where the table does not hold new_lens[b])
 *   k_cache, v_cache    [num_layers, num_pages, page_bytes] in/out, 16-byte aligned; v_cache may be NULL (one cache: the one in 4 bits)
 *   status       i32 [1] or NULL                            in/out
 *
 * A page id out of range in the middle of which seq_lens[b] falls sets BAD_PAGE and stays.  Four launches.
 */
int reader_pages_reserve(const reader_dims *dims, int32_t num_layers, int64_t page_bytes, const int32_t *seq_lens, const int32_t *new_lens,
                         void *k_cache, void *v_cache, int32_t *page_table, int32_t *page_refs, void *workspace,
                         size_t workspace_bytes, int32_t *status, void *stream);

#ifdef __cplusplus
}
#endif
#endif /* READER_H */

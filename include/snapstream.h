/*
 * snapstream.h -- C ABI of the SnapStream hot path for NVIDIA B200 (sm_100a).
 *
 * SnapStream (arXiv 2511.03092) compresses a prompt's KV cache once, at prefill, into a
 * fixed number of slots  [ sinks | recent-token ring | SnapKV top-K ]  (Section 3.1) and then
 * decodes over that fixed-size cache, writing each new token's K/V into the ring at the index
 * of Eq. 3 (Section 3.3).  This library implements exactly that path:
 *
 *   snap_cache_layout   slot arithmetic of Section 3.1
 *   snap_compress       Section 3.2: Eq. 4 scores -> Eq. 1 window sum -> Eq. 2 pool + top-K ->
 *                       ring construction (Section 3.2.1) and gather into the cache
 *   snap_append_kv      Eq. 3 scatter of one new token per sequence
 *   snap_decode_attn    Section 3.3: (optional Eq. 3 scatter, then) attention of one query token
 *                       per sequence over the valid cache slots
 *
 * and, around it: snap_decode_attn_multi (several new tokens per sequence and step),
 * snap_decode_attn_static (the decode step without a caller-provided scratch buffer),
 * snap_append_kv_concat (the slice-and-concatenate update of Section 3.2.1, as a baseline),
 * snap_prefill_attn + snap_compress_with_row_stats (the prompt's causal attention emitting
 * the normalisers of Eq. 4, and the compression that consumes them),
 * and snap_block_stats + snap_block_select + snap_decode_attn_blocks (a per-step block top-K
 * over the whole middle of the prompt instead of the one-time top-K, the variant the paper's
 * related-work section leaves to future work),
 * and, for the uncompressed cache a serving program keeps next to it: snap_rope (rotary positions
 * of queries and keys), snap_paged_append + snap_paged_decode_attn (a cache in pages and the
 * attention of one new token per sequence over it) and snap_paged_evict (cutting a paged cache
 * back to l_sink + topk + l_recent rows by accumulated attention weight); snap_paged_plan (which
 * pages a step's new tokens go to, decided on the device); and the same cache in 8 bits:
 * snap_paged_q8_append, snap_paged_q8_decode_attn (one or several tokens per sequence) and
 * snap_paged_q8_gather (rows back as the dense keys and values that snap_prefill_attn and
 * snap_compress take).
 *
 * Conventions
 *   - "dev" pointers are CUDA device pointers on the current device, "host" pointers are plain
 *     host memory.  Every device buffer must be 16-byte aligned (the tensors, caches, outputs and
 *     workspaces are checked: SNAP_ERR_INVALID_ARG, nothing launched).
 *   - The caller owns every buffer.  The library allocates no device memory; all work is
 *     enqueued on the CUDA stream given and the calls return without synchronising.
 *   - What the library keeps between calls, all of it on the host: per device, the SM count and
 *     which kernels already had their shared-memory limit raised (so the first call of each
 *     entry point on a device must come before any stream capture); per host thread, the
 *     tensor maps of the last few cache buffers the decode kernel was given, keyed on their
 *     addresses and shape; per process, a launch counter and the testing options of
 *     snap_debug_set_option.  Nothing of one call's data outlives the call, except in the fixed
 *     scratch array of snap_decode_attn_static, which says so below.
 *   - Token positions are 0-indexed.  Ls = l_sink, Lr = l_recent, K = topk, Lsr = Ls + Lr,
 *     Sc = Ls + Lr + K, g = n_q_heads / n_kv_heads.
 *   - Element type: all of q, k, v, caches and out share cfg->dtype.
 *   - Return value: SNAP_OK (0) or a negative snap_status.  Nothing throws, aborts or traps.
 *     Conditions only the device can see (a cache slot id out of range, a bounded wait that
 *     ran out, a refinement band that overflowed) are OR-ed into *status_dev when given.
 */
#ifndef SNAPSTREAM_H_
#define SNAPSTREAM_H_

#include <stddef.h>
#include <stdint.h>

#ifdef __cplusplus
extern "C" {
#endif

#define SNAP_F32 0
#define SNAP_BF16 1

#define SNAP_POOL_AVG 0
#define SNAP_POOL_MAX 1

typedef enum snap_status {
  SNAP_OK = 0,
  SNAP_ERR_INVALID_ARG = -1,        /* a value outside the documented domain */
  SNAP_ERR_UNSUPPORTED = -2,        /* valid, but no kernel is built for this shape */
  SNAP_ERR_WORKSPACE_TOO_SMALL = -3,
  SNAP_ERR_NULL_POINTER = -4,
  SNAP_ERR_CUDA = -5,               /* a CUDA runtime call failed; see cudaGetLastError */
  SNAP_ERR_STATIC_SCRATCH_EXCEEDED = -6  /* snap_decode_attn_static: the problem needs more than
                                            SNAP_STATIC_SCRATCH_BYTES of scratch; nothing ran */
} snap_status;

/* bits of *status_dev */
#define SNAP_DEV_BAD_SLOT 1u        /* a slot id was outside [0, max_seqs): that sequence was skipped */
#define SNAP_DEV_WAIT_TIMEOUT 2u    /* a bounded wait on an async copy gave up: results invalid */
#define SNAP_DEV_BAND_OVERFLOW 4u   /* snap_compress: a KV head had more candidates within the re-scoring
                                       band of its top-K threshold than the band buffer holds (512, or
                                       256 for layers with more than 2^18 query elements per KV head);
                                       snap_block_select: more than 256 blocks that single precision
                                       cannot tell from the threshold.  That head keeps its
                                       single-precision order.  The results are valid; exactly tied
                                       scores, which go to the lower position in either precision, are
                                       the usual cause */

#define SNAP_DEV_INDEX_CHECK 8u     /* only from the checked build of the library (compiled with
                                       -DSNAP_DEBUG_BOUNDS): a data-dependent index -- a selected
                                       position, a ring slot, an output rank, a band entry -- fell
                                       outside its array; the access was skipped */

#define SNAP_DEV_BAD_PAGE 16u       /* paged cache: a page number outside [0, n_pages), or a row or a length past
                                       the page table: those rows were skipped */
#define SNAP_DEV_NO_ROOM 32u        /* snap_paged_plan: not enough free pages, or no room in the list of tokens: those
                                       requests were refused */

/* One attention layer's shape and SnapStream hyper-parameters (appendix table
 * "SnapStream Hyperparameters": sink, top-K, recent, observation window, pooling kernel). */
typedef struct snap_config {
  int32_t n_q_heads;      /* Hq */
  int32_t n_kv_heads;     /* Hkv, divides Hq */
  int32_t d_qk;           /* key/query row length, multiple of 16 */
  int32_t d_v;            /* value row length, multiple of 16, <= 512 */
  int32_t v_aliases_k;    /* 1: latent attention, V row = first d_v elements of the K row, no V buffers */
  int32_t dtype;          /* SNAP_F32 or SNAP_BF16 */
  int32_t l_sink;         /* Ls >= 0 */
  int32_t l_recent;       /* Lr >= 1 */
  int32_t topk;           /* K  >= 0 */
  int32_t l_obs;          /* Lo, 1 <= Lo <= Lr (every candidate precedes every window query) */
  int32_t pool_kernel;    /* w, odd >= 1 */
  int32_t pool_mode;      /* SNAP_POOL_AVG (Eq. 2) or SNAP_POOL_MAX */
  float softmax_scale;    /* Eq. 4's 1/sqrt(d), supplied by the caller */
  int32_t max_seqs;       /* number of cache slots (sequences resident at once) */
} snap_config_t;

/* Section 3.1: where the three sections live, and the strides of the caches.
 * K cache: [max_seqs][Hkv][Sc][d_qk], V cache: [max_seqs][Hkv][Sc][d_v], row-major, dense. */
typedef struct snap_layout {
  int32_t slots;          /* Sc = Ls + Lr + K  (L_snapstream, Section 3) */
  int32_t sink_off;       /* 0 */
  int32_t ring_off;       /* Ls */
  int32_t topk_off;       /* Ls + Lr */
  int64_t k_row_bytes, v_row_bytes;
  int64_t k_head_stride_bytes, v_head_stride_bytes;   /* Sc * row bytes */
  int64_t k_seq_stride_bytes, v_seq_stride_bytes;     /* Hkv * head stride */
  int64_t k_cache_bytes, v_cache_bytes;               /* max_seqs * seq stride (v: 0 if aliased) */
} snap_layout_t;

/* Section 3.1.  Host only, pure arithmetic.  Validates cfg (INVALID_ARG / UNSUPPORTED). */
int snap_cache_layout(const snap_config_t* cfg, snap_layout_t* out);

/* Bytes of device scratch snap_compress needs for these prompt lengths (cu_seqlens_host has
 * n_seq + 1 entries, prompt i is tokens [cu[i], cu[i+1])).  Negative snap_status on error. */
int64_t snap_compress_workspace_bytes(const snap_config_t* cfg, const int32_t* cu_seqlens_host,
                                      int32_t n_seq);

/* Bytes of device scratch snap_decode_attn needs for n_active sequences. */
int64_t snap_decode_workspace_bytes(const snap_config_t* cfg, int32_t n_active);

/*
 * Prefill compression of n_seq prompts (Section 3.2; appendix listing "SnapStream Prefill KV
 * Cache Compression" describes the same inputs and outputs).
 *
 *   q_obs_dev   [n_seq][Hq][Lo][d_qk]  queries of each prompt's last Lo positions, after any
 *               positional encoding (Section 3.2: encodings are applied before caching).
 *               Ignored (may be NULL) when no prompt has more than Lsr + K tokens.
 *   k_dev,v_dev prompt keys/values, token-major and ragged: element (t, h, c) of prompt i is at
 *               k_dev[(cu[i] + t) * k_token_stride + h * k_head_stride + c]; strides in elements,
 *               multiples of 16 bytes.  v_dev is ignored when cfg->v_aliases_k.
 *   cu_seqlens_host, slot_ids_host   host arrays (n_seq + 1 and n_seq entries); slot_ids give the
 *               cache slot each prompt is compressed into, distinct, in [0, max_seqs).
 *   k_cache_dev, v_cache_dev   the caches (snap_layout_t strides).  For each prompt the whole slot
 *               is rewritten: sinks [0, min(L, Ls)), ring rows of positions [max(Ls, L - Lr), L) at
 *               slot Ls + (p - Ls) mod Lr, selected rows ascending by position from slot Lsr,
 *               zeros elsewhere.
 *   seq_len_dev, valid_topk_dev   [max_seqs] int32; entry slot_ids[i] is set to L_i and to
 *               min(max(L_i - Lsr, 0), K).
 *   topk_idx_dev  NULL, or [n_seq][Hkv][K] int32 receiving the selected absolute positions,
 *               ascending, -1 after the valid ones.
 *   A prompt with L <= Lsr + K is not scored: all its candidates are kept.  Otherwise the K
 *   largest pooled scores win, ties to the lower position.
 *   Precision of the selection: scores are computed in single precision (the part of their error
 *   that can reorder two pooled scores was measured at 1e-7 relative, 2.2e-7 at most, on 32k-
 *   to 128k-token prompts); every candidate whose pooled score lies within 1e-4 relative of the
 *   K-th largest (2e-5 for layers with more than 2^18 query elements per KV head, such as the
 *   latent layout) is then scored again in double precision from q_obs and k, with the
 *   normalisers of Eq. 4 from the single-precision pass, and the order inside that band decides
 *   (measured order error 2e-9, 1.3e-8 at most).  Pooling kernels wider than 33 are not
 *   re-scored.  SNAP_DEV_BAND_OVERFLOW reports a band that did not fit its buffer.
 */
int snap_compress(const snap_config_t* cfg, const snap_layout_t* layout,
                  const void* q_obs_dev,
                  const void* k_dev, int64_t k_token_stride, int64_t k_head_stride,
                  const void* v_dev, int64_t v_token_stride, int64_t v_head_stride,
                  const int32_t* cu_seqlens_host, const int32_t* slot_ids_host, int32_t n_seq,
                  void* k_cache_dev, void* v_cache_dev,
                  int32_t* seq_len_dev, int32_t* valid_topk_dev,
                  int32_t* topk_idx_dev,
                  void* workspace_dev, size_t workspace_bytes,
                  uint32_t* status_dev, void* cuda_stream);

/*
 * Causal attention of n_seq whole prompts that also yields the denominators of Eq. 4
 * (Section 3.2.2 names the score recomputation as the step left to optimise: the normalisers
 * of the observation window's scores are by-products of the prompt's own attention pass).
 *
 *   q_dev     [T][Hq][d_qk] dense, token-major and ragged like k_dev (T = cu[n_seq]); the
 *             queries after positional encoding
 *   k_dev, v_dev and their strides: as in snap_compress
 *   out_dev   [T][Hq][d_v] dense: row t of head h is softmax(scale * q_t . K[0..t]^T) V[0..t]
 *             over the keys of KV head h / (Hq/Hkv) of the same prompt
 *   row_mu_dev  NULL, or [n_seq][Hq][Lo] float: for the prompt's last Lo positions (entry i is
 *             position L - Lo + i; entries of positions below 0 are left untouched)
 *               log2( sum over candidates j in [Ls, L - Lr) of exp(scale * q . k_j) ),
 *             -inf when the prompt has no candidate.  This is what snap_compress_with_row_stats
 *             takes in place of its own first pass over the keys.
 * bf16 layers with d_qk = d_v = 128 and a separate V run on the tensor cores; every other layer
 * (fp32, other head sizes, the latent layout, where v_dev is ignored) runs on a portable kernel
 * that is there for coverage, not for speed.
 * Needs no workspace.  cfg is validated as a whole (as by snap_cache_layout); the kernels use its
 * model-shape fields, l_sink, l_recent, l_obs and softmax_scale.  Errors: SNAP_ERR_NULL_POINTER,
 * SNAP_ERR_INVALID_ARG (cfg, offsets that decrease, strides that are not multiples of 16 bytes):
 * nothing was launched; SNAP_ERR_CUDA: a launch failed.
 */
int snap_prefill_attn(const snap_config_t* cfg, const void* q_dev,
                      const void* k_dev, int64_t k_token_stride, int64_t k_head_stride,
                      const void* v_dev, int64_t v_token_stride, int64_t v_head_stride,
                      const int32_t* cu_seqlens_host, int32_t n_seq,
                      void* out_dev, float* row_mu_dev,
                      uint32_t* status_dev, void* cuda_stream);

/*
 * snap_compress with the Eq. 4 normalisers supplied by the caller (row_mu_dev as written by
 * snap_prefill_attn; NULL = compute them here, which is snap_compress): the score kernel then
 * makes one pass over the candidate keys instead of two.  Same arguments, results, workspace
 * and errors as snap_compress otherwise; every score kernel takes them.  The selection can
 * differ from snap_compress's only where two pooled scores are equal to within single-precision
 * rounding.
 */
int snap_compress_with_row_stats(const snap_config_t* cfg, const snap_layout_t* layout,
                  const void* q_obs_dev, const float* row_mu_dev,
                  const void* k_dev, int64_t k_token_stride, int64_t k_head_stride,
                  const void* v_dev, int64_t v_token_stride, int64_t v_head_stride,
                  const int32_t* cu_seqlens_host, const int32_t* slot_ids_host, int32_t n_seq,
                  void* k_cache_dev, void* v_cache_dev,
                  int32_t* seq_len_dev, int32_t* valid_topk_dev,
                  int32_t* topk_idx_dev,
                  void* workspace_dev, size_t workspace_bytes,
                  uint32_t* status_dev, void* cuda_stream);

/*
 * Eq. 3: for each of n_active sequences write the new token's K/V rows
 * (k_new_dev [n_active][Hkv][d_qk], v_new_dev [n_active][Hkv][d_v], dense) into cache slot
 *   L < Ls ? L : (L - Ls + Lr) mod Lr + Ls,   L = seq_len_dev[slot]  (tokens seen so far),
 * then add one to seq_len_dev[slot].  slot_ids_dev: [n_active] int32 on the device, distinct.
 */
int snap_append_kv(const snap_config_t* cfg, const snap_layout_t* layout,
                   const void* k_new_dev, const void* v_new_dev,
                   const int32_t* slot_ids_dev, int32_t n_active,
                   void* k_cache_dev, void* v_cache_dev, int32_t* seq_len_dev,
                   uint32_t* status_dev, void* cuda_stream);

/*
 * Section 3.3: one decode step.  With k_new_dev != NULL the new token is first written as in
 * snap_append_kv (and seq_len advanced); then out[i][h] = softmax(scale * q[i][h] . K^T) V over
 * the valid slots of sequence i: [0, min(len, Lsr)) and [Lsr, Lsr + valid_topk).
 * With k_new_dev == NULL the cache is only read.
 *   q_dev [n_active][Hq][d_qk], out_dev [n_active][Hq][d_v], dense.  A sequence with no valid
 *   slot gets zeros.  Sequences in one call must use distinct slots.
 */
int snap_decode_attn(const snap_config_t* cfg, const snap_layout_t* layout,
                     const void* q_dev, const void* k_new_dev, const void* v_new_dev,
                     const int32_t* slot_ids_dev, int32_t n_active,
                     void* k_cache_dev, void* v_cache_dev,
                     int32_t* seq_len_dev, const int32_t* valid_topk_dev,
                     void* out_dev,
                     void* workspace_dev, size_t workspace_bytes,
                     uint32_t* status_dev, void* cuda_stream);

/*
 * A decode step with q_len new tokens per sequence (the multi-token prediction that the
 * throughput evaluation of Section 5 assumes: several tokens per forward pass over the same
 * cache).  Defined as q_len steps of
 * snap_decode_attn: token u is appended as in Eq. 3, then query u attends over the cache as it
 * is after tokens 0..u -- a window row that token u evicts is still seen by the queries before
 * u and by none from u on.
 *   q_dev     [n_active][q_len][Hq][d_qk]
 *   k_new_dev [n_active][q_len][Hkv][d_qk], v_new_dev [n_active][q_len][Hkv][d_v]   (required)
 *   out_dev   [n_active][q_len][Hq][d_v];  seq_len_dev[slot] += q_len
 * 1 <= q_len <= Lr (SNAP_ERR_INVALID_ARG otherwise).  bf16 layers with 64-, 128- or 256-wide heads
 * and up to 16 query heads per KV head take 16 / (Hq / Hkv) tokens per pass over the cache (all
 * q_len in one pass when q_len * (Hq / Hkv) <= 16, otherwise several passes, each reading its
 * tokens' rows in place); every other layer (fp32, the latent layout -- v_new_dev is then ignored
 * --) is served as the definition reads, q_len single steps: same results, no saving in cache
 * traffic.  The tcgen05 latent kernel reads each token's rows in place; the other single-step
 * kernels have them staged in the workspace first.
 * Scratch: snap_decode_multi_workspace_bytes(cfg, n_active, q_len).
 */
int64_t snap_decode_multi_workspace_bytes(const snap_config_t* cfg, int32_t n_active, int32_t q_len);
int snap_decode_attn_multi(const snap_config_t* cfg, const snap_layout_t* layout,
                           const void* q_dev, const void* k_new_dev, const void* v_new_dev,
                           const int32_t* slot_ids_dev, int32_t n_active, int32_t q_len,
                           void* k_cache_dev, void* v_cache_dev,
                           int32_t* seq_len_dev, const int32_t* valid_topk_dev,
                           void* out_dev,
                           void* workspace_dev, size_t workspace_bytes,
                           uint32_t* status_dev, void* cuda_stream);

/* Size of the scratch array built into the library for snap_decode_attn_static. */
#define SNAP_STATIC_SCRATCH_BYTES (8u << 20)

/*
 * A decode step for callers that cannot allocate.  (The paper has no counterpart; this is a
 * property of the library, not of the method.)
 *
 * Same operation, arguments and results as snap_decode_attn, but without the workspace
 * arguments: the per-split partial results go to a fixed SNAP_STATIC_SCRATCH_BYTES array that
 * lives inside the library, so the call performs no cudaMalloc/cudaFree and needs no buffer
 * from the caller beyond the inputs and outputs.  It is meant for code that must not allocate
 * where decode steps are issued: a serving loop whose device memory was partitioned up front
 * and is full, a plugin running inside another runtime's callback, a process under a policy
 * that treats late allocations as failures.
 *
 *   - Every GPU that loads this library holds the array from load until process exit.
 *   - The step runs the same kernels with the same split count as snap_decode_attn (the latent
 *     layout included) and needs snap_decode_workspace_bytes(cfg, n_active) - 256 bytes of the
 *     array: n_active * n_q_heads * splits * (d_v + 2) floats (d_v + 4 for the latent layout),
 *     splits being the library's choice for that batch size.  If that exceeds the array the call returns
 *     SNAP_ERR_STATIC_SCRATCH_EXCEEDED and launches nothing; use snap_decode_attn instead.
 *     The 32-sequence, 32-head, d_v = 128 batch of a Llama-3.1-8B layer needs about 4.3 MB.
 *   - All calls share the one array and it keeps the previous call's contents.  Nothing has to
 *     be cleared (every partial that is read was written by the same call), but two calls
 *     that can overlap on the GPU -- different streams without a dependency -- race.
 *   - The first call on each device looks up the array's device address (no allocation);
 *     make that first call outside any stream capture, with that device current.
 */
int snap_decode_attn_static(const snap_config_t* cfg, const snap_layout_t* layout,
                            const void* q_dev, const void* k_new_dev, const void* v_new_dev,
                            const int32_t* slot_ids_dev, int32_t n_active,
                            void* k_cache_dev, void* v_cache_dev,
                            int32_t* seq_len_dev, const int32_t* valid_topk_dev,
                            void* out_dev, uint32_t* status_dev, void* cuda_stream);

/*
 * Section 3.2.1's counter-example, as a measured baseline: the rolling window kept in position
 * order and updated by slicing and concatenating, which yields a NEW cache every step.
 * For each active sequence (L = seq_len_dev[slot]), rows of the output cache are
 *   L <  Ls + Lr:  the input rows, with row L replaced by the new token (a plain scatter);
 *   L >= Ls + Lr:  sinks [0, Ls) and selected rows [Ls+Lr, Sc) copied, window row r takes input
 *                  row r + 1 for Ls <= r < Ls+Lr-1, and the new token goes to row Ls+Lr-1.
 * Then seq_len_dev[slot] += 1.  Slots that are not listed in slot_ids_dev are not copied.
 * The output buffers must differ from the input buffers (SNAP_ERR_INVALID_ARG otherwise); both
 * have the cache layout of snap_cache_layout and are owned by the caller.  A cache that
 * snap_compress built has its window in ring order (Eq. 3); it is in position order as well
 * exactly when (L - Ls) is a multiple of Lr or L <= Ls + Lr.  snap_decode_attn with
 * k_new_dev == NULL reads either order, since attention does not depend on the row order.
 * Traffic per step: the whole cache read and written, against one row for snap_append_kv.
 */
int snap_append_kv_concat(const snap_config_t* cfg, const snap_layout_t* layout,
                          const void* k_new_dev, const void* v_new_dev,
                          const int32_t* slot_ids_dev, int32_t n_active,
                          const void* k_cache_in_dev, const void* v_cache_in_dev,
                          void* k_cache_out_dev, void* v_cache_out_dev,
                          int32_t* seq_len_dev, uint32_t* status_dev, void* cuda_stream);

/*
 * Per-step block top-K (the paper's related-work section: KV blocks with pre-computed statistics,
 * of which the top ones are looked up for every newly decoded token, left there to future
 * work; the criterion is the published query-aware one).  The paper fixes nothing further, so
 * the definition is this library's:
 *   - the cache is built by snap_compress with a top-K budget of at least the prompt's middle
 *     (topk >= L - Ls - Lr): every candidate is then kept, in position order, in the third
 *     section, valid_topk rows of it;
 *   - that section is cut into blocks of block_tokens consecutive rows (a multiple of 16, at
 *     most 1024; the last block may be shorter); a block's statistics are the element-wise
 *     minimum and maximum of its keys per KV head;
 *   - a decode query scores block b of KV head kvh by
 *       U = sum over the query heads h of kvh and the dims d of max(q[h][d] * kmin[b][d], q[h][d] * kmax[b][d]),
 *     an upper bound of the group-summed logit of every key of the block, and the n_blocks
 *     highest-scoring blocks are attended, ties to the lower block index, together with the
 *     sinks and the rolling window, which behave as in snap_decode_attn (Eq. 3 append
 *     included); rows that leave the window during decoding are dropped as before.
 * bf16 layers with 64-, 128- or 256-wide heads, a separate V and at most 16 query heads per KV
 * head; at most 8192 blocks per sequence; SNAP_ERR_UNSUPPORTED otherwise.  The scores are summed
 * in single precision for every block; the blocks that single precision cannot tell from the
 * last selected one (a rigorous error bound per block) are scored again in double precision and
 * ranked by that, so the selection is the one the exact scores give down to relative differences
 * of about 1e-15.  More than 256 such blocks for one (sequence, KV head): the single-precision
 * order stands and SNAP_DEV_BAND_OVERFLOW is raised in *status_dev.
 *
 * snap_block_stats    once per prompt, after snap_compress:
 *   stats_dev  out [max_seqs][Hkv][ceil(topk / block_tokens)][2][d_qk] in the cache's dtype (minimum, then
 *              maximum), snap_block_stats_bytes(cfg, block_tokens) bytes; the blocks of slot_ids_dev[0 .. n_seqs)
 *              are written, rows of blocks past a prompt's last one are left alone.
 * snap_block_select   every step, before the attention:
 *   q_dev [n_active][Hq][d_qk];  block_idx_dev out [n_active][Hkv][n_blocks] ascending block numbers;
 *   n_selected_dev out [n_active][Hkv] = min(n_blocks, blocks of that prompt);
 *   scratch: snap_block_select_workspace_bytes(cfg, n_active, block_tokens) (the scores of every block).
 * snap_decode_attn_blocks   snap_decode_attn that visits only the listed blocks of the third section
 *   (arguments as there, plus the two arrays snap_block_select wrote, same n_blocks);
 *   scratch: snap_decode_blocks_workspace_bytes(cfg, n_active, block_tokens, n_blocks).
 * All three enqueue on cuda_stream and return; device-side conditions go to status_dev.
 */
int64_t snap_block_stats_bytes(const snap_config_t* cfg, int32_t block_tokens);
int snap_block_stats(const snap_config_t* cfg, const snap_layout_t* layout, const int32_t* slot_ids_dev,
                     int32_t n_seqs, const void* k_cache_dev, const int32_t* valid_topk_dev,
                     int32_t block_tokens, void* stats_dev, uint32_t* status_dev, void* cuda_stream);
int snap_block_select(const snap_config_t* cfg, const snap_layout_t* layout, const void* q_dev,
                      const int32_t* slot_ids_dev, int32_t n_active, const void* stats_dev,
                      const int32_t* valid_topk_dev, int32_t block_tokens, int32_t n_blocks,
                      int32_t* block_idx_dev, int32_t* n_selected_dev, void* workspace_dev, size_t workspace_bytes,
                      uint32_t* status_dev, void* cuda_stream);
int64_t snap_block_select_workspace_bytes(const snap_config_t* cfg, int32_t n_active, int32_t block_tokens);
int64_t snap_decode_blocks_workspace_bytes(const snap_config_t* cfg, int32_t n_active, int32_t block_tokens,
                                           int32_t n_blocks);
int snap_decode_attn_blocks(const snap_config_t* cfg, const snap_layout_t* layout, const void* q_dev,
                            const void* k_new_dev, const void* v_new_dev, const int32_t* slot_ids_dev,
                            int32_t n_active, void* k_cache_dev, void* v_cache_dev, int32_t* seq_len_dev,
                            const int32_t* valid_topk_dev, int32_t block_tokens, int32_t n_blocks,
                            const int32_t* block_idx_dev, const int32_t* n_selected_dev, void* out_dev,
                            void* workspace_dev, size_t workspace_bytes, uint32_t* status_dev, void* cuda_stream);

/*
 * Rotary positions (the encoding that Section 3.2 takes as applied before caching).
 *
 * Pair i of rot_dim / 2 turns by the angle position * f_i:
 *     a' = m (a cos - b sin),   b' = m (b cos + a sin)
 * with (a, b) the dims (rot_offset + i, rot_offset + rot_dim / 2 + i) of a head, or, interleaved,
 * (rot_offset + 2 i, rot_offset + 2 i + 1); the head's other dims pass unchanged.  The frequencies
 * f_i are radians per position in double precision, on the device; snap_rope_table fills a host
 * array with them (any other frequencies can be passed as well):
 *   PLAIN    f_i = base^(-2 i / rot_dim)
 *   LINEAR   f_i / factor
 *   LLAMA3   f_i / factor for wavelengths over original_len / low_freq, f_i for those under
 *            original_len / high_freq, between them ((1 - s) / factor + s) f_i with
 *            s = (original_len / wavelength - low_freq) / (high_freq - low_freq)
 *   YARN     (1 - r) f_i + r f_i / factor, r = clamp((i - lo) / (hi - lo), 0, 1) with
 *            lo = floor(c(beta_fast)), hi = ceil(c(beta_slow)), limited to [0, rot_dim - 1], and
 *            c(n) = rot_dim ln(original_len / (2 pi n)) / (2 ln base)
 * and m = magnitude, or, when that is 0, 1 (YARN: 0.1 ln(factor) + 1).
 */
#define SNAP_ROPE_PLAIN 0
#define SNAP_ROPE_LINEAR 1
#define SNAP_ROPE_LLAMA3 2
#define SNAP_ROPE_YARN 3
typedef struct snap_rope_config {
  int32_t rot_dim;        /* dims of a head that are rotated: even, >= 2 */
  int32_t rot_offset;     /* the first of them (latent layout: 512 of 576) */
  int32_t interleaved;    /* 0: a pair is dims i and i + rot_dim / 2, 1: dims 2 i and 2 i + 1 */
  int32_t scaling;        /* SNAP_ROPE_* */
  double base, factor;    /* > 1; >= 1 (LINEAR, LLAMA3, YARN) */
  double original_len;    /* LLAMA3, YARN: the context the model was trained on */
  double low_freq, high_freq;    /* LLAMA3, 0 < low_freq < high_freq */
  double beta_fast, beta_slow;   /* YARN, beta_fast > beta_slow > 0 */
  double magnitude;       /* >= 0; 0: the scaling's own */
} snap_rope_config_t;

/* Host only: the rot_dim / 2 frequencies and the magnitude (either may be NULL). */
int snap_rope_table(const snap_rope_config_t* rope, double* freqs_host, double* magnitude_host);

/*
 * Rotates the queries and / or keys of n_tokens tokens (at most 2^31 - 256); token t is at positions_dev[t].
 *   q_dev, q_out_dev  element (t, h, c) at [t * token_stride + h * head_stride + c], Hq heads; k_dev, k_out_dev
 *             alike with Hkv heads.  q_dev and q_out_dev, or k_dev and k_out_dev, may both be NULL.
 *             An output may be its own input (same pointer and strides); any other overlap is not allowed.
 *             Strides in elements, multiples of 16 bytes, and no head of an output may overlap another.
 *   freqs_dev [rot_dim / 2] double;  positions_dev [n_tokens] int32, any value
 *   inverse   1: turns by minus the angle (magnitude as before): the transposed map, i.e. the
 *             gradient with respect to the input, given the gradient of the output
 * Angles and their reduction are in double precision, the rotation in single, one rounding at the
 * end.  Only rot_dim, rot_offset, interleaved, scaling, factor and magnitude of rope are used.  No workspace.
 */
int snap_rope(const snap_config_t* cfg, const snap_rope_config_t* rope, const double* freqs_dev,
              const int32_t* positions_dev, int32_t n_tokens,
              const void* q_dev, int64_t q_token_stride, int64_t q_head_stride,
              void* q_out_dev, int64_t q_out_token_stride, int64_t q_out_head_stride,
              const void* k_dev, int64_t k_token_stride, int64_t k_head_stride,
              void* k_out_dev, int64_t k_out_token_stride, int64_t k_out_head_stride,
              int32_t inverse, void* cuda_stream);

/*
 * A cache in pages (the uncompressed cache that the paper's baseline decodes over).
 *
 * A page holds page_tokens rows of every KV head; row r of a sequence is row r mod page_tokens of
 * its page number page_table[slot][r / page_tokens].  Element c of row o of KV head h of page p is
 *     k_pages_dev[p * k_page_stride + h * k_head_stride + o * k_row_stride + c]
 * (strides in elements, multiples of 16 bytes; both [page][head][row][dim] and [page][row][head][dim]
 * are such layouts), V alike with d_v.
 *   page_table_dev  [max_seqs][max_pages] int32; entries past a sequence's last row are not read
 *   seq_len_dev     [max_seqs] int32: rows of each slot's sequence
 *   weights         [max_seqs][Hkv][max_pages * page_tokens] float: accumulated attention weight of each row
 * Rows need not be in position order: attention does not depend on it, and snap_paged_append takes
 * positions apart from rows.  Sequences may share pages that are only read.
 * The calls take heads up to 256 wide and no latent layout (SNAP_ERR_UNSUPPORTED otherwise).  bf16 layers are attended
 * fastest with heads of 64, 128 or 256 dims and pages of a multiple of 16 rows, then of 8.
 * All can be captured into CUDA graphs.  Lengths, tables and slots are read on the device when a call runs; nothing may
 * change them while it does.
 */
typedef struct snap_paged {
  int32_t page_tokens;    /* rows of a page, >= 1 */
  int32_t n_pages;        /* pages of the pool */
  int32_t max_pages;      /* entries of a page-table row; page_tokens * max_pages <= 2^30 */
  int32_t reserved;       /* 0 */
  int64_t k_page_stride, k_head_stride, k_row_stride;
  int64_t v_page_stride, v_head_stride, v_row_stride;
} snap_paged_t;

/*
 * Writes the K/V rows of n_tokens new tokens (at most 2^31 - 256), rotating the keys (and queries) on the way when rope is given.
 *   slot_ids_dev [n_tokens] int32: the slot of each token's sequence; -1 = padding, nothing of that token is
 *             read or written
 *   rows_dev  [n_tokens] int32: the row each token is written to; afterwards seq_len[slot] is at least row + 1.
 *             No (slot, row) twice.  NULL: every token is its sequence's next one, row = seq_len[slot], and
 *             seq_len[slot] grows by one; a slot that is listed a second time in the call is skipped
 *             (SNAP_DEV_BAD_SLOT); at most 65536 tokens (SNAP_ERR_INVALID_ARG).
 *   rope, freqs_dev, positions_dev: as in snap_rope; rope NULL = the keys are stored as given (the other
 *             two are ignored); positions_dev NULL = the position is the row
 *   k_dev, v_dev  (t, h, c) at [t * token_stride + h * head_stride + c]
 *   k_out_dev NULL, or [n_tokens][Hkv][d_qk] dense: the keys as stored (what snap_prefill_attn reads); may be
 *             k_dev when that is dense
 *   q_dev, q_out_dev  NULL, or the queries and where they go rotated, q_out dense [n_tokens][Hq][d_qk]; may be
 *             q_dev when that is dense
 *   weights_dev  NULL, or the weights array: the entries of the rows written are set to 0
 * A token whose row lies past the page table, or on a page number out of range, is skipped (SNAP_DEV_BAD_PAGE),
 * its outputs too.  No workspace.
 */
int snap_paged_append(const snap_config_t* cfg, const snap_paged_t* paged,
                      const int32_t* slot_ids_dev, const int32_t* rows_dev, int32_t n_tokens,
                      const snap_rope_config_t* rope, const double* freqs_dev, const int32_t* positions_dev,
                      const void* q_dev, int64_t q_token_stride, int64_t q_head_stride, void* q_out_dev,
                      const void* k_dev, int64_t k_token_stride, int64_t k_head_stride, void* k_out_dev,
                      const void* v_dev, int64_t v_token_stride, int64_t v_head_stride,
                      void* k_pages_dev, void* v_pages_dev, const int32_t* page_table_dev,
                      int32_t* seq_len_dev, float* weights_dev, uint32_t* status_dev, void* cuda_stream);

/*
 * Attention of one token per sequence over its pages: out[i][h] = softmax(scale * q[i][h] . K^T) V over rows
 * [0, seq_len[slot_ids[i]]) of KV head h / (Hq/Hkv).  Nothing is appended.
 *   q_dev [n_active][Hq][d_qk], out_dev [n_active][Hq][d_v], dense.  A sequence without rows, and a slot out of
 *             range (SNAP_DEV_BAD_SLOT), get zeros; a slot id of -1 is padding: its out rows are zeros too.
 *             Rows on a page number out of range are left out (SNAP_DEV_BAD_PAGE), as are rows past the page table.
 *   seq_len_dev  need not be the cache's own lengths: with shorter ones the token sees the rows before them
 *   weights_out_dev  NULL, or the weights array: for every row r the token attends,
 *                 weights_out[slot][kvh][r] = weights_in[slot][kvh][r] + sum over the group's heads of its softmax weight
 *             (weights_in_dev NULL = 0; it may be weights_out_dev).  Other entries are left alone, those of rows that are
 *             left out among them.  The slots of
 *             one call must then be distinct: of a slot that is listed again only the first entry's weights
 *             count (SNAP_DEV_BAD_SLOT).  At most 2048 query heads per KV head (SNAP_ERR_UNSUPPORTED).
 * A NaN or an infinity among the rows a token attends makes the outputs it enters non-finite, which of the two is not
 * specified (in single precision a key or query above 3.402e38 may count as infinite); rows that are left out, and what lies
 * behind a sequence's last row, may hold anything.  A token whose every logit is -infinity gets zeros.  A sequence of one
 * row returns its values unrounded (those of at least 1e-30 in size; a zero may lose its sign).
 * The rows of all sequences are split evenly over the GPU whatever their lengths and joined in a fixed order:
 * equal inputs give equal bits.  n_active times the rows that a slot can have must stay below about
 * 2^33, and times the KV heads below 2^39 (SNAP_ERR_UNSUPPORTED).
 * Scratch: snap_paged_decode_workspace_bytes(cfg, paged, n_active, with_weights); calls that can overlap on the
 * GPU need scratch of their own.
 */
int64_t snap_paged_decode_workspace_bytes(const snap_config_t* cfg, const snap_paged_t* paged, int32_t n_active,
                                          int32_t with_weights);
int snap_paged_decode_attn(const snap_config_t* cfg, const snap_paged_t* paged, const void* q_dev,
                           const int32_t* slot_ids_dev, int32_t n_active,
                           const void* k_pages_dev, const void* v_pages_dev, const int32_t* page_table_dev,
                           const int32_t* seq_len_dev, const float* weights_in_dev, float* weights_out_dev,
                           void* out_dev, void* workspace_dev, size_t workspace_bytes,
                           uint32_t* status_dev, void* cuda_stream);

/*
 * Eviction by accumulated attention weight.  For each of n_seqs sequences the rows that stay are copied from
 * slot src_slots[i] to slot dst_slots[i] (whose page-table row holds the caller's free pages), per KV head and
 * in order: of len = seq_len[src] rows,
 *     all of them                                                          when len <= Ls + K + Lr
 *     [0, Ls), the K rows of [Ls, len - Lr) with the largest weights_in[src][kvh][row]
 *     (ties to the lower row; NaN ranks lowest), [len - Lr, len)           otherwise
 * with l_sink, topk and l_recent of cfg.  The source slot and its pages stay as they are; the caller then uses
 * dst and frees src.
 *   seq_len_dev   [max_seqs]; seq_len[dst] = min(len, Ls + K + Lr)
 *   weights_out_dev  NULL, or the weights array the kept rows' weights go to at [dst] (weights_in_dev itself is fine)
 *   kept_rows_dev NULL, or [n_seqs][Hkv][Ls + K + Lr] int32: the source rows kept, -1 after the last
 * A slot out of range, or a dst that is a src of the call or an earlier entry's dst, skips that sequence
 * (SNAP_DEV_BAD_SLOT; its kept_rows are -1).  A destination page may hold nothing that is in use, the source's rows
 * included, and is listed once (not checked).  A source or destination page number out of range skips its rows
 * (SNAP_DEV_BAD_PAGE).
 * Scratch: snap_paged_evict_workspace_bytes(cfg, paged, n_seqs).
 */
int64_t snap_paged_evict_workspace_bytes(const snap_config_t* cfg, const snap_paged_t* paged, int32_t n_seqs);
int snap_paged_evict(const snap_config_t* cfg, const snap_paged_t* paged, const int32_t* src_slots_dev,
                     const int32_t* dst_slots_dev, int32_t n_seqs, void* k_pages_dev, void* v_pages_dev,
                     const int32_t* page_table_dev, int32_t* seq_len_dev, const float* weights_in_dev,
                     float* weights_out_dev, int32_t* kept_rows_dev, void* workspace_dev, size_t workspace_bytes,
                     uint32_t* status_dev, void* cuda_stream);

/*
 * A step's pages and tokens, decided on the device: which pages the new rows of each sequence go to, and the lists that
 * snap_paged_append, snap_rope and snap_paged_q8_append take.  Request i is slot slot_ids[i] and n = new_tokens[i]; requests
 * are served as if one after the other:
 *   n < 0   the sequence has ended.  Every page that its table row holds (an entry in [0, n_pages)) goes onto the stack of free
 *           pages, in the row's order; the row becomes -1 and seq_len[slot] 0.  (The pages of all sequences that end go onto
 *           the stack before any is granted.)
 *   n >= 0  the sequence, of len = seq_len[slot] rows, is to grow by n.  Missing are those of the entries
 *           [ceil(len / page_tokens), ceil((len + n) / page_tokens)) of its row that hold no page (others keep the one they hold: one
 *           set aside before, or granted to tokens that were given up); the k-th page granted in the call is the k-th from the
 *           stack's top.  Refused, as a whole, is a request whose len + n lies past the page table (SNAP_DEV_BAD_PAGE), or with
 *           which the tokens wanted so far (its own and those of all requests before it, refused ones as well, but for those
 *           past the table) exceed n_tokens_max, or, when it misses any, the pages missing so far those that are
 *           free (SNAP_DEV_NO_ROOM).
 *   A slot of -1 is padding; a slot out of range or listed before is skipped (SNAP_DEV_BAD_SLOT).
 *   page_table_in_dev, page_table_out_dev  [max_seqs][max_pages], the same array or two that do not overlap (checked): with two, the rows of the
 *             slots listed are written whole and the table that a running step reads stays as it is; rows of other slots are neither read
 *             nor written, so a program that uses two tables in turn lists every slot that lives, those that do not grow with 0
 *   seq_len_dev [max_seqs]: read; 0 where the sequence has ended (appending counts the new rows, not this call)
 *   free_pages_dev [n_pages]: the stack of free pages, its top last; n_free_in_dev, n_free_out_dev [1]: how many it holds before and
 *             after (the same or two).  Entries are written only from n_free_in on.  More than n_pages: SNAP_DEV_BAD_PAGE, the rest is dropped.
 *   granted_dev NULL, or [n_seqs]: n of the requests served, 0 of the others
 *   first_rows_dev [n_seqs]: the row of each request's first new token, seq_len[slot] (0: ended, skipped)
 *   cu_tokens_dev [n_seqs + 1]: sums of the granted tokens before each request, and of all
 *   token_slots_dev, token_rows_dev [n_tokens_max]: slot and row of every token granted, request by request; -1 and 0 behind the last (as
 *             snap_paged_append takes them for slot_ids and rows, with n_tokens_max tokens, and snap_rope the rows for positions)
 * Of paged, only page_tokens, n_pages and max_pages are used; of cfg, max_seqs.  At most 65536 requests.  Sequences that share
 * pages must not end through this call (a page would go onto the stack twice).
 * Scratch: snap_paged_plan_workspace_bytes(cfg, paged, n_seqs).
 */
int64_t snap_paged_plan_workspace_bytes(const snap_config_t* cfg, const snap_paged_t* paged, int32_t n_seqs);
int snap_paged_plan(const snap_config_t* cfg, const snap_paged_t* paged, const int32_t* slot_ids_dev,
                    const int32_t* new_tokens_dev, int32_t n_seqs, const int32_t* page_table_in_dev,
                    int32_t* page_table_out_dev, int32_t* seq_len_dev, int32_t* free_pages_dev,
                    const int32_t* n_free_in_dev, int32_t* n_free_out_dev, int32_t n_tokens_max, int32_t* granted_dev,
                    int32_t* first_rows_dev, int32_t* cu_tokens_dev, int32_t* token_slots_dev, int32_t* token_rows_dev,
                    void* workspace_dev, size_t workspace_bytes, uint32_t* status_dev, void* cuda_stream);

/*
 * A cache in pages of 8-bit numbers.  Element c of row o of KV head h of page p is
 *     e4m3(k_pages_dev[p * k_page_stride + h * k_head_stride + o * k_row_stride + c])
 *         * k_scales_dev[(p * Hkv + h) * (page_tokens / block_tokens) + o / block_tokens]
 * (strides in bytes, multiples of 16), V alike: block_tokens consecutive rows of a KV head share a scale, positive and finite.
 * What the append writes are powers of two: of a floating format a finer scale keeps no more bits, and a number moves to
 * a larger one unrounded, unless it falls below 2^-6 of it.  Page tables, lengths and slots are those of the cache
 * in pages above; cfg->dtype is the type of queries, keys, values and outputs.  Heads up to 256 wide, no latent layout.
 */
typedef struct snap_paged_q8 {
  snap_paged_t pages;     /* strides in bytes */
  int32_t block_tokens;   /* rows that share a scale: a divisor of page_tokens */
  int32_t reserved;       /* 0 */
} snap_paged_q8_t;

/*
 * Writes the K/V rows of new tokens, rotating the keys (and queries) on the way when rope is given.  Entry i adds the tokens
 * [cu_tokens[i], cu_tokens[i + 1]) to sequence slot_ids[i] as the rows from first_rows[i] on, which then are its last:
 * seq_len[slot] = first_rows[i] + their number (no tokens: it stays).
 *   slot_ids_dev [n_seqs]: -1 = padding, nothing of that entry is read or written; a slot out of range, or listed before, is
 *             skipped (SNAP_DEV_BAD_SLOT).  At most 65536 entries.
 *   cu_tokens_dev [n_seqs + 1]: must not decrease (not checked).  Tokens from cu_tokens[n_seqs] on are padding, of which nothing is
 *             read or written; n_tokens (at most 2^31 - 65536) is what there is room for.
 *   first_rows_dev [n_seqs]: may be less than the sequence's length: rows from there on are given up.  May not be seq_len_dev itself.
 *   rope, freqs_dev, positions_dev [n_tokens], k_dev, v_dev, k_out_dev, q_dev, q_out_dev: as in snap_paged_append (positions_dev
 *             NULL: the row; k_out is rounded from the rotated key, not from what the page holds)
 * The scale of a block is 2^e, e the smallest integer from -126 to 120 with f * max |x| <= 448 * 2^e over the
 * inputs x of the rows written to it, f = max(1, sqrt(2) magnitude) for keys that are rotated and 1 otherwise
 * (a pair grows by sqrt(2) magnitude at most); of a block that holds rows of the sequence already, below
 * first_rows, it is no less than before, and where it grows those rows move to it.  A number is rotated in
 * single precision, divided by the scale (whatever positive number a block that holds rows has) and rounded
 * once, to nearest even; beyond 448 (only past 2^120) it is 448.  NaN stays NaN and does not count for the
 * scale; a block with an infinity has the scale 2^120.
 * Rows past the page table or on a page number out of range are skipped (SNAP_DEV_BAD_PAGE), their outputs too; so is an
 * entry with a negative first row, as a whole.  A page that is written may be listed once (not checked).  No workspace.
 */
int snap_paged_q8_append(const snap_config_t* cfg, const snap_paged_q8_t* paged,
                         const int32_t* slot_ids_dev, const int32_t* cu_tokens_dev, const int32_t* first_rows_dev,
                         int32_t n_seqs, int32_t n_tokens,
                         const snap_rope_config_t* rope, const double* freqs_dev, const int32_t* positions_dev,
                         const void* q_dev, int64_t q_token_stride, int64_t q_head_stride, void* q_out_dev,
                         const void* k_dev, int64_t k_token_stride, int64_t k_head_stride, void* k_out_dev,
                         const void* v_dev, int64_t v_token_stride, int64_t v_head_stride,
                         void* k_pages_dev, void* v_pages_dev, float* k_scales_dev, float* v_scales_dev,
                         const int32_t* page_table_dev, int32_t* seq_len_dev, uint32_t* status_dev, void* cuda_stream);

/*
 * Attention of the last q_len tokens of each sequence over its pages: with len = seq_len[slot_ids[i]],
 *     out[i][u][h] = softmax(scale * q[i][u][h] . K^T) V   over rows [0, len - q_len + 1 + u)
 * of KV head h / (Hq/Hkv): every token sees the rows up to its own.  Nothing is appended.
 *   q_dev [n_active][q_len][Hq][d_qk], out_dev [n_active][q_len][Hq][d_v], dense; 1 <= q_len <= 1024.  A token that sees no row gets zeros;
 *             slots, padding, page numbers out of range and lengths as in snap_paged_decode_attn
 * Numbers enter the products as they are stored (queries of single precision to 22 bits; of any query what
 * lies 2^29 and more below its largest number loses bits, at 2^39 it is cut off); logits, weights and sums are
 * in single precision, whatever the scales. Each weight enters as a number of 21 bits or, far below the
 * largest product of weight and scale of the same query head among 32 rows on scales within 2^6 of one
 * another, as a multiple of 2^-24 of that (single-precision layers 2^-36); one below 2^-126 of the largest
 * weight is zero.  The largest value times the rows of a sequence has to lie below 2^121 (sums are of single
 * precision).  A NaN among the rows that a token attends makes the outputs it enters NaN, and those of no
 * other token.  (An infinity that was appended is 448 * 2^120, past single precision as a value.)
 * Rows that are left out, and what lies behind a sequence's last row, may hold anything, their scales too.
 * Work is split and joined as in snap_paged_decode_attn: equal inputs give equal bits.
 * Scratch: snap_paged_q8_decode_workspace_bytes(cfg, paged, n_active, q_len); calls that can overlap on the GPU need scratch
 * of their own.
 */
int64_t snap_paged_q8_decode_workspace_bytes(const snap_config_t* cfg, const snap_paged_q8_t* paged, int32_t n_active,
                                             int32_t q_len);
int snap_paged_q8_decode_attn(const snap_config_t* cfg, const snap_paged_q8_t* paged, const void* q_dev,
                              const int32_t* slot_ids_dev, int32_t n_active, int32_t q_len,
                              const void* k_pages_dev, const void* v_pages_dev, const float* k_scales_dev,
                              const float* v_scales_dev, const int32_t* page_table_dev, const int32_t* seq_len_dev,
                              void* out_dev, void* workspace_dev, size_t workspace_bytes, uint32_t* status_dev,
                              void* cuda_stream);

/*
 * The reverse of the append: token cu_tokens[i] + j of k_dev and v_dev receives row first_rows[i] + j of
 * sequence slot_ids[i], rounded once (bf16: exact on scales that are powers of two, unless they leave its
 * range).  Entries, tokens and padding as in snap_paged_q8_append, but a slot may be listed any number of times
 * and no length is looked at.
 *   k_dev, v_dev  (t, h, c) at [t * token_stride + h * head_stride + c], strides multiples of 16 bytes, no head of an
 *             output may overlap another
 * Tokens of rows past the page table, or on a page number out of range (SNAP_DEV_BAD_PAGE), are left as they are.  No workspace.
 */
int snap_paged_q8_gather(const snap_config_t* cfg, const snap_paged_q8_t* paged,
                         const int32_t* slot_ids_dev, const int32_t* cu_tokens_dev, const int32_t* first_rows_dev,
                         int32_t n_seqs, int32_t n_tokens,
                         const void* k_pages_dev, const void* v_pages_dev, const float* k_scales_dev, const float* v_scales_dev,
                         const int32_t* page_table_dev,
                         void* k_dev, int64_t k_token_stride, int64_t k_head_stride,
                         void* v_dev, int64_t v_token_stride, int64_t v_head_stride,
                         uint32_t* status_dev, void* cuda_stream);

/*
 * Testing and tuning aids (the paper has no counterpart).  Each option is one non-negative
 * integer, process-wide, 0 by default = the library's own choice; changing one while calls are
 * in flight on other threads is not synchronised.  Every kernel choice yields the same results
 * within the tolerances of the tests; the options exist so that the slower kernels and other
 * split counts can be tested and timed.  At the first use of any option each is seeded once
 * from its environment variable (named on the right); the environment is not read again.
 * Returns the option's previous value, or SNAP_ERR_INVALID_ARG.
 */
#define SNAP_OPT_SCORE_KERNEL 0          /* 1: mma.sync score kernel, 2: SIMT, 3: tcgen05 without CTA pairs  SNAP_SCORE_PATH=mma|simt|single */
#define SNAP_OPT_DECODE_GQA_KERNEL 1     /* 1: packed-FP32 GQA decode kernel; the tensor-core kernel 2: always with a merge
                                               launch, 3: with the in-kernel merge of small batches outside stream capture
                                               too (by default only under capture)   SNAP_DECODE_GQA=simt|split|fused */
#define SNAP_OPT_DECODE_LATENT_KERNEL 2  /* 1: mma.sync latent decode kernel        SNAP_DECODE_MLA=mma      */
#define SNAP_OPT_DECODE_NSPLIT 3         /* n: splits per (sequence, KV head)       SNAP_DECODE_NSPLIT=n     */
#define SNAP_OPT_SCORE_NSPLIT 4          /* n: candidate splits of the longest prompt  SNAP_SCORE_NSPLIT=n   */
#define SNAP_OPT_WIDE_STAGES 5           /* n: ring depth of the wide score kernel  SNAP_WIDE_STAGES=n       */
#define SNAP_OPT_PREFILL_KERNEL 6        /* 1: portable prefill attention kernel    SNAP_PREFILL_PATH=simt   */
#define SNAP_OPT_PREFILL_SINGLE_HEADS 7  /* 1: one head per CTA in prefill attention  SNAP_PREFILL_HEADS=1   */
#define SNAP_OPT_REFINE_OFF 8            /* 1: skip the double-precision re-scoring near the top-K
                                               threshold and near the block-selection threshold
                                               (single-precision order)            SNAP_REFINE=0            */
#define SNAP_OPT_COUNT 9
int snap_debug_set_option(int option, int value);

/* Text for a snap_status value (static storage). */
const char* snap_status_string(int status);

/* Number of kernels this library has launched in this process (for benchmarks' bookkeeping). */
int64_t snap_kernel_launch_count(void);

#ifdef __cplusplus
}
#endif
#endif /* SNAPSTREAM_H_ */

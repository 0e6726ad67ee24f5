/*
 * delta_attn.h -- C ABI of the MI355X (gfx950) Delta Attention prefill library.
 *
 * Delta Attention (arXiv 2505.11254, Sec. 3, Algorithm 1) corrects a sparse
 * attention output with the difference between dense and sparse attention
 * taken at every gamma-th query row:
 *
 *   out_i = (A*V)_i + [ (A~V)_a - (A*V)_a ],   a = floor(i/gamma)*gamma   (Eq. 6)
 *
 * where A*V is StreamingLLM attention (sink tokens + sliding window, softmax
 * normalised over the selected keys) and A~V is dense causal attention
 * evaluated only at the anchor rows a (Eq. 4).  Rows past the last whole
 * group of gamma rows are computed densely (implementation-details appendix).
 *
 * Conventions shared by every entry point
 * ---------------------------------------
 * Tensors are token-major, contiguous, IEEE bfloat16 (bit patterns):
 *   q, out : [T, Hq, d]      k, v : [T, Hkv, d]
 * T = B*N for the fixed-length calls; T = cu_seqlens[B] for the _varlen
 * calls, where sequence b occupies token rows [cu_seqlens[b], cu_seqlens[b+1]).
 * All positions (causality, sinks, window, anchors) are local to a sequence;
 * sequences never attend to each other.
 *   - scale 1/sqrt(d) (Eq. 1), causal with the diagonal included (Sec. 2);
 *   - GQA: query head h reads kv head floor(h / (Hq/Hkv));
 *   - sparse key set of row i: { j <= i : j < n_sink  or  i - j < window };
 *   - anchors: rows i with i mod gamma = 0 and i < floor(L/gamma)*gamma.
 * d must be 64 or 128.  Every pointer is a device pointer, 16-byte aligned;
 * the caller owns all memory.  `out` must not overlap q, k, v or the
 * workspace.  `stream` is a hipStream_t (NULL: the null stream).
 *
 * Calls validate every argument before any HIP call; on error nothing is
 * enqueued and `out` is untouched.  On success the work is only enqueued on
 * `stream`; nothing synchronises.  Device faults surface at the caller's
 * next synchronisation.  cu_seqlens (int32, B+1 entries, device) must start
 * at 0 and be non-decreasing with every length <= max_seqlen; the library
 * cannot check device-resident values, and violating this is undefined.
 * Concurrent calls must not share a workspace.  No call keeps a pointer.
 */
#ifndef DELTA_ATTN_H
#define DELTA_ATTN_H

#include <stddef.h>
#include <stdint.h>

#ifdef __cplusplus
extern "C" {
#endif

#define DA_ABI_VERSION 2

typedef enum {
  DA_OK = 0,
  DA_ERR_NULL = 1,        /* a required pointer is NULL */
  DA_ERR_SHAPE = 2,       /* B, N/max_seqlen, Hq or Hkv < 1, Hq % Hkv != 0, or sizes overflow */
  DA_ERR_PARAM = 3,       /* window < 1, n_sink < 0 or gamma < 1 */
  DA_ERR_UNSUPPORTED = 4, /* d not in {64, 128}, or the current device is not gfx950 */
  DA_ERR_ALIGN = 5,       /* a tensor or workspace pointer is not 16-byte aligned */
  DA_ERR_WORKSPACE = 6,   /* workspace NULL or too small (see da_workspace_bytes()) */
  DA_ERR_HIP = 7          /* a HIP runtime call failed; see da_last_hip_error() */
} da_status;

/*
 * Delta Attention prefill (Algorithm 1), fixed-length batch of B sequences
 * of N tokens.  Writes the corrected output to `out`.
 * workspace: device memory of da_workspace_bytes(B, N, Hq, Hkv, d, gamma)
 * bytes or more (less: see there), used for the strided rows' partial results
 * and fp32 rows at the anchors; its contents on entry do not matter.
 * Two launch schedules compute the result (see delta_attn_prefill_steps);
 * this call takes the fused one whenever da_fused_supported(Hq, Hkv, gamma),
 * else the unfused one.  The fused schedule rounds a corrected row to bf16
 * once (bf16(sparse + Delta)); the unfused one rounds the sparse row first
 * and again after adding Delta.  Anchor rows, covered groups and dense tail
 * rows are bitwise the same under both.
 */
da_status delta_attn_prefill(const void* q, const void* k, const void* v, void* out,
                             int B, int Hq, int Hkv, int N, int d,
                             int window, int n_sink, int gamma,
                             void* workspace, size_t workspace_bytes, void* stream);

/* As delta_attn_prefill for a ragged batch packed with cu_seqlens (device, int32). */
da_status delta_attn_prefill_varlen(const void* q, const void* k, const void* v, void* out,
                                    const int32_t* cu_seqlens, int B, int max_seqlen,
                                    int Hq, int Hkv, int d, int window, int n_sink, int gamma,
                                    void* workspace, size_t workspace_bytes, void* stream);

/*
 * The steps of Algorithm 1 one at a time, for measuring each kernel on its
 * own.  `steps` is a non-empty subset of DA_STEP_SPARSE, DA_STEP_DENSE_ROWS
 * and DA_STEP_CORRECT, optionally with DA_STEP_FUSED; the steps it names run
 * in the schedule's order, on `stream`, with the same buffers.  A later step
 * reads what earlier calls left in `out` and the workspace.
 * Unfused schedule (no DA_STEP_FUSED), in this order:
 *   DA_STEP_SPARSE      step 1: A*V for every row into `out`, plus an fp32 copy
 *                       of the anchor rows in the workspace;
 *   DA_STEP_DENSE_ROWS  steps 2-3: A~V at the anchors (Eq. 4) and at the dense
 *                       tail rows, as key-chunk partial results in the workspace;
 *   DA_STEP_CORRECT     steps 4-5 (Eq. 6): merge the partials, form Delta and
 *                       add it to the gamma rows of each group in `out`.
 * Fused schedule (DA_STEP_FUSED), in this order:
 *   DA_STEP_DENSE_ROWS  as above;
 *   DA_STEP_CORRECT     merge the partials into fp32 dense rows (workspace);
 *   DA_STEP_SPARSE      steps 1, 4-5: A*V for every row, stored as
 *                       bf16(A*V + Delta) (Eq. 6) with Delta formed from the
 *                       anchor's fp32 sparse row inside the kernel; anchor and
 *                       tail rows store the dense row.
 * The fused schedule needs every group of gamma rows inside one head's row
 * slab of a sparse-kernel workgroup (da_fused_supported); otherwise
 * DA_STEP_FUSED gives DA_ERR_UNSUPPORTED.  All steps of one schedule, in
 * order (or one call with DA_STEP_ALL, plus DA_STEP_FUSED for the fused
 * one), equal one delta_attn_prefill[_varlen] call that takes that schedule,
 * given da_workspace_bytes() or more.  DA_STEP_DENSE_ROWS and DA_STEP_CORRECT in
 * calls of their own lay the partials out alike for any two sizes from
 * da_workspace_bytes() on, and for any two accepted ones below it.
 * cu_seqlens may be NULL: then B sequences of max_seqlen tokens each.
 * Other arguments and errors as delta_attn_prefill_varlen; a `steps` value
 * with none of the three step bits, or with other bits, gives DA_ERR_PARAM.
 */
#define DA_STEP_SPARSE 1u
#define DA_STEP_DENSE_ROWS 2u
#define DA_STEP_CORRECT 4u
#define DA_STEP_ALL 7u
#define DA_STEP_FUSED 8u
da_status delta_attn_prefill_steps(const void* q, const void* k, const void* v, void* out,
                                   const int32_t* cu_seqlens, int B, int max_seqlen, int Hq,
                                   int Hkv, int d, int window, int n_sink, int gamma,
                                   void* workspace, size_t workspace_bytes, void* stream,
                                   unsigned steps);

/*
 * 1 if the fused schedule serves these sizes, else 0: some power of two h
 * dividing Hq/Hkv, h <= 8, has 256/h (the rows per query head of one sparse
 * workgroup) a multiple of gamma.  The fused schedule swaps the in-place
 * correction pass over `out` for a merge of the dense rows before the
 * sparse kernel, which then stores the corrected rows itself.
 */
int da_fused_supported(int Hq, int Hkv, int gamma);

/*
 * Correction variants of step 5 of Algorithm 1 (Sec. 3 and the interpolation
 * appendix): Steps 1-4 as in delta_attn_prefill; then, for the rows r of the
 * whole groups, out_r = (A*V)_r + c_r with, for anchor a_i = i*gamma and
 * Delta_i = (A~V)_{a_i} - (A*V)_{a_i}:
 *   DA_CORR_DELTA      c_r = Delta_{floor(r/gamma)}                    (Eq. 6)
 *   DA_CORR_RECOMPUTE  c_r = Delta_i at r = a_i, 0 elsewhere: the dense row
 *                      replaces the sparse one at anchors only         (Eq. 5)
 *   DA_CORR_INTERP     c_{a_i+k} = (1-b_k) Delta_i + b_k Delta_{i+1},
 *                      b_k = k/(gamma-1) rising from 0 to 1 over the group;
 *                      the last group keeps Delta_i.  Uses the next anchor,
 *                      so it is not causal.
 *   DA_CORR_EMA        exponential moving average with weight p0 in [0,1]
 *                      over repeat(Delta, gamma): E_r = (1-p0) E_{r-1} +
 *                      p0 D_r, E_{-1} = D_0; c_r = E_r
 *   DA_CORR_ABG        alpha-beta-gamma filter over Delta_0, Delta_1, ...
 *                      with coefficients (p0, p1, p2) for position, velocity
 *                      and acceleration; c_r = filtered Delta_{floor(r/gamma)}.
 *                      The recursion is unstable where the spectral radius of
 *                      (I - g e0^T) F exceeds 1 (gain g = (p0, p1, p2), F the
 *                      constant-acceleration transition with unit step), as
 *                      for (0.05, 1.25e-4, 2.08e-5): 1.0023 per anchor.  Its
 *                      output then grows geometrically with the anchor count,
 *                      and so do its rounding differences from an exact
 *                      evaluation.
 * Rows past the last whole group take the dense result.  DA_CORR_DELTA and
 * DA_CORR_RECOMPUTE take the fused schedule when da_fused_supported() (as
 * delta_attn_prefill does), the other modes the unfused one.  cu_seqlens may be
 * NULL (B sequences of max_seqlen tokens).  workspace needs
 * da_workspace_bytes_correction(..., mode) bytes.  Errors as
 * delta_attn_prefill_varlen, plus DA_ERR_PARAM for an unknown mode, a
 * non-finite parameter or an EMA weight outside [0,1].
 */
#define DA_CORR_DELTA 0
#define DA_CORR_RECOMPUTE 1
#define DA_CORR_INTERP 2
#define DA_CORR_EMA 3
#define DA_CORR_ABG 4
da_status delta_attn_prefill_correction(const void* q, const void* k, const void* v, void* out,
                                        const int32_t* cu_seqlens, int B, int max_seqlen, int Hq,
                                        int Hkv, int d, int window, int n_sink, int gamma,
                                        int mode, float p0, float p1, float p2, void* workspace,
                                        size_t workspace_bytes, void* stream);

/*
 * Delta Attention over other sparse bases (Sec. 3: the correction applies to
 * any sparse attention f*; Sec. 4 pairs it with StreamingLLM, MInference, HiP
 * and Star Attention).  f* is given by key-block lists: keys are grouped in
 * tiles of 64 positions and query rows in blocks of block_q rows, both local
 * to each sequence.  For sequence b, kv head g and query block qb the list
 * names the key tiles that the block's rows attend to; the tiles overlapping
 * the query block itself (tile >= qb*block_q/64) are always attended.  Row i
 * of a query head of group g then sees
 *   S(i) = { j <= i : tile(j) listed for (b, g, i/block_q), or
 *                     tile(j) >= (i/block_q)*block_q/64 },
 * normalised over S(i) only; Algorithm 1 runs on top unchanged.
 *
 * block_ptr: int32 [B][Hkv][nqb + 1], nqb = ceil(max_seqlen / block_q):
 *   offsets into block_idx; the list of (b, g, qb) is
 *   block_idx[block_ptr[(b*Hkv + g)*(nqb+1) + qb] .. block_ptr[... + qb + 1]).
 * block_idx: int32 key tile indices, ascending and unique within each list.
 *   Entries outside [0, qb*block_q/64) are skipped.
 * Both arrays are device memory owned by the caller; like cu_seqlens, their
 * consistency (offsets non-decreasing and inside block_idx, lists ascending
 * without repeats) is the caller's responsibility: the library cannot check
 * device-resident values, and violating it is undefined.
 * block_q must be 64, 128 or 256, and 256/h rows, h the largest power of two
 * dividing Hq/Hkv (at most 8), must not exceed it (one sparse workgroup's rows
 * per head lie in one query block); otherwise DA_ERR_UNSUPPORTED.
 */

/* f* alone under key-block lists, for every row.  cu_seqlens may be NULL (B
 * sequences of max_seqlen tokens).  Errors as sparse_attn_prefill_varlen,
 * plus DA_ERR_NULL (no lists), DA_ERR_PARAM (block_q) and DA_ERR_UNSUPPORTED. */
da_status blocksparse_attn_prefill(const void* q, const void* k, const void* v, void* out,
                                   const int32_t* cu_seqlens, int B, int max_seqlen, int Hq,
                                   int Hkv, int d, int block_q, const int32_t* block_ptr,
                                   const int32_t* block_idx, void* stream);

/* Delta Attention with f* under key-block lists.  steps = 0 runs the whole
 * path in the schedule the library picks (fused when
 * da_fused_supported_blocksparse()); other values select steps and schedule
 * as in delta_attn_prefill_steps.  Anchors are never assumed covered: Delta
 * is formed at every anchor.  workspace: da_workspace_bytes(B, max_seqlen,
 * Hq, Hkv, d, gamma) bytes. */
da_status delta_attn_prefill_blocksparse(const void* q, const void* k, const void* v, void* out,
                                         const int32_t* cu_seqlens, int B, int max_seqlen,
                                         int Hq, int Hkv, int d, int block_q,
                                         const int32_t* block_ptr, const int32_t* block_idx,
                                         int gamma, void* workspace, size_t workspace_bytes,
                                         void* stream, unsigned steps);

/* As da_fused_supported, with the sparse workgroup's rows per head also
 * within one query block of block_q rows (256/h <= block_q). */
int da_fused_supported_blocksparse(int Hq, int Hkv, int gamma, int block_q);

/* Workspace bytes delta_attn_prefill_correction needs (0 if the sizes or mode are invalid). */
size_t da_workspace_bytes_correction(int B, int max_seqlen, int Hq, int Hkv, int d, int gamma,
                                     int mode);

/*
 * Sparse attention alone (f*, StreamingLLM sink + window; the first step of
 * Algorithm 1): out_i = (A*V)_i for every row.  Needs no workspace.
 */
da_status sparse_attn_prefill(const void* q, const void* k, const void* v, void* out,
                              int B, int Hq, int Hkv, int N, int d, int window, int n_sink,
                              void* stream);
da_status sparse_attn_prefill_varlen(const void* q, const void* k, const void* v, void* out,
                                     const int32_t* cu_seqlens, int B, int max_seqlen,
                                     int Hq, int Hkv, int d, int window, int n_sink,
                                     void* stream);

/*
 * Dense causal attention for every row (f, Eq. 1): the quadratic baseline the
 * method is compared with (Sec. 4.1 latency study).  Needs no workspace.
 */
da_status dense_causal_attn_prefill(const void* q, const void* k, const void* v, void* out,
                                    int B, int Hq, int Hkv, int N, int d, void* stream);
da_status dense_causal_attn_prefill_varlen(const void* q, const void* k, const void* v,
                                           void* out, const int32_t* cu_seqlens, int B,
                                           int max_seqlen, int Hq, int Hkv, int d,
                                           void* stream);

/*
 * The same attentions under changed scores, for models that cap them or bias them by distance:
 *   s_ij = q_i.k_j / sqrt d,  s' = cap tanh(s / cap) if cap > 0, else s,
 *   weight_ij = exp(s'_ij - slopes[h] |i - j|) over the keys that row i sees.
 * cap: 0 (none), or from 2^-10 to 2^10; a capped score is off by up to cap 2^-20.  A score that is NaN
 *   stays NaN, and so does the row that sees its key, as without a cap.
 * slopes: fp32 [Hq] on the device, from -2^10 to 2^10, or NULL (none); a bias adds to a score's error up to
 *   |slope| 2^-10, and 2^-21 of |slope (i - j)| and of the row's largest score.
 * prefix (dense rows only): int32 [B] on the device, or NULL: rows of sequence b see its first
 *   prefix[b] tokens (as many as there are; none below 1) whole, and the others up to themselves.
 * cu_seqlens may be NULL (B sequences of max_seqlen tokens); packed documents see only themselves,
 * as in the other calls.  The correction is DA_CORR_DELTA's, its workspace
 * da_workspace_bytes(); everything else, errors included, is as in dense_causal_attn_prefill_varlen,
 * sparse_attn_prefill_varlen and delta_attn_prefill_varlen, whose results these calls give with
 * cap 0 and no slopes (dense: nor prefix), and DA_ERR_PARAM for another cap.
 */
da_status dense_attn_prefill_scored(const void* q, const void* k, const void* v, void* out,
                                    const int32_t* cu_seqlens, int B, int max_seqlen, int Hq,
                                    int Hkv, int d, float cap, const float* slopes,
                                    const int32_t* prefix, void* stream);
da_status sparse_attn_prefill_scored(const void* q, const void* k, const void* v, void* out,
                                     const int32_t* cu_seqlens, int B, int max_seqlen, int Hq,
                                     int Hkv, int d, int window, int n_sink, float cap,
                                     const float* slopes, void* stream);
da_status delta_attn_prefill_scored(const void* q, const void* k, const void* v, void* out,
                                    const int32_t* cu_seqlens, int B, int max_seqlen, int Hq,
                                    int Hkv, int d, int window, int n_sink, int gamma, float cap,
                                    const float* slopes, void* workspace, size_t workspace_bytes,
                                    void* stream);

/*
 * For callers that cannot allocate device memory (code under HIP graph
 * capture, tight serving loops, harnesses that forbid hipMalloc): the whole
 * Delta path of delta_attn_prefill[_varlen] (cu_seqlens NULL: B sequences of
 * max_seqlen tokens each), with its workspace in a static device array of
 * DA_NOALLOC_SCRATCH_BYTES that every device the library runs on holds until
 * the process ends.  The call allocates nothing.  The strided rows split
 * their key axis into as many chunks as fit that array (fewer than
 * delta_attn_prefill takes when its workspace would not fit), so the two
 * calls can differ by rounding.  Returns DA_ERR_WORKSPACE when even one key
 * chunk does not fit (for instance a single 1M-token sequence with 32 query
 * heads); otherwise the statuses of delta_attn_prefill.  All calls on one
 * device share its array, which keeps the last call's contents: calls that
 * overlap on one device (other streams, other threads) race, so serialise
 * them.
 */
#define DA_NOALLOC_SCRATCH_BYTES ((size_t)256 << 20)
da_status delta_attn_prefill_noalloc(const void* q, const void* k, const void* v, void* out,
                                     const int32_t* cu_seqlens, int B, int max_seqlen, int Hq,
                                     int Hkv, int d, int window, int n_sink, int gamma,
                                     void* stream);

/*
 * Workspace bytes delta_attn_prefill[_varlen] uses for these sizes
 * (max_seqlen = N for the fixed-length call).  0 if the sizes are invalid.
 * Short sequences can use more than longer ones, as they split their key axis
 * finer, and very long ones less than shorter ones, as their partial results
 * are held to 8 GiB by fewer chunks.  Given less, down to what key chunks of at
 * least 2560 keys need, a call splits it coarser (which changes the result by
 * rounding), and one given less than that returns DA_ERR_WORKSPACE.  A
 * workspace laid out for a longer max_seqlen with the other sizes the same
 * serves every whole-path call.
 */
size_t da_workspace_bytes(int B, int max_seqlen, int Hq, int Hkv, int d, int gamma);

/*
 * Checks, on the GPU, the device-resident inputs the other calls take on
 * trust, and waits for the answer (this call synchronises `stream`; it is a
 * debugging aid, not for the hot path):
 *   cu_seqlens (when not NULL, B+1 entries): starts at 0, is non-decreasing,
 *     and no length exceeds max_seqlen;
 *   block_ptr / block_idx (when block_ptr is not NULL; the layout of
 *     delta_attn_prefill_blocksparse with nqb = ceil(max_seqlen / block_q),
 *     block_idx holding block_nnz entries): per (sequence, kv head) the
 *     offsets lie in [0, block_nnz] and do not decrease, and every list is
 *     strictly ascending.
 * `result` (device, int32, 4-byte aligned, caller-owned) receives the number
 * of violations.  Returns DA_OK when there are none and DA_ERR_PARAM when
 * there are some; DA_ERR_NULL without result or without anything to check,
 * DA_ERR_SHAPE / DA_ERR_PARAM for bad sizes or block_q, DA_ERR_HIP when a HIP
 * call fails.  The arrays must have the sizes stated above.
 */
da_status da_check_inputs(const int32_t* cu_seqlens, int B, int max_seqlen, int Hkv, int block_q,
                          const int32_t* block_ptr, const int32_t* block_idx, int64_t block_nnz,
                          int32_t* result, void* stream);

/*
 * How the library tiles a problem, as the launch sequence of
 * delta_attn_prefill[_varlen] uses it (block_q = 0), or of the key-block-list
 * calls (block_q = 64, 128 or 256): a host-only query, no HIP call.  A caller
 * counts the work the kernels execute (whole tiles of key_tile keys by
 * rows_per_wave query rows per wavefront) from these numbers instead of
 * restating the plan.  Each full-size attention workgroup holds waves_per_block
 * wavefronts: heads query heads of one GQA group, each with waves_per_block /
 * heads row sub-tiles of rows_per_wave rows.  A launch may take workgroups of
 * half as many wavefronts, and then other heads (see da_launch_workgroups): every
 * wavefront's rows and tiles, and so these counts, are the same.  The strided
 * dense rows split their key axis into key_chunks chunks of chunk_keys keys.
 * Returns DA_ERR_NULL without `plan`, otherwise the status the whole-path
 * call would return for these sizes before touching the device.
 */
typedef struct {
  int fused;            /* 1: the whole-path call takes the fused schedule */
  int sparse_heads;     /* query heads per full-size sparse workgroup in that schedule */
  int rows_heads;       /* query heads per full-size strided-row (and dense causal) workgroup */
  int key_chunks;       /* key chunks of the strided dense rows */
  int chunk_keys;       /* keys per chunk, a multiple of key_tile */
  int key_tile;         /* keys per tile */
  int rows_per_wave;    /* query rows per wavefront */
  int waves_per_block;  /* wavefronts per full-size attention workgroup */
  int sparse_slab_rows; /* rows per query head of a full-size sparse workgroup in that schedule:
                           waves_per_block / sparse_heads * rows_per_wave (a multiple of gamma
                           when fused) */
} da_plan;

da_status da_launch_plan(int B, int max_seqlen, int Hq, int Hkv, int d, int gamma, int block_q,
                         da_plan* plan);

/*
 * The workgroups that the attention launches of these sizes take (host only, no
 * HIP call): wavefronts, waves_per_block of da_launch_plan or half of it, and
 * query heads per workgroup; a workgroup holds waves / heads row sub-tiles per
 * head.  packed: 0 for the fixed-length calls, 1 with cu_seqlens.  mode: the
 * correction (DA_CORR_DELTA for delta_attn_prefill).  block_q: 0, or the block
 * size of the key-block-list calls (window 1 and n_sink 0 then).  With
 * da_workspace_bytes() of workspace or more, where it matters.
 * Returns DA_ERR_NULL without `w`, otherwise the status the whole-path call would
 * return for these sizes before touching the device.
 */
typedef struct {
  int sparse_waves, sparse_heads; /* sparse rows of the whole-path call */
  int rows_waves, rows_heads;     /* its strided dense rows */
  int together;                   /* 1: one launch runs both */
  int base_waves, base_heads;     /* sparse_attn_prefill, blocksparse_attn_prefill */
  int dense_waves, dense_heads;   /* dense_causal_attn_prefill */
} da_workgroups;

da_status da_launch_workgroups(int B, int max_seqlen, int packed, int Hq, int Hkv, int d,
                               int window, int n_sink, int gamma, int block_q, int mode,
                               da_workgroups* w);

/*
 * ---------------------------------------------------------------------------
 * Serving after the prefill: a paged cache, the attention of new tokens over it,
 * and the selection of key blocks.
 *
 * A cache is pages of DA_PAGE_TOKENS tokens (the attention kernels' key tile):
 *   k_pages, v_pages  [P, Hkv, 64, d] bf16, or [layers, P, Hkv, 64, d] for the calls
 *                     that take `layers` (one page id names the page of every layer)
 *   table             int32 [S, M]: page ids of each sequence ("slot"), -1: none
 *   lens              int32 [S]: tokens of each slot, 0: empty
 *   refs              int32 [P]: how many slots hold each page, 0: free
 * all on the device.  Token j of slot s is row j % 64 of page table[s][j / 64].  A
 * slot of L tokens holds exactly its first ceil(L / 64) entries, the others are -1;
 * a cache starts with table -1, lens 0 and refs 0, and the da_pages_* calls keep
 * that.  What a page holds past the last token does not matter (any bits, NaN
 * included) and is left as it is.
 *
 * Requests of one call (n of them, at most DA_PAGES_MAX_REQUESTS) are served as if
 * in order, with results that do not depend on timing.  A request that cannot be
 * served is refused: its result is negative and its slot stays as it was.  The
 * kernels check every slot, length and page id they read against S, M and P, so a
 * wrong one is refused or skipped, never followed.  B sequences of a batch take the
 * slots slots[0 .. B-1] (distinct, where the call writes), or 0 .. B-1 when `slots`
 * is NULL (then B <= S).  cu_seqlens and max_seqlen name the new tokens of each
 * sequence as in the prefill calls; rows of a sequence past max_seqlen are ignored.
 * Other conventions (streams, validation, errors) are those above; integer arrays
 * are 4-byte aligned, `result` of resize and compact 16-byte.  Only bf16, d 64 or
 * 128, any Hq / Hkv.  Launches have at most 2^32 - 1 threads: of 256 per kv head of a page
 * that may be copied or compacted (n * layers * 2 * Hkv), of a query block, of 4 pages to
 * be summarised, of 8 query heads of new tokens, of 16 KB to be appended, and of a token to
 * select pages for (512 there up to max_len 65599, 1024 past 262207); more is DA_ERR_SHAPE.
 */
#define DA_PAGE_TOKENS 64
#define DA_PAGES_MAX_REQUESTS 1024

/*
 * Slot dst[i] becomes a copy of slot src[i] that shares all its pages (no token is
 * copied; da_pages_resize copies a shared page before it is written).
 * result[i] = the length, or -1: a slot out of range, dst[i] not empty or named
 * before in the call, or src[i] the destination of some request of the call.
 */
da_status da_pages_fork(int32_t* table, int32_t* lens, int32_t* refs, int S, int M, int P,
                        const int32_t* src, const int32_t* dst, int n, int32_t* result,
                        void* stream);

/*
 * Slot slots[i] gets new_lens[i] tokens; new_lens NULL: 0 (the slots are freed).  First
 * all pages past new ends are given back.  Then slots that grow, in order, get the
 * lowest free pages; where the page that holds the slot's last token is not full and
 * other slots hold it too, the slot first gets a page of its own with a copy of its
 * tokens (all layers).  Of several slots of the call that share such a page the last
 * keeps it when no other slot does.  New tokens' rows hold whatever the pages held.
 * result [n, 4]: {new length, the page copied from or -1, the page copied to or -1,
 * tokens copied}; a new length of -1: a slot out of range or named before, a length
 * outside [0, 64 M], or too few free pages (then every later slot of the call that
 * would grow is refused as well).
 */
da_status da_pages_resize(void* k_pages, void* v_pages, int layers, int Hkv, int d,
                          int32_t* table, int32_t* lens, int32_t* refs, int S, int M, int P,
                          const int32_t* slots, const int32_t* new_lens, int n, int32_t* result,
                          void* stream);

/*
 * Writes the keys and values k, v [layers, T, Hkv, d] of new tokens as the last ones of
 * their slots, which da_pages_resize has made room for: row i of the m rows of
 * sequence b goes to token lens[slot] - m + i.  k and v lie outside the pages.
 * A slot whose growth was refused has its old tokens there, perhaps in pages that other
 * slots hold too.  da_pages_append_to leaves such slots as they are: it writes the rows of
 * sequence b only where lens[slot] is new_lens[b] (new_lens [B], what da_pages_resize was
 * asked for; NULL: whatever the length).  da_pages_append is for callers that have looked
 * at the results; steps that are enqueued or captured whole take da_pages_append_to.
 * (The attention of such a step is over the slot as it is: its outputs are to be dropped.)
 */
da_status da_pages_append(const void* k, const void* v, int64_t T, void* k_pages, void* v_pages,
                          int layers, int Hkv, int d, const int32_t* table, const int32_t* lens,
                          int S, int M, int P, const int32_t* slots, const int32_t* cu_seqlens,
                          int B, int max_seqlen, void* stream);
da_status da_pages_append_to(const void* k, const void* v, int64_t T, void* k_pages, void* v_pages,
                             int layers, int Hkv, int d, const int32_t* table, const int32_t* lens,
                             int S, int M, int P, const int32_t* slots, const int32_t* cu_seqlens,
                             int B, int max_seqlen, const int32_t* new_lens, void* stream);

/*
 * Keeps some of a slot's tokens from start[i] on: those at start[i] + keep[j], j in
 * [cu_keep[i], cu_keep[i + 1]), ascending, move up to start[i], in every layer, the
 * rest is dropped and pages past the new end are given back (the accepted path of a
 * draft tree, or tokens that stay when others are evicted).
 * result [n, 4]: {tokens kept from start on, ...}, the rest for the call's own use; -1: a
 * slot out of range or named before, a start outside the slot, places that do not
 * ascend or lie outside it, offsets outside [0, n_keep], or a page that would be
 * written while another slot holds it (pages that the call itself gives back are
 * held until its end).
 */
da_status da_pages_compact(void* k_pages, void* v_pages, int layers, int Hkv, int d,
                           int32_t* table, int32_t* lens, int32_t* refs, int S, int M, int P,
                           const int32_t* slots, const int32_t* start, const int32_t* keep,
                           int64_t n_keep, const int32_t* cu_keep, int n, int32_t* result,
                           void* stream);

/*
 * Attention of the last m tokens of each sequence (drafted tokens, whose keys and
 * values are in the cache already: lens counts them).  Row i (token L - m + i, L
 * the slot's length) sees every token before the m new ones, and of the new ones
 *   mask NULL: those up to itself (single tokens, causal chunks);
 *   mask [T, mask_words] of 64-bit words: new token j where bit j % 64 of word j / 64
 *     is set (64 * mask_words >= max_seqlen), itself included or not.
 * A row that sees no token is 0.  Keys and values of all L tokens must be finite.
 * max_len: no slot is longer; tokens past it are ignored.  lse (fp32 [T, Hq], may be
 * NULL): log of the sum of exp(q.k / sqrt d), -inf for a row that sees nothing.  Where more
 * than 32 rows (new tokens times heads) share a kv head its terms are rounded to bf16, by at
 * most 2^-8 of each, as the weights of the values are, and lse is off by up to 2^-8; with
 * up to 32 rows (max_seqlen * Hq / Hkv of them) the terms are fp32.
 * workspace: da_paged_workspace_bytes(B, max_seqlen, Hq, Hkv, d, max_len, 0) bytes (may
 * be 0).  At most 2^31 - 1 pages may be read in all, counted per kv head and workgroup's
 * worth of rows (32 to 256), with every length max_len: else DA_ERR_SHAPE.
 */
da_status tree_attn_paged(const void* q, const void* k_pages, const void* v_pages, void* out,
                          float* lse, const int32_t* table, const int32_t* lens, int S, int M,
                          int P, const int32_t* slots, const int32_t* cu_seqlens, int B,
                          int max_seqlen, int max_len, int Hq, int Hkv, int d,
                          const uint64_t* mask, int mask_words, void* workspace,
                          size_t workspace_bytes, void* stream);

/*
 * Summaries of whole blocks of 64 keys, for the selections below: the mean key as 8-bit
 * codes and one scale.  With S_c the sum of the 64 keys' channel c and A = max_c |S_c|:
 *   code_c = round(127 S_c / A) (ties to even, 0 if A is 0), scale = A / (127 * 64).
 * da_key_summary: of k [T, Hkv, d], into codes int8 [blocks, Hkv, d] and scales fp32
 * [blocks, Hkv]; block j of sequence b has the place floor(base / 64) + b + j, base its
 * first token, and da_key_summary_blocks(T, B) places are enough (places that no
 * whole block has are left as they are).
 * da_page_summary: of pages, into [P, Hkv, d] and [P, Hkv]: the whole pages of each
 * sequence from the page of token first[b] (first NULL: 0) on, up to max_new tokens
 * further.
 */
da_status da_key_summary(const void* k, const int32_t* cu_seqlens, int B, int max_seqlen,
                         int Hkv, int d, void* codes, float* scales, void* stream);
int64_t da_key_summary_blocks(int64_t T, int B);
da_status da_page_summary(const void* k_pages, int Hkv, int d, const int32_t* table,
                          const int32_t* lens, int S, int M, int P, const int32_t* slots,
                          const int32_t* first, int B, int max_new, void* codes, float* scales,
                          void* stream);

/*
 * The blocks that a group of query rows attends to: of its n candidates the last
 * n_recent, the first n_sink and those with the highest scores, top_k in all (n where n
 * <= top_k), ties to the lowest.  With a the largest |q| of the group,
 *   score = scale * max over the group's rows of sum_c round(127 q_c / a) code_c,
 * the sum a whole number and the product rounded once to fp32, so that the choice
 * is the same however it is computed.  n_sink + n_recent <= top_k.
 *
 * da_select_blocks (prefill): a group is the rows of a query block of block_q rows (64,
 * 128 or 256) in the heads of one kv head, its candidates the key tiles before the
 * block.  Writes lists for blocksparse_attn_prefill and
 * delta_attn_prefill_blocksparse: block_ptr [B, Hkv, ceil(max_seqlen / block_q) + 1]
 * and block_idx of da_select_blocks_entries(B, max_seqlen, Hkv, top_k, block_q) entries
 * (-1 where a shorter sequence has no lists; may be 0).  Up to 1,572,864 tokens, and
 * query blocks below 4 GiB.
 *
 * da_select_pages (decode): a group is one token in the heads of one kv head, its
 * candidates the pages before the token's own.  Writes page positions (indices into
 * the slot's table row) pages [T, Hkv, top_k], ascending, -1 behind the last; top_k is at
 * most 2^30, and a group has less than 2^31 channels.
 * workspace: da_select_pages_workspace_bytes() bytes (0 up to max_len 65599); none when
 * max_len / 64 <= top_k.
 */
int64_t da_select_blocks_entries(int B, int max_seqlen, int Hkv, int top_k, int block_q);
da_status da_select_blocks(const void* q, const void* codes, const float* scales,
                           const int32_t* cu_seqlens, int B, int max_seqlen, int Hq, int Hkv,
                           int d, int top_k, int n_sink, int n_recent, int block_q,
                           int32_t* block_ptr, int32_t* block_idx, void* stream);
size_t da_select_pages_workspace_bytes(int B, int max_seqlen, int Hkv, int max_len);
da_status da_select_pages(const void* q, const void* codes, const float* scales,
                          const int32_t* table, const int32_t* lens, int S, int M, int P,
                          const int32_t* slots, const int32_t* cu_seqlens, int B, int max_seqlen,
                          int max_len, int Hq, int Hkv, int d, int top_k, int n_sink,
                          int n_recent, int32_t* pages, void* workspace, size_t workspace_bytes,
                          void* stream);

/*
 * Attention of the last m tokens of each sequence over selected pages: the row of
 * token p in kv head g sees the whole pages pages[row][g][0 .. top_k-1] (positions below
 * p / 64, each at most once; other values are skipped) and its own page up to itself.
 * top_k is at most 2^30.  lse as tree_attn_paged, its rows being the heads of one token;
 * workspace: da_paged_workspace_bytes(B, max_seqlen, Hq, Hkv, d, 1, top_k) bytes.
 */
da_status selected_attn_paged(const void* q, const void* k_pages, const void* v_pages, void* out,
                              float* lse, const int32_t* table, const int32_t* lens, int S, int M,
                              int P, const int32_t* slots, const int32_t* cu_seqlens, int B,
                              int max_seqlen, int Hq, int Hkv, int d, const int32_t* pages,
                              int top_k, void* workspace, size_t workspace_bytes, void* stream);

/*
 * As tree_attn_paged, under the changed scores of dense_attn_prefill_scored (lse is of those).
 * The distance is that of the tokens' places in the cache, which in a tree of drafts is not that
 * along a path: slopes with a mask give DA_ERR_PARAM.
 */
da_status tree_attn_paged_scored(const void* q, const void* k_pages, const void* v_pages,
                                 void* out, float* lse, const int32_t* table, const int32_t* lens,
                                 int S, int M, int P, const int32_t* slots,
                                 const int32_t* cu_seqlens, int B, int max_seqlen, int max_len,
                                 int Hq, int Hkv, int d, const uint64_t* mask, int mask_words,
                                 float cap, const float* slopes, void* workspace,
                                 size_t workspace_bytes, void* stream);

/*
 * ---------------------------------------------------------------------------
 * The cache in 8 bits, half the bytes of a bf16 one: k_pages and v_pages hold e4m3 codes
 * (OCP "fn", a byte each) in the same layout, [P, Hkv, 64, d] or [layers, P, Hkv, 64, d], and
 *   k_scales, v_scales  fp32 [P, Hkv] or [layers, P, Hkv]
 * the power of two that the codes of each page and kv head count in: value = code * scale,
 * which bf16 holds exactly.  An append to a new page makes its scale the least 2^e, e from -110 to
 * 119, for which no value passes 448 * 2^e; later ones raise it to that, and nothing lowers it while the
 * page keeps tokens, not even that its largest ones leave (by a resize down or a compaction).
 * Codes are the nearest, ties to even, and so a value as it is
 * written is off by at most 2^-4 of itself, or 2^-10 of the scale if that is more.  Where the scale of
 * its page has grown since, that holds for values from 2^-6 of the scale on, and smaller ones, which are
 * rounded again, are off by less than 2^-4 of themselves plus 2^-9 of the scale, however often it
 * grew.  Magnitudes past 448 * 2^119 count as that; what is not finite becomes NaN and does not
 * count for the scale.
 * Table, lens, refs, slots and requests are as above: da_pages_fork serves both kinds of cache.
 * The scales are what these calls leave there; a page that holds no token needs none.
 *
 * da_pages8_resize, da_pages8_compact: as da_pages_resize and da_pages_compact.
 * da_pages8_append: as da_pages_append_to (new_lens may be NULL: whatever the length).  New tokens
 *   that begin a page set its scale anew; others raise it where they need to, and the page's
 *   older codes then count in the new one (exactly, as long as they stay above 2^-6 of it, the
 *   range in which e4m3 keeps its 4 bits; below they are rounded to multiples of 2^-9).
 * In a compaction a page that tokens move into gets the largest of the scales that its tokens
 *   had (those of their pages), and their codes count in that likewise.
 * da_pages8_read: the values of cached tokens as rows k, v [layers, T, Hkv, d] of bf16: row i of
 *   the m rows of sequence b is token first[b] + i (first NULL: 0); rows of tokens that the
 *   slot does not hold are left as they are.
 * da_page8_summary: as da_page_summary, of the values.
 * append and read are refused (DA_ERR_SHAPE) where B * layers * 2 times Hkv * ((max_seqlen + 62) / 64 + 1),
 * the pages of a sequence that may be touched, or times ceil(max_seqlen * Hkv * d / 4096), is more than
 * 2^24 - 1, or max_seqlen * Hkv * d / 16 more than 2^31 - 1.
 */
da_status da_pages8_resize(void* k_pages, void* v_pages, float* k_scales, float* v_scales,
                           int layers, int Hkv, int d, int32_t* table, int32_t* lens,
                           int32_t* refs, int S, int M, int P, const int32_t* slots,
                           const int32_t* new_lens, int n, int32_t* result, void* stream);
da_status da_pages8_append(const void* k, const void* v, int64_t T, void* k_pages, void* v_pages,
                           float* k_scales, float* v_scales, int layers, int Hkv, int d,
                           const int32_t* table, const int32_t* lens, int S, int M, int P,
                           const int32_t* slots, const int32_t* cu_seqlens, int B,
                           int max_seqlen, const int32_t* new_lens, void* stream);
da_status da_pages8_compact(void* k_pages, void* v_pages, float* k_scales, float* v_scales,
                            int layers, int Hkv, int d, int32_t* table, int32_t* lens,
                            int32_t* refs, int S, int M, int P, const int32_t* slots,
                            const int32_t* start, const int32_t* keep, int64_t n_keep,
                            const int32_t* cu_keep, int n, int32_t* result, void* stream);
da_status da_pages8_read(void* k, void* v, int64_t T, const void* k_pages, const void* v_pages,
                         const float* k_scales, const float* v_scales, int layers, int Hkv, int d,
                         const int32_t* table, const int32_t* lens, int S, int M, int P,
                         const int32_t* slots, const int32_t* cu_seqlens, int B, int max_seqlen,
                         const int32_t* first, void* stream);
da_status da_page8_summary(const void* k_pages, const float* k_scales, int Hkv, int d,
                           const int32_t* table, const int32_t* lens, int S, int M, int P,
                           const int32_t* slots, const int32_t* first, int B, int max_new,
                           void* codes, float* scales, void* stream);

/*
 * Attention over that cache: as tree_attn_paged_scored (cap 0 and slopes NULL: as
 * tree_attn_paged) and selected_attn_paged of the values.  workspace:
 * da_paged8_workspace_bytes(), with the arguments of da_paged_workspace_bytes().
 */
da_status tree_attn_paged8(const void* q, const void* k_pages, const void* v_pages,
                           const float* k_scales, const float* v_scales, void* out, float* lse,
                           const int32_t* table, const int32_t* lens, int S, int M, int P,
                           const int32_t* slots, const int32_t* cu_seqlens, int B,
                           int max_seqlen, int max_len, int Hq, int Hkv, int d,
                           const uint64_t* mask, int mask_words, float cap, const float* slopes,
                           void* workspace, size_t workspace_bytes, void* stream);
da_status selected_attn_paged8(const void* q, const void* k_pages, const void* v_pages,
                               const float* k_scales, const float* v_scales, void* out,
                               float* lse, const int32_t* table, const int32_t* lens, int S,
                               int M, int P, const int32_t* slots, const int32_t* cu_seqlens,
                               int B, int max_seqlen, int Hq, int Hkv, int d,
                               const int32_t* pages, int top_k, void* workspace,
                               size_t workspace_bytes, void* stream);
size_t da_paged8_workspace_bytes(int B, int max_seqlen, int Hq, int Hkv, int d, int max_len,
                                 int top_k);

/* Workspace of tree_attn_paged[_scored] (top_k 0) and selected_attn_paged (max_len 1); 0 if none is
 * needed or the sizes are invalid.  Its contents on entry do not matter. */
size_t da_paged_workspace_bytes(int B, int max_seqlen, int Hq, int Hkv, int d, int max_len,
                                int top_k);

/* Static, NUL-terminated name of a status code. */
const char* da_status_string(da_status s);

/* The hipError_t of the last DA_ERR_HIP on the calling thread (0 if none). */
int da_last_hip_error(void);

/* DA_ABI_VERSION of the loaded library. */
int da_abi_version(void);

#ifdef __cplusplus
}
#endif

#endif /* DELTA_ATTN_H */

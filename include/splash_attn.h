/*
 * libsplash_attn -- owner-local paged MLA decode attention for MI355X (gfx950).
 *
 * The operation (Sec. 3 "DOP: Computation"; Sec. 3 "Cost"; App. B "Per-Step
 * Cost Model"): an owner GPU holds its N_r = B*q current query rows for all H
 * heads, [N_r, H, d_q] with d_q = d_c + d_r = 576, and the whole latent history
 * of each request it owns, kept in pages.  For every row and every head it
 * attends over the complete causal prefix of that request's history (Sec. 4.1
 * "Handoff") and returns a d_z = d_c = 512 wide output per head.  MLA keeps one
 * head-shared latent row per token (Sec. 1), so one cache row [latent 512 |
 * rope 64] serves as the key of every head, and its first 512 entries serve as
 * the value.  DP-attention and DOP run this same owner-local core (App. B).
 *
 * For request b with history length s_b (s_b counts the current chunk,
 * 1 <= q_chunk <= s_b), chunk row i and head h, output row n = b*q_chunk + i:
 *   visible keys j = 0 .. s_b - q_chunk + i
 *   K_j  = pool row  block_table[b*max_pages_per_seq + j/64]*64 + j%64
 *          (fp8 cache: K_j = e4m3(code) * kv_scales[that row])
 *   z_j  = softmax_scale * <q[n,h,:], K_j>
 *   lse[n,h]   = ln sum_j exp(z_j)                (natural log, scaled logits)
 *   out[n,h,:] = sum_j exp(z_j - lse[n,h]) * K_j[0:512]
 *
 * Entry points: the whole step (splash_mla_attend), its phases (plan,
 * attend_units, combine_splits, run), the standalone LSE merge
 * (splash_mla_combine), and around the same core: one position shard of the
 * histories (splash_mla_attend_shard), attention over listed positions only
 * (splash_mla_attend_topk), and the DOP regroup of query and output rows
 * (splash_dop_*).  Beside it, each in a section of its own below: the serving step
 * around grouped-query attention, and the latent-attention layer around this cache
 * (the rows' way in and out, the projections, a prompt's expanded attention).
 *
 * Conventions for every entry point:
 *  - All tensor pointers are DEVICE pointers owned by the caller; the library
 *    never allocates or frees device memory in these calls and keeps no
 *    pointer after it returns.  `stream` is a hipStream_t (NULL: the null
 *    stream); all work is enqueued on it with no host synchronisation (except
 *    under SPLASH_FLAG_DEBUG_CHECK), so the calls can be captured in a graph.
 *  - Return value: SPLASH_OK or a negative status; no C++ exception crosses
 *    the boundary.  splash_status_string() names a status and
 *    splash_last_error() holds the last detailed message of the calling
 *    thread.
 *  - Device data is trusted on the fast path: seq_lens[b] < q_chunk or a
 *    block-table entry outside [0, num_pages) is undefined behaviour unless
 *    SPLASH_FLAG_DEBUG_CHECK is set, which validates them first.
 *  - Unused block-table slots (past ceil(s_b/64)) and pool rows past a
 *    history's end are never used in the result.
 */
#ifndef SPLASH_ATTN_H
#define SPLASH_ATTN_H

#include <stddef.h>
#include <stdint.h>

#ifdef __cplusplus
extern "C" {
#endif

/* ---- status codes -------------------------------------------------------- */
#define SPLASH_OK                        0
#define SPLASH_ERR_INVALID_ARGUMENT     (-1) /* null pointer, q_chunk<1, dims != 576/512, bad scale, bad device data */
#define SPLASH_ERR_UNSUPPORTED          (-2) /* H not in {16,32,...,128}, page size != 64, unknown kv dtype */
#define SPLASH_ERR_MISALIGNED           (-3) /* a tensor base pointer not 16-byte aligned */
#define SPLASH_ERR_WORKSPACE_TOO_SMALL  (-4)
#define SPLASH_ERR_HIP                  (-5) /* a HIP call or launch failed; see splash_last_error() */

/* ---- cache formats --------------------------------------------------------- */
#define SPLASH_KV_BF16      0  /* pool: [num_pages, 64, 576] bf16 */
#define SPLASH_KV_FP8_E4M3  1  /* pool: [num_pages, 64, 576] OCP E4M3 ("fn") bytes + kv_scales [num_pages, 64] fp32 */
/* Latent-row cache (App. B, theoretical scenarios for DCU and H200,
 * residency assumptions: FP8 latent with its scales and BF16 RoPE; the
 * paper fixes neither the split nor the scale granularity).  Pool:
 * [num_pages, 64, 656] bytes; a row is 512 OCP E4M3 latent codes, four
 * little-endian fp32 scales (scale t covers latent columns [128t, 128t+128))
 * and the 64 RoPE values as bf16: K[d] = e4m3(code[d]) * scale[d / 128] for
 * d < 512, K[512 + r] = rope[r].  Scales must be positive normal powers
 * of two no larger than 2^63 (the conversion uses only a scale's exponent,
 * and the weights take it as an exponent step); rows no history reaches may
 * hold anything.  Under SPLASH_FLAG_DEBUG_CHECK every entry point rejects a
 * reached (top-k: listed) row whose scale is not.  kv_scales is ignored.
 * Every attend entry point (whole histories, shards, top-k) and the gather
 * take it. */
#define SPLASH_KV_FP8_LATENT 2

/* ---- flags ------------------------------------------------------------------ */
#define SPLASH_FLAG_DEBUG_CHECK  1u  /* validate seq_lens / block table on the device first; synchronises `stream` */
#define SPLASH_FLAG_FORCE_SPLIT  2u  /* split every history into work units of `split_pages` pages */
/* fp8 caches (App. C: FP8 E4M3 KV): QK with K converted exactly to bf16 and
 * the bf16 MFMA's fp32 sums, instead of the default: K's own codes on the fp8
 * matrix pipe against the query split exactly into two E4M3 terms, which is
 * faster (16 requests x 8 rows of 8,192 to 32,768 positions: attend 570 against
 * 644 us, latent rows 667 against 749).  The fp8 pipe aligns the products of
 * up to 32 dims to the largest of them and drops what lies below 2^-13 of it.
 * Measured over rows of N(0, 1) values, a sum of 576 products is off by up to
 * 6e-6 of sum |q_i k_i| (7.5e-7 on average), a score by that times
 * softmax_scale; dims whose products stand far above the others' cost more, up
 * to 2^-13 of them for each other product beside them.  No effect on the bf16
 * cache. */
#define SPLASH_FLAG_EXACT_QK     4u

#define SPLASH_DIM_QK     576
#define SPLASH_DIM_V      512
#define SPLASH_PAGE_SIZE  64
#define SPLASH_MAX_HEADS  128

/* Description of one call.  Sizes are element counts. */
typedef struct splash_mla_desc {
    int32_t batch;              /* B: requests owned by this GPU (0: idle owner, every call is a no-op) */
    int32_t num_heads;          /* H: query heads, a multiple of 16 in [16, 128] */
    int32_t dim_qk;             /* must be 576 = 512 latent + 64 rope */
    int32_t dim_v;              /* must be 512 */
    int32_t page_size;          /* must be 64 */
    int32_t max_pages_per_seq;  /* row stride of block_table (>= ceil(max s_b / 64)) */
    int32_t num_pages;          /* pages in the pool */
    int32_t kv_dtype;           /* SPLASH_KV_* */
    const float* kv_scales;     /* device [num_pages, 64] fp32 per-token scales; SPLASH_KV_FP8_E4M3 only, else ignored */
    float softmax_scale;        /* multiplies <q, k>; finite and > 0 (1/sqrt(192) for DeepSeek-V3 dims) */
    uint32_t flags;             /* SPLASH_FLAG_* */
    int32_t split_pages;        /* with SPLASH_FLAG_FORCE_SPLIT: pages per work unit, >= 1 */
} splash_mla_desc;

/*
 * Workspace.  One caller-allocated device buffer carries the plan (work list,
 * split offsets) and the partial results of split histories.
 * `max_partials` bounds how many partial results (one per work unit of a
 * split history, room for H x 512 fp32 each) the planner may use; <= 0 selects
 * SPLASH_DEFAULT_MAX_PARTIALS.  The planner never exceeds the capacity that
 * the passed ws_bytes provides: with too little room it splits less.
 * Layout (byte offsets from splash_mla_workspace_offsets, 256-byte aligned):
 *   [0] header int32[1152]: [1] number of work units, [2] partial slots
 *       used, [3] pages per unit chosen (0 for a fold plan), [4] debug
 *       status, [6] number of split tiles, [7] total pages, [8] most parts of
 *       a split tile, [9] workers of a fold plan (0: the queue, ordered
 *       longest unit first and dealt to the workers in a snake), [10] the fold
 *       plan's cap; from [64] the fold plan's first unit of each worker
 *       (workers + 1 entries).  [0] and [5] are written as 0 and unused.
 *   [1] work units int32[max_units][4] = {tile, first page, end page, slot},
 *       tile = b*q_chunk + i, slot = partial index or -1 (unit writes out/lse)
 *   [2] split offsets int32[B*q_chunk + 1] (partial slots of tile t are
 *       [off[t], off[t+1]); empty when the tile is a single unit)
 *   [3] split tiles int32[B*q_chunk] (the tiles with partials, ascending)
 *   [4] partial lse fp32 [max_partials, H]
 *   [5] partial out: room for fp32 [max_partials, H, 512]; the library keeps
 *       them as fp16 [max_partials, H, 512] (the first half of the region),
 *       each (slot, head) 128-column quarter q multiplied by 2^-e, with e
 *       byte q of uint32 [max_partials, H] right after them (e = 0 unless
 *       the quarter's largest magnitude reaches 2^15; then every stored
 *       value stays below 2^15).  Internal: only splash_mla_combine_splits
 *       reads them.
 */
#define SPLASH_DEFAULT_MAX_PARTIALS 1024
size_t splash_mla_workspace_size(int32_t batch, int32_t q_chunk, int32_t num_heads,
                                 int32_t max_partials);
/* Writes the six byte offsets above into offsets[6]; returns the total size. */
size_t splash_mla_workspace_offsets(int32_t batch, int32_t q_chunk, int32_t num_heads,
                                    int32_t max_partials, size_t* offsets);

/*
 * splash_mla_attend: the whole step -- plan, attend, combine -- on `stream`.
 *   q            bf16 [B*q_chunk, H, 576], row n = b*q_chunk + i, each head's 576
 *                entries packed [no-position 512 | rotary 64] (App. E)
 *   kv_pages     pool, see SPLASH_KV_*
 *   block_table  int32 [B, max_pages_per_seq]; logical page k of request b is
 *                physical page block_table[b*max_pages_per_seq + k]
 *   seq_lens     int32 [B], history length including the current chunk
 *   q_chunk      query rows per request (1: decode), 1 <= q_chunk <= seq_lens[b]
 *   out          bf16 [B*q_chunk, H, 512] (round to nearest even)
 *   lse          fp32 [B*q_chunk, H] natural-log LSE of the scaled logits; may be NULL
 * Results are deterministic: the same inputs give the same bits, independent
 * of page placement in the pool and of how units land on compute units.
 */
int splash_mla_attend(const void* q, const void* kv_pages, const int32_t* block_table,
                      const int32_t* seq_lens, int32_t q_chunk, void* out, float* lse,
                      const splash_mla_desc* desc, void* workspace, size_t ws_bytes,
                      void* stream);

/*
 * splash_mla_attend_noalloc: splash_mla_attend for callers that cannot
 * allocate device memory (code under graph capture, tight serving loops,
 * harnesses that forbid allocation): the same step on a workspace the
 * library owns, so the caller passes inputs and outputs only.
 *   The workspace is a device array of SPLASH_NOALLOC_SCRATCH_BYTES inside
 *   the library, one per GPU the library runs on, held until the process
 *   ends; its address is looked up once per device.  The call allocates
 *   nothing and enqueues only kernels on `stream`.
 *   Every call on one GPU shares that GPU's array: calls that overlap on one
 *   GPU (other streams, other threads) race and give undefined results;
 *   calls in one stream order are fine.  Nothing in the array needs to
 *   start at zero: the plan writes everything the later kernels read.
 *   Arguments as for splash_mla_attend.  Errors: as splash_mla_attend, plus
 *   SPLASH_ERR_WORKSPACE_TOO_SMALL when the batch's minimum workspace (its
 *   plan, plus the partials that histories longer than 1024 pages force)
 *   exceeds the array; with less room than splash_mla_attend's default
 *   workspace the planner splits less.  SPLASH_FLAG_DEBUG_CHECK is refused
 *   (SPLASH_ERR_UNSUPPORTED): its check reads a result back to the host.
 */
#define SPLASH_NOALLOC_SCRATCH_BYTES ((size_t)128 << 20)
int splash_mla_attend_noalloc(const void* q, const void* kv_pages, const int32_t* block_table,
                              const int32_t* seq_lens, int32_t q_chunk, void* out, float* lse,
                              const splash_mla_desc* desc, void* stream);

/*
 * splash_mla_plan + splash_mla_run: the same step in two halves, so that a
 * plan made once per step (it depends only on seq_lens, q_chunk and desc) can
 * serve every layer.  splash_mla_run must see the workspace of a plan made
 * with the same seq_lens, q_chunk and desc, earlier in stream order.
 * The split heuristic (a cost-model argmin over candidate unit sizes, in the
 * spirit of Sec. 4.2's calibrated argmin) balances pages over the compute
 * units and splits a history only where that shortens the step.
 */
int splash_mla_plan(const int32_t* seq_lens, int32_t q_chunk, const splash_mla_desc* desc,
                    void* workspace, size_t ws_bytes, void* stream);
int splash_mla_run(const void* q, const void* kv_pages, const int32_t* block_table,
                   const int32_t* seq_lens, int32_t q_chunk, void* out, float* lse,
                   const splash_mla_desc* desc, void* workspace, size_t ws_bytes,
                   void* stream);

/*
 * splash_mla_attend_units + splash_mla_combine_splits: splash_mla_run in its
 * two launches.  attend_units processes every work unit of the plan: a tile
 * (query row with all heads) that is one unit writes its out/lse rows
 * directly; the units of a split tile write partials (fp16 with a
 * power-of-two scale, see the workspace layout) into the workspace.  combine_splits merges those partials into out/lse (its
 * arguments must match the attend_units call).  Same argument rules as
 * splash_mla_run.
 */
int splash_mla_attend_units(const void* q, const void* kv_pages, const int32_t* block_table,
                            const int32_t* seq_lens, int32_t q_chunk, void* out, float* lse,
                            const splash_mla_desc* desc, void* workspace, size_t ws_bytes,
                            void* stream);
int splash_mla_combine_splits(int32_t q_chunk, void* out, float* lse, const splash_mla_desc* desc,
                              void* workspace, size_t ws_bytes, void* stream);

/*
 * splash_mla_attend_topk: top-k (sparse) attention, the attention the paper's
 * sparse backend runs (each row attends a selected subset of its history,
 * chosen by an indexer that is not part of this library).  Row n =
 * b*q_chunk + i attends the token positions topk_idx[n][0 .. topk_count[n])
 * of request b's history, with the logits, values, softmax and LSE of
 * splash_mla_attend restricted to those keys:
 *   topk_idx    device int32 [B*q_chunk, topk]: positions, each in the row's
 *               visible prefix [0, seq_lens[b] - q_chunk + i]; entries past
 *               the count are not read.  A position listed twice counts twice.
 *   topk_count  device int32 [B*q_chunk], 0 <= count <= topk; a row with an
 *               empty list gets out = 0, lse = -inf.
 * Only the block-table entries of listed positions are read.  Lists longer
 * than 2048 entries are split into partials (the workspace needs room for
 * B*q_chunk*ceil(ceil(topk/64)/32) of them, else WORKSPACE_TOO_SMALL);
 * SPLASH_FLAG_FORCE_SPLIT takes split_pages <= 32 (groups of 64 entries).
 * SPLASH_FLAG_DEBUG_CHECK validates counts, positions and their pages.  Other
 * arguments as for splash_mla_attend.
 */
int splash_mla_attend_topk(const void* q, const void* kv_pages, const int32_t* block_table,
                           const int32_t* seq_lens, int32_t q_chunk, const int32_t* topk_idx,
                           const int32_t* topk_count, int32_t topk, void* out, float* lse,
                           const splash_mla_desc* desc, void* workspace, size_t ws_bytes,
                           void* stream);

/*
 * DOP regroup (Sec. 3 "DOP: Computation"; App. E, DOP transfer).  With
 * sharded projections, rank t of T holds all N current query rows for its
 * heads_local = H/T heads (global heads [t*H/T, (t+1)*H/T)); the owner of a
 * request needs that request's rows for all H heads.  A variable-size
 * all-to-all (not part of this library; its split sizes are the per-owner
 * row counts) moves one contiguous block between every pair.  These calls
 * build and take apart those blocks; rows keep their identity, heads their
 * order, and each packed query row carries the no-position part followed by
 * the rotary part.  All tensors are bf16, contiguous, 16-byte aligned
 * device buffers; row_order is a device int32 [num_rows] permutation of the
 * rows, grouped by owner (owner 0's rows first); it is not validated.
 *
 * splash_dop_pack_q (rank side, before attention):
 *   q_nope [num_rows, heads_local, 512], q_rope [num_rows, heads_local, 64]
 *   -> send [num_rows, heads_local, 576], send[k] = q_nope[row_order[k]] | q_rope[row_order[k]]
 * splash_dop_unpack_q (owner side): recv [num_ranks, owner_rows, heads_local,
 *   576] (rank t's block t) -> q_owner [owner_rows, num_ranks*heads_local, 576],
 *   q_owner[i][t*heads_local + h] = recv[t][i][h]
 * splash_dop_pack_out (owner side, after attention): out_owner [owner_rows,
 *   num_ranks*heads_local, 512] -> send [num_ranks, owner_rows, heads_local,
 *   512], send[t][i][h] = out_owner[i][t*heads_local + h]
 * splash_dop_unpack_out (rank side): recv [num_rows, heads_local, 512] in
 *   row_order -> out [num_rows, heads_local, 512], out[row_order[k]] = recv[k]
 *
 * Zero rows is a no-op (an owner with no rows still takes part in the
 * exchange).  Errors: INVALID_ARGUMENT for negative or zero sizes or NULL
 * buffers, MISALIGNED, UNSUPPORTED when rows * H * 72 reaches 2^31.
 */
int splash_dop_pack_q(const void* q_nope, const void* q_rope, const int32_t* row_order,
                      int32_t num_rows, int32_t heads_local, void* send, void* stream);
int splash_dop_unpack_q(const void* recv, int32_t num_ranks, int32_t owner_rows,
                        int32_t heads_local, void* q_owner, void* stream);
int splash_dop_pack_out(const void* out_owner, int32_t num_ranks, int32_t owner_rows,
                        int32_t heads_local, void* send, void* stream);
int splash_dop_unpack_out(const void* recv, const int32_t* row_order, int32_t num_rows,
                          int32_t heads_local, void* out, void* stream);

/*
 * splash_mla_attend_shard: the partial result of one position shard (App. E,
 * position-sharded CP: each rank holds a slice of a request's token history,
 * and the ranks' partial results are merged by their log-sum-exp).  For every
 * query row n = b*q_chunk + i and head h it attends over the keys of request
 * b in [key_begin[b], key_end[b]) that row n sees (j <= seq_lens[b] - q_chunk
 * + i), and writes the normalised fp32 output and its natural-log LSE into
 * slot b*num_shards + shard:
 *   part_out  fp32 [B*num_shards, q_chunk, H, 512]: rows of request b, shard k
 *             at slot b*num_shards + k (this call writes its shard's slots)
 *   part_lse  fp32 [B*num_shards, q_chunk, H]
 * A row that sees no key of the shard gets out = 0 and lse = -inf.  After the
 * num_shards calls (any order, same workspace reused), splash_mla_combine
 * with split_indptr[b] = b*num_shards merges them into the result over the
 * union of the shards: with shards that tile [0, seq_len) it equals
 * splash_mla_attend.
 *   key_begin, key_end  device int32 [B]; key_begin[b] a multiple of 64 (the
 *             shard starts on a page), 0 <= key_begin[b] <= key_end[b]; only
 *             the block-table entries of the shard's pages are read.
 * The workspace needs a partial slot per query row (max_partials >= B *
 * q_chunk, else SPLASH_ERR_WORKSPACE_TOO_SMALL).  Other arguments as for
 * splash_mla_attend; SPLASH_FLAG_FORCE_SPLIT is rejected (UNSUPPORTED), and
 * SPLASH_FLAG_DEBUG_CHECK also checks the key ranges.
 */
int splash_mla_attend_shard(const void* q, const void* kv_pages, const int32_t* block_table,
                            const int32_t* seq_lens, int32_t q_chunk, const int32_t* key_begin,
                            const int32_t* key_end, int32_t num_shards, int32_t shard, float* part_out,
                            float* part_lse, const splash_mla_desc* desc, void* workspace,
                            size_t ws_bytes, void* stream);

/*
 * splash_mla_combine: merge partial attention results over disjoint key sets
 * into the result over their union (the merge a position-sharded history
 * needs, App. E).  For request b, partial slots s in
 * [split_indptr[b], split_indptr[b+1]) each hold rows i < q_chunk:
 *   partials     fp32 [S_tot, q_chunk, H, 512], normalised outputs
 *   partial_lse  fp32 [S_tot, q_chunk, H]; -inf marks a part with no key
 *   L = ln sum_s exp(lse_s);  out = sum_s exp(lse_s - L) * partial_s
 *   out          bf16 [B*q_chunk, H, 512]; out_lse fp32 [B*q_chunk, H] or NULL
 * A request with no partial, or whose parts are all -inf, gets out = 0 and
 * lse = -inf.  split_indptr is a device int32 [B+1] array.
 */
int splash_mla_combine(const float* partials, const float* partial_lse,
                       const int32_t* split_indptr, int32_t batch, int32_t q_chunk,
                       int32_t num_heads, void* out, float* out_lse, void* stream);

/*
 * splash_mla_debug_gather (tests): copy every history, token by token, into
 * a dense buffer through the same page-address code the attention kernel
 * uses.  dense_out holds sum_b seq_lens[b] rows of the pool's row bytes
 * (1152 for bf16, 576 for fp8, 656 for latent rows), request after request.
 */
int splash_mla_debug_gather(const void* kv_pages, const int32_t* block_table,
                            const int32_t* seq_lens, const splash_mla_desc* desc,
                            void* dense_out, void* stream);

/*
 * splash_mla_plan_host: the planner run on the CPU over HOST seq_lens, for
 * tests and for callers that want to inspect a plan.  It computes exactly
 * what splash_mla_plan computes on the device for `num_workers` compute units
 * and `max_partials` partial slots.  units_out: int32 [max_units][4];
 * indptr_out: int32 [B*q_chunk + 1]; stats_out: int32[7] = {units, partial
 * slots used, pages per unit (0 for a fold plan), total pages, workers of a
 * fold plan (0: the queue, dealt to the workers in a snake), the pages a fold plan
 * lets a long history keep (the rest goes to a second worker), the most
 * parts of any split tile}; worker_start_out (may be NULL): int32
 * [num_workers + 1], for a fold plan the first unit of each worker (worker g
 * runs units [w[g], w[g+1])), untouched otherwise.  Returns SPLASH_OK, or
 * SPLASH_ERR_WORKSPACE_TOO_SMALL when max_units is too small.
 */
int splash_mla_plan_host(const int32_t* seq_lens_host, int32_t q_chunk,
                         const splash_mla_desc* desc, int32_t num_workers,
                         int32_t max_partials, int32_t* units_out, int32_t max_units,
                         int32_t* indptr_out, int32_t* stats_out, int32_t* worker_start_out);

/*
 * ---- the serving step around grouped-query attention -----------------------
 *
 * For models with a few KV heads instead of one shared latent row: num_heads
 * query heads share num_kv_heads K and V heads (query head h reads KV head
 * h / (num_heads / num_kv_heads)), and K and V are kept in 8 bits.  One step:
 *   splash_step_tables   the new tokens' pages, slots and positions
 *   splash_rope          rotary positions on the step's queries and keys
 *   splash_gqa_append    the new K and V rows into the cache
 *   splash_gqa_attend    attention of the step's query rows
 * splash_step_tables and splash_rope serve the MLA calls above as well: the
 * block table and slots are the same, and the rotary part of a packed query
 * row or a latent row is a strided view.  The MLA calls trust the table: after a
 * step that found no page for a token (taken_out[1] > 0) the requests that went
 * short are not theirs to attend.
 *
 * These four calls stay inside their buffers whatever the device data holds:
 * lengths are clamped to the block-table row, a block-table entry or slot
 * outside the pool is skipped (that is how a page that splash_step_tables
 * could not get is passed on), and a row that sees no key gets out = 0 and
 * lse = -inf.  All of them can be captured in a graph.
 *
 * Cache: a block is the 64 tokens of one page for one KV head,
 *   k_pages, v_pages    [num_pages, num_kv_heads, 64, head_dim] codes, one byte each
 *   k_scales, v_scales  fp32 [num_pages, num_kv_heads], finite and > 0:
 *                       value = code * scale of its block
 * A block's scale as splash_gqa_append writes it is a power of two, so that a
 * growing block is brought to a new scale by shifting its codes' exponents (E4M3
 * codes that reach the subnormals, and INT8 codes, are rounded again).
 */
#define SPLASH_GQA_E4M3 0   /* codes: OCP E4M3 ("fn") bytes */
#define SPLASH_GQA_INT8 1   /* codes: signed bytes */

typedef struct splash_gqa_desc {
    int32_t batch;              /* B: requests (0: every call is a no-op) */
    int32_t num_heads;          /* query heads, a multiple of num_kv_heads, at most 1024 */
    int32_t num_kv_heads;       /* 1 .. 128 */
    int32_t head_dim;           /* 64, 128 or 256 */
    int32_t page_size;          /* must be 64 */
    int32_t max_pages_per_seq;  /* row stride of block_table, 1 .. 2^25 - 1 */
    int32_t num_pages;          /* pages in the pool, 1 .. 2^25 */
    int32_t code_type;          /* SPLASH_GQA_* */
    float softmax_scale;        /* multiplies <q, k>; finite and > 0 */
} splash_gqa_desc;

/*
 * splash_step_tables: block table, slots and positions of a step's new tokens
 * from the requests' lengths.  Request b's history has s_b = seq_lens[b]
 * tokens after the step, the last n_b of them new (n_b = new_lens[b], or
 * q_chunk where new_lens is NULL); 0 <= s_b <= 64 * max_pages_per_seq and
 * 0 <= n_b <= s_b (values outside are clamped).  Pages ceil((s_b - n_b) / 64)
 * .. ceil(s_b / 64) - 1 of the request are new and are taken from the free
 * list in the order of the requests:
 *   free_pages   int32 [num_free] pages that no request holds
 *   taken_in     int32 [2]; [0] entries of the list taken by earlier steps
 *                (clamped to [0, num_free]), [1] is not read
 *   taken_out    int32 [2]; [0] entries taken after this step, [1] new pages
 *                that the list had no entry for (0: every page was found).
 *                Must not overlap taken_in; the next step's taken_in.
 *   block_table  int32 [B, max_pages_per_seq]; the new pages' entries are
 *                written (-1 where the list has run out), all others are left
 *                as they are
 *   new_indptr   int32 [B+1]: request b's new tokens are rows
 *                new_indptr[b] .. new_indptr[b+1] - 1 of the step
 *   slots        int32 [max_tokens]: 64 * page + place in the page of every
 *                row's token, -1 where its block-table entry is outside
 *                [0, num_pages) and on the rows behind the last new token
 *   positions    int32 [max_tokens]: the token's place in its history (0 on
 *                the rows behind)
 *   requests     int32 [max_tokens]: the row's request (-1 on the rows behind)
 * Rows past max_tokens are not written; new_indptr counts them.  One launch.
 * Errors: INVALID_ARGUMENT (NULL buffer, batch or max_tokens or num_free < 0,
 * q_chunk < 0, max_pages_per_seq < 1, num_pages < 1, taken_out over taken_in),
 * MISALIGNED (a buffer not 4-byte aligned), UNSUPPORTED (batch > 8192,
 * num_pages > 2^25, 64 * max_pages_per_seq * batch past 2^31 - 1).
 */
int splash_step_tables(const int32_t* seq_lens, const int32_t* new_lens, int32_t q_chunk, int32_t batch,
                       const int32_t* free_pages, int32_t num_free, const int32_t* taken_in, int32_t* taken_out,
                       int32_t* block_table, int32_t max_pages_per_seq, int32_t num_pages, int32_t max_tokens,
                       int32_t* new_indptr, int32_t* slots, int32_t* positions, int32_t* requests, void* stream);

/*
 * splash_rope: rotary positions with one to four axes (text: one; video and
 * images: time, height, width).  Pair j of a row (j < rot_dim / 2) turns by
 *   angle = positions[axis_j][n] * inv_freq[j]
 *   (a, b) -> scale * (a cos - b sin, b cos + a sin)
 * with (a, b) = (x[j], x[j + rot_dim / 2]), or (x[2j], x[2j + 1]) where
 * `interleaved`.  The angle is formed and reduced to a turn's fraction in 64
 * bits (so far positions lose nothing), sine, cosine and products are fp32,
 * rounded once to bf16.  Up to two tensors (a step's queries and keys) turn in one launch.
 *   view   x, y: bf16, element d of head h of token n at
 *          n * token_stride + h * head_stride + d (strides in elements, of x
 *          and y each); y == x with the same strides rotates in place, else
 *          the two must not overlap, and no y another view.  Rows of one y that
 *          overlap are refused (of one x they may, where y is elsewhere), and so
 *          is a y that begins where the other view's x or y does.  Only rot_dim
 *          elements of a head are read and written.
 *   positions  int32, axis a's position of token n at [a * position_stride + n];
 *          where num_axes > 1, position_stride >= num_tokens, or 0 (text: every
 *          axis has the same positions)
 * inv_freq and pair_axis are HOST arrays of rot_dim / 2, read during the call.
 * Errors: INVALID_ARGUMENT (NULL, negative counts or strides, num_axes outside
 * 1 .. 4, an axis outside [0, num_axes), an inv_freq or scale that is not
 * finite, overlapping rows or views as above), UNSUPPORTED (rot_dim odd or outside 2 .. 256, more than 65536
 * heads or 2^25 tokens), MISALIGNED (x or y not 2-byte, positions not 4-byte aligned).
 */
typedef struct splash_rope_view {
    const void* x;
    void* y;
    int64_t x_token_stride, x_head_stride;
    int64_t y_token_stride, y_head_stride;
    int32_t num_heads;
} splash_rope_view;

typedef struct splash_rope_desc {
    int32_t rot_dim;            /* even, 2 .. 256 */
    int32_t interleaved;        /* 0: pairs (j, j + rot_dim / 2); 1: pairs (2j, 2j + 1) */
    int32_t num_axes;           /* 1 .. 4 */
    float scale;                /* multiplies the turned pair (1: none) */
    const double* inv_freq;     /* host [rot_dim / 2], radians per position */
    const uint8_t* pair_axis;   /* host [rot_dim / 2], the axis of each pair; NULL: axis 0 */
} splash_rope_desc;

int splash_rope(const splash_rope_view* views, int32_t num_views, const int32_t* positions, int64_t position_stride,
                int32_t num_tokens, const splash_rope_desc* desc, void* stream);

/*
 * splash_gqa_append: new K and V rows into their blocks.
 *   k_new, v_new  bf16, element d of KV head h of row t at
 *                 t * token_stride + h * head_stride + d (elements, one pair of
 *                 strides for both: views of a fused projection's rows)
 *   slots         int32 [num_tokens]; row t goes to place slots[t] % 64 of page
 *                 slots[t] / 64; a slot outside [0, 64 * num_pages) is skipped.
 *                 Slots are distinct, and the rows of one page stand next to
 *                 each other in the list, with no skipped slot between them
 *                 (as splash_step_tables writes them): two runs of one page race.
 * With TOP = 448 (E4M3) or 127 (INT8), for every block that gets rows:
 *   e   = the least e >= -126 with |x| <= TOP * 2^e for every finite new x;
 *         not below the block's own exponent, unless a new row takes place 0,
 *         which starts the block anew
 *   rows before the last new place that are not new: code -> code * old scale
 *         * 2^-e, rounded to nearest even (only where the scale grows)
 *   new rows: code = x * 2^-e, rounded to nearest even; infinities take the
 *         largest code of their sign; NaN is E4M3's NaN and INT8's 0
 *   scale = 2^e
 * desc->batch, the step's requests, decides only how the work is laid out (8
 * slots a request and more, skipped ones among them, are taken for prompts).
 * A block that is continued must have a power-of-two scale (as this call
 * writes it; of another, its exponent alone is used).  Rows of a block past its
 * last new place are not written.
 * Errors: INVALID_ARGUMENT (desc, NULL, num_tokens < 0, negative stride),
 * UNSUPPORTED (desc, num_tokens * num_kv_heads past 2^25), MISALIGNED (pages not 16-byte, scales or slots not 4-byte,
 * k_new and v_new not 16-byte aligned, strides not multiples of 8 elements).
 */
int splash_gqa_append(const void* k_new, const void* v_new, int64_t token_stride, int64_t head_stride,
                      const int32_t* slots, int32_t num_tokens, void* k_pages, void* v_pages, float* k_scales,
                      float* v_scales, const splash_gqa_desc* desc, void* stream);

/*
 * splash_gqa_attend: attention of q_chunk causal query rows per request.  Row
 * n = b*q_chunk + i sees keys j = 0 .. s_b - q_chunk + i (none where that is
 * negative: out = 0, lse = -inf), K_j and V_j from place j % 64 of page
 * block_table[b*max_pages_per_seq + j/64]:
 *   z_j        = softmax_scale * <q[n,h,:], K_j>
 *   lse[n,h]   = ln sum_j exp(z_j)
 *   out[n,h,:] = sum_j exp(z_j - lse[n,h]) * V_j
 *   q          bf16 [B*q_chunk, num_heads, head_dim]
 *   seq_lens   int32 [B], history lengths including the chunk
 *   out        bf16 [B*q_chunk, num_heads, head_dim] (round to nearest even)
 *   lse        fp32 [B*q_chunk, num_heads]; may be NULL
 *   workspace  splash_gqa_workspace_size(desc, q_chunk) bytes, 16-byte aligned;
 *              what it holds is of one call, and calls that may overlap (other
 *              streams, graphs replayed side by side) take one each
 * Codes are converted exactly (K to bf16, V to fp16), products are summed in
 * fp32.  A weight meets V in fp16 and its sum does not: to 2^-22 where
 * q_chunk * num_heads / num_kv_heads is at most 16, else to 2^-11, or 2^-40 of
 * the row's largest weight in the same page where that is more.  A page whose
 * weights are down to 2^-117 of the row's largest keeps its part in out, however
 * far apart the scales of V lie.
 * Codes of places that no row of the request sees are not used, NaN codes
 * among them, and a place that some rows of a chunk do not see does not touch
 * those rows; NaN reaches the rows that see it (out and lse).  Values of V up
 * to 2^80 cannot overflow the sums, whatever the lengths.  Deterministic: the
 * same inputs give the same bits, wherever the pages lie.
 * Errors: INVALID_ARGUMENT (desc, NULL, q_chunk < 1), UNSUPPORTED (desc;
 * a batch whose pages times heads pass 2^30), MISALIGNED (q, out, pages or
 * workspace not 16-byte, other arrays not 4-byte aligned),
 * WORKSPACE_TOO_SMALL.
 */
size_t splash_gqa_workspace_size(const splash_gqa_desc* desc, int32_t q_chunk);
int splash_gqa_attend(const void* q, const void* k_pages, const void* v_pages, const float* k_scales,
                      const float* v_scales, const int32_t* block_table, const int32_t* seq_lens, int32_t q_chunk,
                      void* out, float* lse, const splash_gqa_desc* desc, void* workspace, size_t ws_bytes,
                      void* stream);

/*
 * ---- the latent-attention layer around the cache ----------------------------
 *
 * What a layer of a model with one shared latent row a token runs around
 * splash_mla_attend (App. E: no-position and rotary parts, up-projections), and
 * in its place for a prompt.  A head's key is [no-position 128 | rotary 64],
 * its value 128 wide; W_UK[h] and W_UV[h], 128 x 512 each, take the latent to
 * them.
 *   decode   splash_mla_absorb_q   q W_UK and the turned rotary part: packed rows
 *            splash_mla_append     the new tokens' rows into the cache
 *            splash_mla_attend     (or its shards, or listed positions)
 *            splash_mla_expand_out latent outputs through W_UV
 *   prompt   splash_mla_append, splash_mla_gather (histories back as dense rows),
 *            the caller's product with the up-projections, splash_rope on the
 *            queries, splash_mla_prefill
 * Both give the same attention: <q W_UK | q_r, [c | k_r]> = <q, W_UK c> + <q_r, k_r>.
 *
 * These calls stay inside their buffers whatever the device data holds, and can
 * be captured in a graph.  They need no workspace but splash_mla_prefill's.
 * Strides count elements (over one token, row, key or head they are not looked at);
 * `stream` and statuses as above.
 */
#define SPLASH_DIM_NOPE   128
#define SPLASH_DIM_ROPE   64
#define SPLASH_DIM_VALUE  128

/*
 * splash_mla_append: the new tokens' rows into the paged cache of any format.
 *   latent       bf16, element d < 512 of row t at t * latent_stride + d
 *   key          bf16, element r < 64 of row t at t * key_stride + r: the shared
 *                rotary key (views of a fused projection's rows)
 *   norm_weight  bf16 [512], or NULL: the latent is taken as it is
 *   positions, rope   as for splash_rope with rot_dim 64; rope NULL: the key is
 *                taken as it is, and positions are not read
 *   slots        int32 [num_tokens]; row t goes to row slots[t] % 64 of page
 *                slots[t] / 64; a slot outside [0, 64 * num_pages) is skipped.
 *                Slots are distinct (two rows of one slot race)
 *   kv_scales    SPLASH_KV_FP8_E4M3: desc->kv_scales, written; else ignored
 * With y[0:512] = latent * weight / sqrt(mean(latent^2) + norm_eps), formed in 64
 * bits and rounded to fp32, and y[512:576] the key's pairs turned (fp32, the angle
 * in 64 bits):
 *   SPLASH_KV_BF16        y rounded to bf16
 *   SPLASH_KV_FP8_E4M3    scale = max|y| / 448 (not below 2^-126; 1 where every y
 *                         is 0), codes = y / scale, an fp32 quotient, rounded to E4M3
 *   SPLASH_KV_FP8_LATENT  each 128 latent columns: scale = the least power of two,
 *                         2^-126 .. 2^63, with max|y| <= 448 * scale (1 where every
 *                         y is 0), codes = y / scale rounded to E4M3; the key
 *                         rounded to bf16
 * all to nearest even.  Maxima are of finite values; infinities (and what lies
 * past 448 * 2^63) take the largest code of their sign, NaN is E4M3's NaN.
 * desc: batch (0: a no-op), page_size, num_pages, kv_dtype and kv_scales are
 * used; num_heads and softmax_scale are only checked; flags are ignored.
 * Errors: INVALID_ARGUMENT (desc, NULL, num_tokens < 0, negative stride, norm_eps
 * negative or not finite, kv_scales other than desc's, rope as for splash_rope or
 * rot_dim != 64), UNSUPPORTED (desc, num_pages or num_tokens past 2^25), MISALIGNED
 * (latent, key, norm_weight or pages not 16-byte, strides not multiples of 8,
 * other arrays not 4-byte aligned).
 */
int splash_mla_append(const void* latent, int64_t latent_stride, const void* key, int64_t key_stride,
                      const void* norm_weight, float norm_eps, const int32_t* positions, int64_t position_stride,
                      const splash_rope_desc* rope, const int32_t* slots, int32_t num_tokens, void* kv_pages,
                      float* kv_scales, const splash_mla_desc* desc, void* stream);

/*
 * splash_mla_gather: rows of the cache back as dense bf16.  Rows row_indptr[b] ..
 * row_indptr[b+1] - 1 of the outputs are the tokens begin_b, begin_b + 1, ... of
 * request b's history (begin_b = key_begin[b], or 0 where key_begin is NULL):
 *   row_indptr   int32 [B+1], not decreasing; rows outside [row_indptr[0],
 *                row_indptr[B]) and past max_rows are left as they are
 *   latent_out   bf16 [max_rows, 512], row stride latent_stride
 *   key_out      bf16 [max_rows, 64], row stride key_stride (both may be parts
 *                of one [max_rows, 576] buffer)
 * A value is code * scale in fp32, rounded once to bf16 (exact where the scale
 * is a power of two and the value in bf16's range).  A token outside [0, 64 *
 * max_pages_per_seq), or whose block-table entry is outside the pool, gives a row of
 * zeros.  Errors: INVALID_ARGUMENT (desc, NULL, max_rows < 0, strides below the
 * row), UNSUPPORTED (desc, num_pages or max_rows past 2^25, max_pages_per_seq past
 * 2^25 - 1), MISALIGNED (pages or outputs not 16-byte, strides not multiples of
 * 8, other arrays not 4-byte aligned).
 */
int splash_mla_gather(const void* kv_pages, const int32_t* block_table, const int32_t* key_begin,
                      const int32_t* row_indptr, int32_t max_rows, void* latent_out, int64_t latent_stride,
                      void* key_out, int64_t key_stride, const splash_mla_desc* desc, void* stream);

/*
 * splash_mla_absorb_q: packed query rows for splash_mla_attend,
 *   q_out[n,h,0:512] = sum_d q[n,h,d] * w_uk[h,d,:]    (d < 128; fp32 sums)
 *   q_out[n,h,512:576] = q[n,h,128:192] turned by the token's position (rope NULL:
 *                        as it is, and positions are not read)
 * each rounded once to bf16.
 *   q       bf16, element d < 192 of head h of token n at n * q_token_stride +
 *           h * q_head_stride + d
 *   w_uk    bf16, element c < 512 of row d < 128 of head h at h * w_head_stride +
 *           d * w_row_stride + c (as it stands in a [heads, 256, 512]
 *           up-projection of keys and values)
 *   q_out   bf16 [num_tokens, num_heads, 576], over none of the inputs
 * splash_mla_expand_out: the attention's outputs through the value projection,
 *   y[n,h,v] = sum_c w_uv[h,v,c] * out[n,h,c]          (c < 512; fp32 sums)
 *   out     bf16 [num_tokens, num_heads, 512]
 *   w_uv    bf16, laid out as w_uk: row v < 128 of head h
 *   y       bf16, element v of head h of token n at n * y_token_stride + h *
 *           y_head_stride + v; rows must not overlap each other or the inputs
 * Errors of both: INVALID_ARGUMENT (NULL, negative counts or strides, rows of y
 * that overlap, rope as for splash_rope or rot_dim != 64), UNSUPPORTED (num_heads
 * past 1024, num_tokens past 2^24, their product past 2^28), MISALIGNED (tensors not 16-byte, strides not
 * multiples of 8, positions not 4-byte aligned).
 */
int splash_mla_absorb_q(const void* q, int64_t q_token_stride, int64_t q_head_stride, const void* w_uk,
                        int64_t w_head_stride, int64_t w_row_stride, const int32_t* positions, int64_t position_stride,
                        const splash_rope_desc* rope, int32_t num_tokens, int32_t num_heads, void* q_out,
                        void* stream);
int splash_mla_expand_out(const void* out, const void* w_uv, int64_t w_head_stride, int64_t w_row_stride,
                          int32_t num_tokens, int32_t num_heads, void* y, int64_t y_token_stride, int64_t y_head_stride,
                          void* stream);

/*
 * splash_mla_prefill: causal attention of ragged prompts over expanded keys and
 * values.  Request b's query rows are q_indptr[b] .. q_indptr[b+1] - 1 (nq of
 * them), its keys the rows kv_indptr[b] .. kv_indptr[b+1] - 1 (nk); query row i
 * of the request is its token nk - nq + i and sees keys j = 0 .. nk - nq + i (none
 * where that is negative: out = 0, lse = -inf):
 *   z_j        = softmax_scale * (<q[n,h,0:128], k[j,h,:]> + <q[n,h,128:192], key[j,:]>)
 *   lse[n,h]   = ln sum_j exp(z_j)
 *   out[n,h,:] = sum_j exp(z_j - lse[n,h]) * v[j,h,:]
 *   q     bf16 [num_rows, num_heads, 192] (rotary part turned), k, v bf16
 *         [num_keys, num_heads, 128], each with a token and a head stride (k and
 *         v may be the halves of one [.., 256] projection); key bf16 [num_keys, 64]
 *         with a token stride
 *   q_indptr, kv_indptr   int32 [batch+1], not decreasing; what lies past num_rows
 *         or num_keys is cut off.  Query rows outside [q_indptr[0], q_indptr[batch])
 *         are left as they are
 *   out   bf16 [num_rows, num_heads, 128] (round to nearest even), over none of the
 *         inputs
 *   lse   fp32 [num_rows, num_heads]; may be NULL
 *   workspace   splash_mla_prefill_workspace_size bytes (68 MB whatever the sizes: two
 *         parts of a tile for each workgroup of the chip), 16-byte aligned; it holds
 *         what one call leaves for its own second launch, and calls that may overlap
 *         take one each
 * Products are summed in fp32; a weight is rounded to bf16 where it meets V (2^-8), its
 * sum is not.  Weights in the sum are 1/8 a key at most on average: finite values past
 * 2^129 / nk may overflow it to an infinity or NaN.  Keys that a row does not see do not
 * touch it, whatever they hold (NaN and infinities in k, key and v among them); a score
 * that is NaN or +inf makes its row NaN.  An infinity or NaN in a v that a row sees
 * makes that value of the row infinite (both signs: NaN) or NaN, whatever the key's
 * weight, unless the row has no weight at all (every score -inf: out = 0, lse = -inf).
 * A score's own rounding, 2^-24 of it, is its weight's relative error: rows whose scores
 * pass 2^20 mean little, and past 2^30 may be NaN.  Deterministic: the same inputs and
 * sizes give the same bits.
 * Errors: INVALID_ARGUMENT (NULL, negative counts or strides, softmax_scale not
 * finite and > 0), UNSUPPORTED (num_heads past 1024, num_rows or num_keys past 2^25,
 * batch past 2^20, a token stride past 2^24, num_rows * num_heads past 2^31 - 1,
 * (num_rows / 128 + min(batch, num_rows)) * num_heads past 2^21),
 * MISALIGNED (tensors or workspace not 16-byte, strides not multiples of 8, other
 * arrays not 4-byte aligned), WORKSPACE_TOO_SMALL.
 */
typedef struct splash_mla_rows {
    const void* x;
    int64_t token_stride, head_stride;
} splash_mla_rows;

size_t splash_mla_prefill_workspace_size(int32_t batch, int32_t num_rows, int32_t num_heads);
int splash_mla_prefill(const splash_mla_rows* q, const splash_mla_rows* k, const void* key, int64_t key_stride,
                       const splash_mla_rows* v, const int32_t* q_indptr, const int32_t* kv_indptr, int32_t batch,
                       int32_t num_rows, int32_t num_keys, int32_t num_heads, float softmax_scale, void* out, float* lse,
                       void* workspace, size_t ws_bytes, void* stream);

/* Number of work units the workspace reserves: B*q_chunk + max_partials. */
int32_t splash_mla_max_units(int32_t batch, int32_t q_chunk, int32_t max_partials);

/* Compute units of the current device as the planner sees them (>= 1). */
int32_t splash_device_workers(void);

const char* splash_status_string(int status);
const char* splash_last_error(void);
const char* splash_version(void);

#ifdef __cplusplus
}
#endif

#endif /* SPLASH_ATTN_H */

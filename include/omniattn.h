/*
 * omniattn.h - C ABI of the MI355X (gfx950) sparse MLA decode library.
 *
 * For layers with grouped queries instead of a latent cache see "Grouped-query layers" at the end.
 * The rest is about one operation: decode-phase attention for absorbed multi-head latent
 * attention, restricted to the KV positions that OmniAttn's cache-compression
 * rule keeps.  For sequence b of length L_b the kept set is the first S
 * ("sink") positions and the last W ("recent") positions, as a set union
 * clipped to [0, L_b) (paper section 3.2.1, second equation, 0-based here),
 * and the result is softmax(q K_M^T * scale) V_M over that set (left-hand side
 * of the first equation of 3.2.1).  One (S, W) applies to every head of the
 * call (section 3.2.2: the layer, not the head, is the unit of compression).
 *
 * MLA layout (the paper only names MLA as compatible; shapes are the
 * DeepSeek-R1 absorbed decode form): each cached token is one latent row of
 * 576 numbers; the key is the whole row, the value is its first 512 numbers;
 * queries arrive already multiplied by the key up-projection.
 *
 * Conventions
 *   - All data pointers marked "device" are HIP device pointers owned by the
 *     caller; "host" pointers are ordinary memory.  The library owns only the
 *     plan object and the small device metadata it uploads for it.
 *   - `hip_stream` is a hipStream_t cast to void* (NULL = the null stream).
 *   - Every function returns 0 on success or a negative OMNIATTN_E* code.
 *     Nothing aborts and no C++ exception crosses this boundary.
 *   - The library is a HIP library: there is no CPU fallback.  On a machine
 *     without a usable GPU, omniattn_plan() and omniattn_decode() fail with
 *     OMNIATTN_EHIP; only the host-side planner (omniattn_plan_host) works.
 */
#ifndef OMNIATTN_H
#define OMNIATTN_H

#include <stddef.h>
#include <stdint.h>

#ifdef __cplusplus
extern "C" {
#endif

#define OMNIATTN_QK_DIM 576
#define OMNIATTN_V_DIM 512
#define OMNIATTN_PAGE 128

enum { OMNIATTN_BF16 = 0, OMNIATTN_FP8_E4M3 = 1, OMNIATTN_FP32 = 2 };

enum {
  OMNIATTN_OK = 0,
  OMNIATTN_EINVAL = -1,       /* null pointer, bad shape, bad size            */
  OMNIATTN_EUNSUPPORTED = -2, /* dtype / head count / dims not supported      */
  OMNIATTN_EWORKSPACE = -3,   /* workspace missing or too small               */
  OMNIATTN_EHIP = -4,         /* a HIP call failed; see omniattn_last_hip_error */
  OMNIATTN_ENOMEM = -5,       /* host allocation failed                       */
  OMNIATTN_ESCRATCH = -6      /* plan too large for omniattn_decode_static    */
};

/* Size of the library-owned device buffer omniattn_decode_static works in. */
#define OMNIATTN_STATIC_SCRATCH_BYTES (40u << 20)

/* Statement of one decode problem.  Fixed by the plan; the tensors come later. */
typedef struct {
  int32_t batch;             /* B >= 1 sequences                                        */
  int32_t num_heads;         /* H >= 1 query heads sharing each sequence's latent cache */
  int32_t qk_dim;            /* must be 576                                             */
  int32_t v_dim;             /* must be 512 (value = first 512 numbers of a cache row)  */
  int32_t page_size;         /* must be 128 tokens                                      */
  int32_t max_pages_per_seq; /* row stride of page_table, in int32 elements             */
  int64_t num_pages;         /* pages in the pool (for validation of host inputs only)  */
  int32_t sink;              /* S = N_sink  >= 0                                        */
  int32_t window;            /* W = N_recent >= 0; S + W >= L_b means dense attention   */
  float softmax_scale;       /* multiplies q.k before the softmax                       */
  int32_t kv_dtype;          /* OMNIATTN_BF16 | OMNIATTN_FP8_E4M3 (OCP e4m3, finite-only;
                                one fp32 scale per token multiplies the whole row)      */
  int32_t out_dtype;         /* OMNIATTN_BF16 | OMNIATTN_FP32                           */
  int32_t num_splits_hint;   /* 0: the library balances work over the GPU's compute
                                units.  n > 0: every sequence's retained tiles are cut
                                into min(n, tiles) pieces (for tests of the split path) */
  int32_t q_len;             /* queries per sequence (the query matrix of the first equation
                                of 3.2.1 has K rows); 0 or 1: one.  T > 1: the queries are
                                the last T tokens of the sequence (all already in the cache
                                and counted in L_b >= T), query t = 0 .. T-1 sits at position
                                L_b - T + t and sees the keys before and at it: the kept-set
                                rule is applied to a sequence of length L_b - (T - 1 - t).
                                q, out and lse then carry [B, T, H, ...] (query-major)    */
} omniattn_problem_t;

typedef struct omniattn_plan_s omniattn_plan_t; /* opaque, library-owned */

/*
 * Steps a1/a2 of the path: build the retained ranges of every sequence (second
 * equation of 3.2.1), cut them into KV tiles, partition tiles into work units
 * and size the workspace.  `seq_lens_host` is a host array of B context
 * lengths L_b >= 0 (the token being decoded is already in the cache and is
 * counted).  Requires ceil(L_b/128) <= max_pages_per_seq.
 *
 * omniattn_plan      also copies the metadata to the current HIP device so that
 *                    omniattn_decode can run: device and pinned host buffers are
 *                    allocated here (hipMalloc, hipHostMalloc; the pinned buffers of a
 *                    few destroyed plans are used again), the copy itself is
 *                    asynchronous on `hip_stream`, and decodes of this plan must be
 *                    ordered after it (same stream, or an event).  Work is balanced
 *                    over that device's CU count.
 * omniattn_plan_update  plans again for new lengths of the same problem (every decode
 *                    step changes every L_b) into the same object: host work, one
 *                    asynchronous copy from the plan's pinned buffer and one small
 *                    kernel on `hip_stream`; nothing is allocated and nothing
 *                    synchronises unless the new plan needs more metadata than any
 *                    before it.  (There are two pinned buffers: an update waits until
 *                    the copy two updates back is done, so the host runs at most two
 *                    updates ahead.)  The plan must not be in use by a decode on another
 *                    stream.  The workspace size may change: ask again.  On failure
 *                    for bad lengths the plan is unchanged.  A plan made by
 *                    omniattn_plan_host is planned again on the host only.
 * omniattn_plan_host builds the same plan for `num_cus` compute units without
 *                    touching HIP; such a plan can be inspected but
 *                    omniattn_decode on it returns OMNIATTN_EINVAL.
 * On failure *plan_out is set to NULL.
 */
int omniattn_plan(omniattn_plan_t** plan_out, const omniattn_problem_t* prob,
                  const int32_t* seq_lens_host, void* hip_stream);
/*
 * omniattn_plan with the metadata's device copy in `buffer` (device memory of the caller's, 16-byte aligned) if it holds
 * them, else in memory of the plan's own, as also after an update that outgrows it.  The buffer stays the caller's: it
 * has to live until the decodes of this plan are done, and destroying the plan then frees no device memory.  Nor does it
 * wait for any work, unless its pinned host buffers have to be freed: those of up to 16 destroyed plans per device are kept
 * for plans to come; those of further ones, those above 256 KB and those that a captured omniattn_plan_update reads are freed.
 * Making a plan, here or by omniattn_plan, waits for no stream but its own, and for that only where 16 are kept and the last
 * copy from each of them is still under way.
 */
int omniattn_plan_in(omniattn_plan_t** plan_out, const omniattn_problem_t* prob, const int32_t* seq_lens_host,
                     void* buffer, size_t buffer_bytes, void* hip_stream);
int omniattn_plan_update(omniattn_plan_t* plan, const int32_t* seq_lens_host, void* hip_stream);
int omniattn_plan_host(omniattn_plan_t** plan_out, const omniattn_problem_t* prob,
                       const int32_t* seq_lens_host, int32_t num_cus);
/* NULL is allowed.  Frees the plan's own device metadata, which waits for the work of the device (see omniattn_plan_in). */
void omniattn_plan_destroy(omniattn_plan_t* plan);

/* Introspection (host only, cheap). */
size_t omniattn_plan_workspace_bytes(const omniattn_plan_t* plan); /* may be 0 */
int64_t omniattn_plan_retained_tokens(const omniattn_plan_t* plan); /* sum_b |M_b| */
int32_t omniattn_plan_num_units(const omniattn_plan_t* plan);      /* grid of the main kernel */
int32_t omniattn_plan_num_segments(const omniattn_plan_t* plan);
int32_t omniattn_plan_num_partials(const omniattn_plan_t* plan);   /* partial results the combine kernel merges */
int32_t omniattn_plan_max_splits(const omniattn_plan_t* plan);     /* most pieces any one sequence was cut into */
int32_t omniattn_plan_num_splits(const omniattn_plan_t* plan);     /* the same number under its other name */
int32_t omniattn_plan_tile_tokens(const omniattn_plan_t* plan);    /* KV tokens per tile */
int32_t omniattn_plan_head_block(const omniattn_plan_t* plan);     /* heads per work unit */
int32_t omniattn_plan_unit_groups(const omniattn_plan_t* plan);    /* work groups that share a unit's heads: 1 or 2 */

/*
 * Copy out the plan's segments, 8 int32 each:
 *   [0] sequence b          [1] head block index     [2] first tile  [3] end tile
 *   [4] partial slot or -1  [5] work unit            [6] L_b         [7] tiles of b
 * Tiles are numbered along the sequence's retained tiles in ascending position.
 * Returns the number of segments written (<= cap) or a negative error.
 */
int32_t omniattn_plan_get_segments(const omniattn_plan_t* plan, int32_t* buf, int32_t cap);
/*
 * Logical token range [*lo, *hi) that retained tile `tile` of sequence `b`
 * spans (tile-aligned; the retained predicate still applies inside it).
 */
int omniattn_plan_tile_range(const omniattn_plan_t* plan, int32_t b, int32_t tile,
                             int32_t* lo, int32_t* hi);

/*
 * Steps a3-a9: gather retained tiles through the page table, QK^T, masking of
 * partial tiles, online softmax, PV, normalisation, and (when some sequence was
 * split) the combine pass.  Asynchronous on `hip_stream`; allocates nothing and
 * does not synchronise.  The current HIP device must be the one the plan was made on
 * (OMNIATTN_EINVAL otherwise).
 *
 *   q          device, bf16 [B, H, 576] contiguous (absorbed queries); [B, T, H, 576]
 *              for q_len = T > 1, and out / lse likewise [B, T, H, 512] / [B, T, H]
 *   kv_cache   device, bf16 or e4m3 bytes [num_pages, 128, 576] contiguous
 *   kv_scales  device, fp32 [num_pages, 128]; NULL unless kv_dtype is fp8.  Scales of
 *              retained tokens are finite and >= 0 (zero: a row of zeros).
 *   page_table device, int32 [B, max_pages_per_seq]; entry i of row b is the
 *              physical page of logical tokens [128 i, 128 i + 128).  Entries of
 *              pages that hold no retained token are never read.
 *   out        device, out_dtype [B, H, 512]
 *   lse        device, fp32 [B, H]: natural-log sum of exp(scale * q.k_j) over
 *              the retained j.  An empty retained set gives out = 0, lse = -inf.
 *   workspace  device, at least omniattn_plan_workspace_bytes(plan) bytes (partial
 *              rows of split sequences, in the output type, and their lse),
 *              256-byte aligned; may be NULL when that is 0.  Two decodes in
 *              flight at once need two workspaces.
 *
 * Slots outside the retained set, and pages not referenced, may hold anything
 * (NaN included) without effect.  Page ids of retained pages must lie in
 * [0, num_pages): the kernel does not check device-side contents.
 * Same plan + same inputs give bitwise identical results (nothing is accumulated atomically).
 * Arithmetic: bf16 cache - bf16 matrix products with fp32 accumulation, softmax weights
 * rounded to bf16.  fp8 cache - both products on the 8-bit matrix instruction; the query
 * enters as two e4m3 terms (exact for all but elements below 2^-14 of the row's largest), so
 * logits and lse carry fp32 accumulation error only; the softmax weights, with the token's
 * scale folded in, are rounded to e4m3 (relative 2^-4 per weight) and out is normalised by
 * the sum of the rounded weights.  A token whose scale is more than 2^10 below the largest
 * scale of its half of a 64-token tile (with blocks of 32 heads: of the whole tile)
 * has its value row taken at 2^-10 of that largest scale (its softmax weight counts in full).
 */
int omniattn_decode(const omniattn_plan_t* plan, const void* q, const void* kv_cache,
                    const float* kv_scales, const int32_t* page_table, void* out,
                    float* lse, void* workspace, size_t workspace_bytes, void* hip_stream);

/*
 * Same as omniattn_decode, and additionally records caller-owned HIP events
 * (hipEvent_t cast to void*, any may be NULL) on `hip_stream`: `ev_begin` before
 * the main kernel, `ev_main_end` after it, `ev_end` after the combine kernel
 * (recorded right after `ev_main_end` when the plan needs no combine).  For
 * benchmarks that report the main kernel's duration on its own; nothing is
 * allocated and nothing synchronises.
 */
int omniattn_decode_timed(const omniattn_plan_t* plan, const void* q, const void* kv_cache,
                          const float* kv_scales, const int32_t* page_table, void* out,
                          float* lse, void* workspace, size_t workspace_bytes, void* hip_stream,
                          void* ev_begin, void* ev_main_end, void* ev_end);

/*
 * For callers that cannot allocate device memory or pass a workspace: code under HIP
 * graph capture, tight serving loops, harnesses that forbid hipMalloc.  Same operation,
 * same kernels and same results as omniattn_decode, but the partial rows of split
 * sequences go to a buffer of OMNIATTN_STATIC_SCRATCH_BYTES (40 MiB) that is part of the
 * library's device image; every GPU the library runs on holds it until the process ends.
 * The call allocates nothing and does not synchronise.  A plan whose
 * omniattn_plan_workspace_bytes() exceeds the buffer is refused with OMNIATTN_ESCRATCH
 * (nothing is launched).  All calls on one GPU share that GPU's buffer: two calls that
 * overlap in time on one GPU (different streams) race; calls on one stream are ordered.
 * Nothing in the buffer has to start at zero: every partial row is written by the main
 * kernel before the merge reads it.
 */
int omniattn_decode_static(const omniattn_plan_t* plan, const void* q, const void* kv_cache,
                           const float* kv_scales, const int32_t* page_table, void* out,
                           float* lse, void* hip_stream);
size_t omniattn_static_scratch_bytes(void);

/*
 * Physically compressed cache of a compressed layer.  Section 3.2.1 keeps only the
 * N_sink first and the N_recent last tokens of a sequence, so such a layer never has
 * to store more: a sequence owns omniattn_ring_pages(S, W) pages however long it
 * grows - ceil(S/128) pinned pages for the logical pages that hold sink tokens, and
 * a ring of ceil(W/128) + 1 pages which all later logical pages use in turn.  A ring
 * page is handed to a new logical page only when every token of its previous
 * logical page has left the window (see omniattn_ring_slot).  The decode entry
 * points need nothing new: the page table simply maps the retained logical pages to
 * these pages, and entries of logical pages that hold no retained token are never
 * read.
 * Several queries per sequence (q_len = T > 1): the earliest of the T queries keeps W
 * positions that end T - 1 tokens before the newest one, so the layer must keep the
 * W + T - 1 most recent tokens.  omniattn_ring_pages and omniattn_ring_slot are functions
 * of that effective window: pass window + T - 1 to them.  omniattn_ring_append reads q_len
 * from `prob` and adds T - 1 itself.
 *
 * omniattn_ring_slot   which of the sequence's own pages (0 .. ring_pages-1) holds
 *                      logical page `logical_page` (host, pure function; negative
 *                      arguments give -1).
 * omniattn_ring_append appends one token to every sequence of the batch (device
 *                      work on `hip_stream`, asynchronous, allocates nothing):
 *   prob       batch, max_pages_per_seq, sink, window, q_len, kv_dtype are used
 *   seq_lens   device int32 [B]: lengths before the call; each is incremented
 *   new_rows   device [B, 576] bf16, or e4m3 bytes for an fp8 cache
 *   new_scales device fp32 [B] for an fp8 cache, else NULL
 *   seq_pages  device int32 [B, omniattn_ring_pages(S, W + T - 1)]: the pool pages each
 *              sequence owns (distinct)
 *   kv_cache, kv_scales  the pool, as for omniattn_decode
 *   page_table device int32 [B, max_pages_per_seq]: entry L/128 of row b is written
 *              when the new token (position L) opens a logical page
 * A sequence whose length has reached 128 * max_pages_per_seq is left unchanged
 * (nothing written, length not incremented); the caller can see that from seq_lens.
 */
int32_t omniattn_ring_pages(int32_t sink, int32_t window);
int32_t omniattn_ring_slot(int32_t sink, int32_t window, int32_t logical_page);
int omniattn_ring_append(const omniattn_problem_t* prob, int32_t* seq_lens, const void* new_rows,
                         const float* new_scales, const int32_t* seq_pages, void* kv_cache,
                         float* kv_scales, int32_t* page_table, void* hip_stream);

/*
 * Grouped-query layers: a paged cache in 8 bits and the three calls of a step.
 *
 * The same rule (the first `sink` and the last `window` tokens are kept) for layers whose cache holds K and V rows
 * of num_kv_heads heads instead of one latent row per token.  The cache holds e4m3 codes; `scale_tokens` tokens of
 * one head share a scale.  Nothing here needs a length on the host: lengths, page tables, slots and the division of
 * the work are read and made on the device, so a whole step can be captured once and replayed while the requests grow.
 *
 *   1. omniattn_table_extend   every request grows by its new tokens and takes the pages it needs
 *   2. omniattn_gqa_append     the new K and V rows of a layer go to their slots, rounded to 8 bits
 *   3. omniattn_gqa_decode     the new tokens' queries against the layer's cache
 *   and omniattn_table_release when requests have finished.
 *
 * All of them are asynchronous on `hip_stream`, allocate nothing, do not synchronise and return the codes above.
 * Sizes and alignment are checked, contents of device arrays are not: page ids lie in [0, num_pages), a request's
 * entries of page_table cover its length, free_pages[0 .. free_count) are distinct.
 */
typedef struct {
  int32_t batch;              /* B >= 1 requests                                                  */
  int32_t page_size;          /* must be 128 tokens                                               */
  int32_t max_pages_per_seq;  /* columns of page_table                                            */
  int32_t max_tokens;         /* entries of slot_map                                              */
  int64_t page_table_stride;  /* int32 elements from one row to the next, >= max_pages_per_seq     */
  int64_t num_pages;          /* pages of the pool, and entries of free_pages; < 2^24             */
} omniattn_table_t;

/*
 * One step's tables.  Request b has seq_lens[b] tokens and brings new_lens[b] >= 0.  In the order of the requests,
 * each takes the pages it lacks, ceil((L + n) / 128) - ceil(L / 128), from the top of the stack free_pages (page number
 * k of the call is free_pages[free_count - 1 - k]) and writes them into its row of page_table.
 *
 *   seq_lens, new_lens, q_start, slot_map, ...   device, int32
 *   seq_lens_out    [B]      lengths with the new tokens.  May be seq_lens itself.
 *   free_count_out  [1]      height of the stack afterwards.  May be free_count itself.
 *   q_start         [B + 1]  first new token of each request among the call's tokens (running sum of new_lens,
 *                           negative ones as 0; it stops at 2^31 - 1)
 *   slot_map        [max_tokens]  per new token: page * 128 + place in the page; -1 behind the last token
 * Arrays of input and output that are not the same must not overlap.
 * A request that does not fit is refused as a whole: its row of page_table would be too short, a length is negative,
 * its tokens reach past max_tokens, or the sum of the pages that requests up to it lack exceeds the stack (requests
 * that lack no page are not affected by that).  Its length stays, its tokens' slots are -1; q_start counts them all the
 * same, since they have their places among the call's rows (attention for them means nothing: their keys are not in the cache).
 *
 * omniattn_table_release puts the pages of the requests with done[b] != 0 back on the stack, in their order, and sets
 * their lengths to 0.  (seq_lens, free_pages and free_count change in place.)
 */
int omniattn_table_extend(const omniattn_table_t* table, const int32_t* seq_lens, const int32_t* new_lens,
                          const int32_t* free_pages, const int32_t* free_count, int32_t* page_table,
                          int32_t* seq_lens_out, int32_t* free_count_out, int32_t* q_start, int32_t* slot_map,
                          void* hip_stream);
int omniattn_table_release(const omniattn_table_t* table, const int32_t* done, int32_t* seq_lens,
                           const int32_t* page_table, int32_t* free_pages, int32_t* free_count, void* hip_stream);

typedef struct {
  int32_t batch;              /* B >= 1 requests                                                  */
  int32_t num_queries;        /* N: rows of q, all requests' query tokens together                */
  int32_t num_q_heads;        /* a multiple of num_kv_heads                                       */
  int32_t num_kv_heads;
  int32_t head_dim;           /* 64, 128 or 256                                                   */
  int32_t page_size;          /* must be 128 tokens                                               */
  int32_t scale_tokens;       /* tokens of one head that share a scale: 32, 64 or 128             */
  int32_t max_pages_per_seq;
  int64_t page_table_stride;  /* int32 elements from one row of page_table to the next            */
  int64_t num_pages;          /* pages of the cache, < 2^24                                       */
  int32_t sink;               /* S >= 0                                                           */
  int32_t window;             /* W >= 0; S + W >= L keeps everything                              */
  float softmax_scale;
  int32_t out_dtype;          /* OMNIATTN_BF16 | OMNIATTN_FP32                                    */
} omniattn_gqa_t;

/*
 * New K and V rows into the cache.  (Of `gqa`: num_kv_heads, head_dim, page_size, scale_tokens and num_pages count.)
 *   k_new, v_new        device, bf16 [num_tokens, num_kv_heads, head_dim]; k_stride and v_stride elements from one token
 *                       to the next (multiples of 8, rows 16-byte aligned)
 *   slot_map            device, int32 [num_tokens]; tokens with a slot that is not in the cache are left out
 *   k_cache, v_cache    device, e4m3 [num_pages, num_kv_heads, 128, head_dim]
 *   k_scales, v_scales  device, fp32 [num_pages, num_kv_heads, 128 / scale_tokens]
 * A block's scale is a power of two, the smallest (from 2^-126) by which its largest finite magnitude is at most 448; 0
 * for a block of zeros.  A number that is not finite becomes NaN.  Tokens of one block in a call have to follow one
 * another in the call and in the block (as slot_map of omniattn_table_extend has them).  A block whose first token is
 * written begins anew.  Otherwise its earlier tokens stay: the scale is the larger of the old one and the new tokens',
 * and where it has grown the earlier codes are multiplied by old / new and rounded again (exact but for numbers that
 * become subnormal).  Tokens behind the last one written are undefined.
 */
int omniattn_gqa_append(const omniattn_gqa_t* gqa, int32_t num_tokens, const void* k_new, int64_t k_stride, const void* v_new,
                        int64_t v_stride, const int32_t* slot_map, void* k_cache, void* v_cache, float* k_scales,
                        float* v_scales, void* hip_stream);

/*
 * Attention of the call's query tokens over the cache.  Request b has seq_lens[b] tokens in the cache; its queries are its
 * last n = q_start[b + 1] - q_start[b] tokens, query t sees the keys before and at its own position L - n + t, and keeps of
 * them the first `sink` and the last `window`.
 *   q           device, bf16 [N, num_q_heads, head_dim]; q_stride elements from one token to the next (a multiple of 8)
 *   k_scales, v_scales   finite, >= 0 for blocks that hold kept tokens; any numbers, not only powers of two
 *   page_table  device, int32 [B, max_pages_per_seq]; entries of pages without kept tokens are not read
 *   seq_lens    device, int32 [B]
 *   q_start     device, int32 [B + 1], ascending, at most N; NULL: one query for each request (N = B)
 *   out         device, out_dtype [N, num_q_heads, head_dim]; rows of no request are left as they are
 *   lse         device, fp32 [N, num_q_heads], natural logarithm.  A query that keeps nothing gives 0 and -inf.
 *   workspace   device, omniattn_gqa_workspace_bytes(gqa) bytes, 256-byte aligned (enough for calls of fewer queries, and of any kept
 *               set and table width, too); calls in flight at once need one each
 * Tokens that a query does not keep may hold anything (NaN too) without effect on it; a kept NaN in a K row makes the query's row and
 * its lse NaN, one in a V row the columns in which it stands.
 * Same inputs give bitwise identical results.  Arithmetic: codes and queries enter the matrix instructions exactly (bf16),
 * logits, sums and outputs are held in fp32; a weight times its value block's scale enters in two f16 terms (relative 2^-22 down to
 * 2^-14 of the row's largest such product, and 2^-36 of that below).  A bf16 result is the fp32 result rounded.
 *
 * omniattn_gqa_workspace_bytes depends on the current device and on batch, num_queries, the head counts and head_dim;
 * 0 for an invalid problem.  It is enough for omniattn_gqa_tree too, whose blocks are larger; omniattn_gqa_decode_workspace_bytes, which is that or less,
 * for omniattn_gqa_decode alone (head_dim 128, more than 32 query rows to a request and KV head, 256 compute units: 17 MB instead of 69).
 */
size_t omniattn_gqa_workspace_bytes(const omniattn_gqa_t* gqa);
size_t omniattn_gqa_decode_workspace_bytes(const omniattn_gqa_t* gqa);
int omniattn_gqa_decode(const omniattn_gqa_t* gqa, const void* q, int64_t q_stride, const void* k_cache, const void* v_cache,
                        const float* k_scales, const float* v_scales, const int32_t* page_table, const int32_t* seq_lens,
                        const int32_t* q_start, void* out, float* lse, void* workspace, size_t workspace_bytes,
                        void* hip_stream);

/*
 * Speculative decoding on grouped-query layers.  Every request brings a tree of drafted tokens instead of one token: node 0 is the last
 * token of its text (the one that the step before has chosen), every other node follows its parent, which comes before it.  The nodes are
 * the request's new tokens: omniattn_table_extend counts them, omniattn_gqa_append puts their rows behind the text, in the nodes'
 * order.  The rest of a step:
 *
 *   1. omniattn_tree_masks      which nodes each node follows, and its position in the text (for a rotation of queries and keys)
 *   2. omniattn_gqa_tree        attention of the nodes' queries, for every layer
 *   3. omniattn_tree_verify     which nodes stay, and the tokens that follow them
 *   4. omniattn_gqa_keep        rows of the nodes that stay move up behind the text, for all layers
 *   5. omniattn_table_truncate  the other nodes and their pages go
 *
 * A request has n = q_start[b + 1] - q_start[b] <= OMNIATTN_TREE_NODES nodes, as omniattn_table_extend numbers them (q_start NULL: one
 * each).  Like the calls above these are asynchronous, allocate nothing and read no length on the host; arrays of nodes lie behind one another
 * as the requests do; rows of no request are left as they are.
 *
 * A node's row can raise the scale of a block that holds text (see omniattn_gqa_append), whose codes are rounded again then.  That stays when
 * the node goes: the scale of such a block never falls, and numbers of the text that have become subnormal under it keep what bits they have left.
 */
#define OMNIATTN_TREE_NODES 64

/*
 *   parents    device, int32 [num_tokens]: the parent's number among the request's nodes.  One that does not come before the node (such as -1):
 *              the node follows the text directly.
 *   seq_lens   device, int32 [batch]: lengths with the nodes
 *   masks      device, uint64 [num_tokens]: bit a is set if the node follows node a or is node a.  0 for every node of a request with
 *              too many.
 *   positions  device, int32 [num_tokens] or NULL: L - n + (bits of the mask) - 1; -1 in a request with too many nodes
 */
int omniattn_tree_masks(int32_t batch, int32_t num_tokens, const int32_t* parents, const int32_t* seq_lens, const int32_t* q_start,
                        uint64_t* masks, int32_t* positions, void* hip_stream);

/*
 * Attention of the nodes' queries.  As omniattn_gqa_decode, except for what a query sees: with t the number of bits of its mask among the
 * request's nodes and P = L - n + t - 1 its position, the tokens j < L - n of the text with j < sink or j > P - window, and the nodes a of its mask
 * whose own positions L - n + (bits of the mask below a) pass the same test.  (Any set of nodes will do, a tree's or not.)  A query whose mask
 * has no bit of a node keeps nothing.
 *   masks       device, uint64 [N].  Bits of nodes that the request does not have do not count; nodes from number 64 on are seen by none.
 *   page_table  entries are read of pages that hold nodes (with window 0: if the text is shorter than sink), or tokens that a query at the
 *               first node's position keeps
 *   workspace   omniattn_gqa_workspace_bytes, as for omniattn_gqa_decode: calls of either kind share one
 */
int omniattn_gqa_tree(const omniattn_gqa_t* gqa, const void* q, int64_t q_stride, const void* k_cache, const void* v_cache, const float* k_scales,
                      const float* v_scales, const int32_t* page_table, const int32_t* seq_lens, const int32_t* q_start,
                      const uint64_t* masks, void* out, float* lse, void* workspace, size_t workspace_bytes, void* hip_stream);

/* What a verification is about. */
typedef struct {
  int32_t batch;              /* B >= 1 requests                                                  */
  int32_t num_tokens;         /* N: all requests' nodes together                                  */
  int32_t vocab;              /* V >= 1                                                           */
  int32_t logits_dtype;       /* OMNIATTN_BF16 | OMNIATTN_FP32                                    */
} omniattn_verify_t;

/*
 * Which drafted tokens stay.  Row i of `logits` is the target's for the token behind node i; p = softmax(logits / T), T the request's
 * temperature.  For every node a token y is chosen:
 *   T not above 0    the first of the largest logits
 *   no draft_probs   y = the first v with p_0 + .. + p_v > u1 (p_0 + .. + p_V-1)
 *   draft_probs      row i is the distribution q that the token of the node's first child was drawn from.  That child x is taken if
 *                    u0 q(x) < p(x).  Otherwise y is chosen as above with max(p - q, 0) in p's place (with p, if that is 0 everywhere).
 *                    A node without children is treated as without q.
 * From node 0 on, the first child whose token is y is the path's next node; the path ends where there is none.  So the tokens along the path
 * and the one behind it are distributed as the target's own, however the drafts were found (other children than a first one must not depend on
 * u1).  u0, u1 = uniforms[i], in [0, 1).
 *
 *   logits       device, logits_dtype [N, V]; logits_stride elements from one row to the next.  NaN counts as -inf.  A row with +inf gives
 *                the first such token, one of -inf only gives -1, which ends the path.  (Its node stays on it, so that no token is new: the text
 *                ends with one whose row is in the cache, and no tree can follow.)
 *   draft_probs  device, fp32 [N, V], draft_stride elements from one row to the next; or NULL
 *   tokens       device, int32 [N]: the nodes' tokens (those outside [0, V) are never taken)
 *   parents      as for omniattn_tree_masks; nodes that do not descend from node 0 are not reached
 *   temperature  device, fp32 [B]
 *   uniforms     device, fp32 [N, 2]
 *   path         device, int32 [N]: for every request the nodes that stay, in ascending order from node 0 on, then -1
 *   out_tokens   device, int32 [N]: the token behind each of them; the last one is new; then -1
 *   logprobs     device, fp32 [N] or NULL: ln p of these tokens (T not above 0: at temperature 1); then 0
 *   dropped      device, int32 [B]: nodes that do not stay
 *   workspace    device, omniattn_tree_verify_workspace_bytes(verify) bytes, 256-byte aligned (enough for fewer nodes, too); calls in
 *                flight at once need one each
 * A request with too many nodes keeps none.  Numbers are held in 64 bits; an exponential is good to 4.7e-11 of itself, a probability to 1.9e-10 (its own and
 * three in the sum); exp(0) is 1.  A token whose weight beside its row's likeliest is not above 2^-1020 has none, with u1 = 0 too.  Same inputs give the same results.
 */
size_t omniattn_tree_verify_workspace_bytes(const omniattn_verify_t* verify);
int omniattn_tree_verify(const omniattn_verify_t* verify, const void* logits, int64_t logits_stride, const float* draft_probs, int64_t draft_stride,
                         const int32_t* tokens, const int32_t* parents, const int32_t* q_start, const float* temperature,
                         const float* uniforms, int32_t* path, int32_t* out_tokens, float* logprobs, int32_t* dropped,
                         void* workspace, size_t workspace_bytes, void* hip_stream);

/*
 * Rows of the nodes that stay move up in the cache: row L - n + path[i] goes to row L - n + i, in num_layers layers that lie behind one
 * another, for K and V.  (Of `gqa`: batch, num_queries (all requests' nodes together), num_kv_heads, head_dim, page_size, scale_tokens,
 * max_pages_per_seq, page_table_stride and num_pages, of a layer, count.)
 *   path        device, int32 [num_queries], as omniattn_tree_verify writes it: a request's path ascends from its first entry on and ends before
 *               the first entry that does not, or is no node (such as -1)
 *   seq_lens    device, int32 [B]: lengths with the nodes (before omniattn_table_truncate)
 *   k_cache, v_cache    device, e4m3 [num_layers, num_pages, num_kv_heads, 128, head_dim]
 *   k_scales, v_scales  device, fp32 [num_layers, num_pages, num_kv_heads, 128 / scale_tokens], finite, >= 0
 * The scale of a block that a row moves to becomes the largest of the scales that its rows of the path came with and, where tokens of the
 * text lie in it, its own; codes of these rows and tokens are multiplied by old / new and rounded (exact for powers of two but for
 * numbers that become subnormal).  Blocks that no row moves to stay as they are, and so do the codes of nodes that nothing moves to (their tokens
 * are undefined once the path is taken).  A request with too many nodes, or more than it has tokens, is left alone.
 */
int omniattn_gqa_keep(const omniattn_gqa_t* gqa, int32_t num_layers, const int32_t* path, const int32_t* seq_lens, const int32_t* q_start,
                      const int32_t* page_table, void* k_cache, void* v_cache, float* k_scales, float* v_scales, void* hip_stream);

/*
 * Requests lose their last tokens: of L, L - min(max(dropped, 0), L) are left, and the pages above them go back on the stack, in the order
 * of the requests and of their rows.  (max_tokens of `table` does not count.)  seq_lens_out may be seq_lens, free_count_out may be free_count.
 */
int omniattn_table_truncate(const omniattn_table_t* table, const int32_t* seq_lens, const int32_t* dropped, const int32_t* page_table,
                            int32_t* free_pages, const int32_t* free_count, int32_t* seq_lens_out, int32_t* free_count_out,
                            void* hip_stream);

const char* omniattn_strerror(int code);
/* Text of the last HIP error seen by the calling thread ("" if none). */
const char* omniattn_last_hip_error(void);

#ifdef __cplusplus
}
#endif
#endif /* OMNIATTN_H */

/*
 * gr.h - C ABI of the MI355X (gfx950) generative-recommendation decode hot path.
 *
 * One decode step of beam-search item generation (xGR paper, arxiv 2512.11529) is
 *   1. attention of all W beam queries of a request over a *separated* KV cache: one shared copy of
 *      the prompt K/V per request plus W short per-beam decode caches (Sections 5.1, 5.2);
 *   2. the beam item step: valid-item mask, log-softmax over valid tokens, cumulative beam score,
 *      and the best W of the W*V candidates (Sections 6.1, 6.2), in fixed caller-owned buffers
 *      (Section 6.3);
 *   3. the move of every surviving beam's own decode cache to its new slot, in place (Section 5.1) - or, moving no
 *      bytes, the update of a slot table that the attention follows (gr_beam_slot_update, gr_beam_attn_slots).
 * Beside the step: the prefill that fills the shared cache (gr_prefill_attn), the step's attention over a shared
 * cache stored in FP8 (gr_beam_attn_fp8kv), a prompt cache in pages with a prefix that requests share (gr_page_map, gr_page_write,
 * gr_page_append, gr_page_read, gr_beam_attn_paged), norms and rotation of queries and keys (gr_qk_norm_rope), penalties, biases and masks on the logits (gr_logits_adjust), an item step for callers that cannot allocate
 * (gr_beam_select_noalloc), and a few diagnostics used by the benchmark (gr_diag_*).
 *
 * Conventions for every entry point
 *   - All data pointers are DEVICE pointers unless a comment says "host".  Parameter structs and
 *     scalar arguments are host values read before the call returns.
 *   - The caller owns every buffer, including workspaces and the mask blob.  The library never
 *     allocates, frees or keeps device memory and holds no state between calls (three exceptions, stated
 *     where they are declared: the static scratch array of gr_beam_select_noalloc, the launch-plan
 *     override of gr_diag_attn_plan and the page of host memory that gr_item_mask_build reports through).
 *   - The attention calls, gr_beam_select and gr_beam_reorder only enqueue kernels on `stream` (a hipStream_t passed as
 *     void*, NULL = default stream); they never synchronise.  gr_item_mask_build is a load-time
 *     call and synchronises `stream` once to report table errors.
 *   - Return value: GR_OK or a negative gr_status.  Nothing is printed, thrown or aborted.
 *     Host-checkable argument errors are reported before anything is enqueued.
 *   - The calls around pages and logits (gr_page_*, gr_beam_attn_paged, gr_qk_norm_rope, gr_logits_adjust) report UNSUPPORTED for shapes whose launch would
 *     have 2^32 threads or more (from 2^24 rows of logits on, or 2^23 blocks of query rows and segments).
 *   - bf16 tensors are raw 16-bit patterns; all tensors are dense, row-major, in the stated shape.
 */
#ifndef GR_H_
#define GR_H_

#include <stddef.h>
#include <stdint.h>

#ifdef __cplusplus
extern "C" {
#endif

typedef int32_t gr_status;
enum {
  GR_OK = 0,
  GR_ERR_INVALID_ARG = -1,        /* NULL pointer, non-positive size, step/u out of range, aliasing rule broken */
  GR_ERR_UNSUPPORTED = -2,        /* shape outside what the kernels implement (see each call) */
  GR_ERR_WORKSPACE_TOO_SMALL = -3,
  GR_ERR_BAD_TABLE = -4,          /* item table unsorted, has duplicates, or a token outside [0, V) */
  GR_ERR_HIP = -5                 /* a HIP runtime call or kernel launch failed */
};

/* Static description of a status code (host pointer, never NULL). */
const char* gr_status_string(gr_status s);

/* ------------------------------------------------------------------------------------------------
 * gr_beam_attn - shared-prefix beam attention (Section 5.1 cache layout, Section 5.2 staging).
 *
 * For every request b, beam w and query head h (KV head h / (Hq/Hkv)) computes softmax attention of
 * q[b,w,h,:] over the L_b prompt tokens of request b (stored ONCE, shared by all W beams) followed
 * by that beam's own u decode tokens:
 *     s_j = sm_scale * <q, k_j>,   out = sum_j softmax(s)_j v_j,   lse = log sum_j exp(s_j).
 * The shared stage streams each prompt K/V tile once per workgroup for many beam queries (bf16
 * MFMA, fp32 accumulation, online softmax); the unshared stage adds each beam's own tokens; the
 * merge combines the (max, sum, output) partials.  No causal mask is applied: every key precedes
 * or is the query position.
 *
 * Supported: d in {64, 128}; Hq % Hkv == 0; 1 <= u <= ND; L_b >= 0 (L_b + u >= 1).  All bf16 tensors must be
 * 16-byte aligned (INVALID_ARG otherwise) and hold finite values.  Sums are fp32 and normalised at the end:
 * |v| * 2^8 * (L_b + u) has to stay below 2^128.  The probabilities, not their sum, are rounded to bf16 for the product with V (an error of at most 2^-8 of a
 * token's share each, beside the rounding of `out`); so do all attention calls here.
 * ------------------------------------------------------------------------------------------------ */
typedef struct {
  int32_t B, W, Hq, Hkv, d;   /* requests, beam width, query heads, KV heads, head dim              */
  int32_t ND, u;              /* decode-token capacity per beam (Section 5.1: sized up front) and   */
                              /* number of valid decode tokens this step                            */
  int32_t max_L;              /* host copy of max_b L_b (sizes the launch; no device read-back)     */
  int64_t total_L;            /* host copy of sum_b L_b = cu_seqlens[B]                             */
  float   sm_scale;           /* softmax scale, normally 1/sqrt(d); must be positive and finite     */
  const void*    q;           /* bf16 [B, W, Hq, d]                                                 */
  const void*    k_shared;    /* bf16 [total_L, Hkv, d]; request b = rows cu_seqlens[b]..[b+1]      */
  const void*    v_shared;    /* bf16 [total_L, Hkv, d]                                             */
  const int32_t* cu_seqlens;  /* int32 [B+1], non-decreasing, cu_seqlens[0] = 0                     */
  const void*    k_unshared;  /* bf16 [B, W, ND, Hkv, d]; token slots [0, u) valid                  */
  const void*    v_unshared;  /* bf16 [B, W, ND, Hkv, d]                                            */
  void*          out;         /* bf16 [B, W, Hq, d]                                                 */
  float*         lse_out;     /* fp32 [B, W, Hq] natural-log sum-exp of the scaled scores; or NULL  */
} gr_attn_params;

/* Bytes of workspace gr_beam_attn needs for these shapes (0 is possible).  Host only. */
size_t gr_beam_attn_workspace_bytes(const gr_attn_params* p);

/* Enqueue the attention.  `workspace` (device, 256-byte aligned) holds split-L partials and, for a
 * ragged batch of more than 128 requests, the order in which they are dispatched (longest prompt first; fewer
 * requests find their place themselves, though the order's bytes are part of the size for any ragged batch); contents
 * before and after the call are unspecified.  Errors: INVALID_ARG, UNSUPPORTED,
 * WORKSPACE_TOO_SMALL, HIP. */
gr_status gr_beam_attn(const gr_attn_params* p, void* workspace, size_t workspace_bytes, void* stream);

/* ------------------------------------------------------------------------------------------------
 * gr_beam_attn_fp8kv - gr_beam_attn over a shared (prompt) cache stored in FP8: the "separated KV cache" of
 * Section 5.1 with its large, read-only half held at one byte per element.  `attn.k_shared` / `attn.v_shared` point
 * to OCP FP8 E4M3 codes, uint8 [total_L, Hkv, d]; the value of an element is code * k_scale (resp. * v_scale),
 * one positive finite scale per tensor.  Everything else (Q, the beams' own decode-token caches, output, workspace,
 * launch rule, errors) is as for gr_beam_attn; the codes are widened to bf16 exactly on their way into LDS and the
 * scales are applied to the scores and to the prompt's share of the output in fp32.
 * ------------------------------------------------------------------------------------------------ */
typedef struct {
  gr_attn_params attn;        /* as for gr_beam_attn, except the element type of k_shared / v_shared */
  float k_scale, v_scale;     /* value = code * scale; must be positive and finite                    */
} gr_attn_fp8kv_params;

/* Workspace: gr_beam_attn_workspace_bytes(&p->attn). */
gr_status gr_beam_attn_fp8kv(const gr_attn_fp8kv_params* p, void* workspace, size_t workspace_bytes, void* stream);

/* ------------------------------------------------------------------------------------------------
 * gr_prefill_attn - causal self-attention over the packed prompts: the prefill phase that produces the
 * shared cache (Section 2.2.1 "Prefill"; Section 5.1: the shared cache stores the prompt's token-level
 * outputs of the prefill phase; the abstract's single staged computation for prefill and decode).
 *
 * For request b, token i (0 <= i < L_b), query head hq with KV head hq / (Hq/Hkv):
 *     out[i, hq, :] = softmax_j( sm_scale * <q[i, hq], k[j, kvh]> ) . v[j, kvh]   over the keys j = 0..i
 * of the same request.  It runs through the tiles of gr_beam_attn (bf16 MFMA, fp32 accumulation, bf16
 * output): a block of query rows walks the request's K/V tiles up to its own last token and masks
 * the tiles on the diagonal.  No workspace.  Only enqueues on `stream`; no synchronisation.
 *
 * Supported: d in {64, 128}; Hq % Hkv == 0; total_L < 2^31; max_L * Hq/Hkv < 2^22;
 * max_L * Hkv * d * 2 < 2^32; max_L * Hq * d < 2^31.  All bf16 tensors 16-byte aligned.
 * ------------------------------------------------------------------------------------------------ */
typedef struct {
  int32_t B, Hq, Hkv, d;
  int32_t max_L;              /* host copy of max_b L_b (sizes the grid)                             */
  int64_t total_L;            /* host copy of cu_seqlens[B] (chooses the plan)                       */
  float   sm_scale;           /* multiplies the scores; must be positive and finite                  */
  const void*    q;           /* bf16 [total_L, Hq, d]  (device), packed like k and v                */
  const void*    k;           /* bf16 [total_L, Hkv, d]                                              */
  const void*    v;           /* bf16 [total_L, Hkv, d]                                              */
  const int32_t* cu_seqlens;  /* int32 [B+1] (device): request b owns rows cu[b] .. cu[b+1]-1        */
  void*          out;         /* bf16 [total_L, Hq, d]                                               */
  float*         lse_out;     /* fp32 [total_L, Hq] natural-log sum-exp of the scaled scores; or NULL */
} gr_prefill_params;

/* Errors: INVALID_ARG, UNSUPPORTED, HIP.  An empty batch (total_L == 0) is GR_OK and launches nothing. */
gr_status gr_prefill_attn(const gr_prefill_params* p, void* stream);

/* ------------------------------------------------------------------------------------------------
 * gr_item_mask_build - valid-item mask, built once at load time (Section 6.1: dense masks are
 * pre-generated during model loading; the last level is kept in sparse form).
 *
 * Input: the table of valid items, int32 [n_items, depth], rows sorted lexicographically and
 * distinct, tokens in [0, V).  Output: one position-independent device blob (offsets, no pointers;
 * may be copied or saved) holding
 *   level 0   bitmask of valid first tokens (V bits);
 *   level 1   dense bitmask of valid second tokens per first token (V x V bits), plus the same
 *             children in sparse CSR form and the table row range of every first token;
 *   level 2   sparse: the third-token column of the table, addressed by row range.
 * The blob is read-only for gr_beam_select and is shared by every step of every request.
 *
 * Supported: depth == 3; 1 <= V <= 32768; 1 <= n_items < 2^31.
 * ------------------------------------------------------------------------------------------------ */
size_t gr_item_mask_bytes(int64_t n_items, int32_t depth, int32_t V);
size_t gr_item_mask_build_workspace_bytes(int64_t n_items, int32_t depth, int32_t V);

/* items_sorted: device int32 [n_items, depth].  mask_out: device, 256-byte aligned, mask_bytes >=
 * gr_item_mask_bytes().  Synchronises `stream`; returns GR_ERR_BAD_TABLE if the on-device check of
 * order / distinctness / token range fails (mask_out is then unspecified).  The first call of a process allocates one
 * page of pinned host memory through which the kernels report (kept until the process ends; calls may run
 * concurrently from any threads, on any streams and GPUs).  As calls that synchronise do, it breaks off a graph capture
 * that another thread has open in global mode. */
gr_status gr_item_mask_build(const int32_t* items_sorted, int64_t n_items, int32_t depth, int32_t V,
                             void* mask_out, size_t mask_bytes, void* workspace, size_t workspace_bytes,
                             void* stream);

/* ------------------------------------------------------------------------------------------------
 * gr_beam_select - beam item step (Sections 6.1-6.3).
 *
 * For each request, for each live beam w (scores_in[w] > -inf) with logits x[v]:
 *     valid(v) = some item starts with (prefix of w, v)                      (mask blob lookup)
 *     m = max over valid x;  S = sum over valid exp(x - m) accumulated in fp64
 *     lse = fp32(m + log S);  bias = scores_in[w] - lse;  cand[w*V+v] = bias + x[v]   (fp32 ops)
 * and the W best candidates by (cand descending, flat index w*V+v ascending) are written, best
 * first.  Selection stops reading as soon as the W survivors are fixed (threshold filtering
 * instead of a sort of all W*V candidates - the early-termination idea of Section 6.2).
 * Slots past the number of finite candidates are dead: parent = token = -1, score = -inf,
 * prefix = -1, range = [0,0), item index = -1.
 *
 * Prefix state carried between steps (Section 6.3: fixed-size structures, overwritten in place by
 * the caller swapping in/out buffers):
 *   prefix  int32 [B, W, depth]  tokens chosen so far (entries >= step+1 are -1 on output)
 *   range   int32 [B, W, 2]      table row range [lo, hi) of the prefix
 * Step 0 ignores prefix_in/range_in.  Step 1 reads prefix_in[...,0]; step 2 reads range_in.
 * Behaviour is undefined if scores or the logits of a live beam contain NaN, or if a live beam's prefix/range is not
 * one this mask produced.  What the logits of dead beams hold is of no effect.
 *
 * mask == NULL: unconstrained (every token valid); range_out = [0,0), item_index_out = -1.
 * Supported: depth == 3; 1 <= W <= 2048; 1 <= V <= 32768; W*V < 2^31.
 * ------------------------------------------------------------------------------------------------ */
enum {
  GR_SELECT_FORCE_DENSE = 1     /* stream every live row in full even when a sparse gather would be cheaper */
};

typedef struct {
  int32_t B, W, V, depth, step;   /* 0 <= step < depth                                              */
  int32_t flags;                  /* GR_SELECT_* bits                                               */
  const void*    mask;            /* blob from gr_item_mask_build (built for the same V, depth)     */
  const float*   logits;          /* fp32 [B, W, V]                                                 */
  const float*   scores_in;       /* fp32 [B, W]; -inf = dead beam                                  */
  const int32_t* prefix_in;       /* int32 [B, W, depth]                                            */
  const int32_t* range_in;        /* int32 [B, W, 2]                                                */
  int32_t*       parent_out;      /* int32 [B, W] index of the beam each survivor extends           */
  int32_t*       token_out;       /* int32 [B, W] token appended                                    */
  float*         scores_out;      /* fp32 [B, W] cumulative log-probability, non-increasing; may be scores_in (all outputs may */
                                  /* lie on scores_in, which is read before any of them is written) */
  int32_t*       prefix_out;      /* int32 [B, W, depth]; must not alias prefix_in                  */
  int32_t*       range_out;       /* int32 [B, W, 2];     must not alias range_in                   */
  int32_t*       item_index_out;  /* int32 [B, W] table row of the finished item when step ==       */
                                  /* depth-1 (else -1); may be NULL                                 */
} gr_select_params;

size_t gr_beam_select_workspace_bytes(int32_t B, int32_t W, int32_t V, int32_t depth);

/* Enqueue the item step.  `workspace`: device, 256-byte aligned, contents unspecified before and
 * after.  Errors: INVALID_ARG, UNSUPPORTED, WORKSPACE_TOO_SMALL, HIP. */
gr_status gr_beam_select(const gr_select_params* p, void* workspace, size_t workspace_bytes, void* stream);

/* ------------------------------------------------------------------------------------------------
 * gr_beam_select_noalloc - gr_beam_select for callers that cannot allocate device memory or carry a
 * workspace around: code under HIP graph capture, tight serving loops, harnesses that forbid hipMalloc.
 *
 * Same parameters, same results and same errors as gr_beam_select; the workspace is a static device array
 * inside the library (gr_beam_select_noalloc_max_workspace_bytes() bytes, 16 MiB: on every GPU the library
 * runs on until the process ends).  A shape whose gr_beam_select_workspace_bytes() exceeds that limit is
 * rejected with GR_ERR_WORKSPACE_TOO_SMALL before anything is enqueued (at V = 8192 the limit is about 16 000
 * beam rows, B * W).  The call allocates nothing and frees nothing; the first call on a device looks up the
 * array's address on that device (no synchronisation).  All calls on one GPU share the array: calls that
 * overlap in time on one GPU (different streams, different host threads) race and give undefined results -
 * order them, or use gr_beam_select with separate workspaces.
 * ------------------------------------------------------------------------------------------------ */
size_t    gr_beam_select_noalloc_max_workspace_bytes(void);
gr_status gr_beam_select_noalloc(const gr_select_params* p, void* stream);

/* ------------------------------------------------------------------------------------------------
 * gr_beam_reorder - in-place update of the unshared cache between two decode steps (Section 5.1).
 *
 * After gr_beam_select, slot j of the new beam generation continues old beam parent[b, j].  The
 * per-beam decode cache follows it inside the single buffer that holds it (no second copy):
 *     cache[b, j, t, :, :] <- cache[b, parent[b, j], t, :, :]     for token slots t in [0, u)
 * for both K and V.  Slots with parent < 0 (dead beams) are zero-filled; token slots >= u are left
 * untouched (the caller writes slot u next).  The paper orders row moves by direction so that no
 * block is overwritten before it is read; this call gives the same guarantee for any parent
 * array (unsorted, repeated parents) by gathering before a barrier and writing after it.
 *
 * parent: device int32 [B, W] (gr_beam_select's parent_out).  k_unshared, v_unshared: device bf16
 * [B, W, ND, Hkv, d], 16-byte aligned, distinct buffers, modified in place.  Only enqueues on
 * `stream`.  Supported: W <= 2048; B <= 65535; Hkv*d a multiple of 8.  Errors: INVALID_ARG,
 * UNSUPPORTED, HIP.
 * ------------------------------------------------------------------------------------------------ */
gr_status gr_beam_reorder(int32_t B, int32_t W, int32_t ND, int32_t Hkv, int32_t d, int32_t u,
                          const int32_t* parent, void* k_unshared, void* v_unshared, void* stream);

/* ------------------------------------------------------------------------------------------------
 * gr_beam_slot_update / gr_beam_attn_slots - the same hand-over of the unshared cache between decode steps
 * (Section 5.1) without moving any cache bytes.
 *
 * The paper moves each surviving beam's rows to its new place.  Here the rows stay where they were written and a
 * slot table follows the beams instead: token t of beam w of request b is read from row slot[b, w, t] of that
 * request's [W * ND] rows of k_unshared / v_unshared (the same [B, W, ND, Hkv, d] buffers, seen as B blocks of
 * W * ND rows).  A row is written once - the caller writes the K/V of beam j's token t to row j * ND + t, as for
 * gr_beam_attn - and never overwritten afterwards, because position t only ever receives tokens of step t.
 *
 * gr_beam_slot_update: slot_out[b, j, t] = slot_in[b, parent[b, j], t] for t < u (the tokens the new beam shares
 *   with its parent); = j * ND + t for t >= u (its own rows, where the next tokens go) and for every t of a dead
 *   slot (parent outside [0, W)).  slot_in == NULL means the identity table (before the first beam step).  parent:
 *   device int32 [B, W]; slot_in, slot_out: device int32 [B, W, ND], distinct.  u = tokens per beam before the
 *   step that produced `parent`, 0 <= u <= ND.
 * gr_beam_attn_slots: gr_beam_attn with `slot` (device int32 [B, W, ND], required) applied to every read of
 *   k_unshared / v_unshared; an entry outside [0, W * ND) is read as the identity entry instead of being followed.
 *   Same parameters, workspace, launch rule and results as gr_beam_attn on a cache reordered by gr_beam_reorder
 *   (bit for bit for live beams).
 * Both only enqueue on `stream`.  Errors: INVALID_ARG, UNSUPPORTED, WORKSPACE_TOO_SMALL, HIP.
 * ------------------------------------------------------------------------------------------------ */
gr_status gr_beam_slot_update(int32_t B, int32_t W, int32_t ND, int32_t u, const int32_t* parent, const int32_t* slot_in,
                              int32_t* slot_out, void* stream);
gr_status gr_beam_attn_slots(const gr_attn_params* p, const int32_t* slot, void* workspace, size_t workspace_bytes, void* stream);

/* ------------------------------------------------------------------------------------------------
 * gr_qk_norm_rope - queries and keys of T rows on their way from a projection to attention: every head normed by itself and rotated by the row's position.
 *     y = x * w / sqrt(mean(x^2) + eps)                                 (q_weight, k_weight; NULL: y = x)
 *     y_a' = y_a cos - y_b sin,  y_b' = y_b cos + y_a sin               for i < rot / 2, (a, b) = (i, i + rot / 2), or with pairs = 1 (2 i, 2 i + 1)
 * with cos = table[pos, i], sin = table[pos, rot / 2 + i]; elements from rot on are not rotated.  In fp32, rounded to bf16 once (so with eps = 0 a mean square
 * has to be at least 2^-126, and a sum of squares below 2^128: of a larger one the finite elements come back as 0).  Before that every operation is rounded to nearest by itself: the sum of the
 * squares (neighbours first: where d and rot are powers of two fours in a chain, of d up to 64 in pairs, then pairs of neighbouring sums), times 1 / d, plus eps, the reciprocal root, x times that,
 * times w; two products, their difference or sum.  Rows lie any strides apart: parts of a fused
 * projection's rows, and the beams' own caches (a row's KV heads at k_unshared + ((b * W + w) * ND + token) * Hkv * d: a stride of ND * Hkv * d).  Queries or keys may be absent (NULL
 * with their output).  v, which is only moved to v_out beside the keys, is for such caches and may be absent too.  With rot > 0 rows whose position is outside [0, n_pos) are left as they
 * were in all outputs.  q_out is q itself (same stride), or does not overlap any input; so is k_out with k; v_out overlaps nothing (an output that begins where another tensor does is refused).
 * Only enqueues on `stream`.  Supported: d a multiple of 16 up to 256; rot a multiple of 16 up to d (0: no rotation; pos and table are not looked at); Hq * d and Hkv * d at most
 * 2^20; strides multiples of 8; T < 2^31.  All tensors but pos 16-byte aligned.  Errors: INVALID_ARG, UNSUPPORTED, HIP.
 * ------------------------------------------------------------------------------------------------ */
typedef struct {
  int64_t T;                      /* rows                                                              */
  int32_t Hq, Hkv, d;
  int32_t rot;                    /* leading elements of a head that are rotated                       */
  int32_t pairs;                  /* 0: element i with i + rot / 2; 1: element 2 i with 2 i + 1        */
  int32_t n_pos;                  /* rows of table                                                     */
  float   eps;                    /* at least 0                                                        */
  int64_t q_stride, k_stride, v_stride;                 /* elements from a row to the next             */
  int64_t q_out_stride, k_out_stride, v_out_stride;
  const void*    q;               /* bf16, Hq * d elements a row, or NULL                              */
  const void*    k;               /* bf16, Hkv * d elements a row, or NULL                             */
  const void*    v;               /* bf16, Hkv * d elements a row, or NULL                             */
  const float*   q_weight;        /* fp32 [d] or NULL                                                  */
  const float*   k_weight;        /* fp32 [d] or NULL                                                  */
  const float*   table;           /* fp32 [n_pos, rot]                                                 */
  const int32_t* pos;             /* int32 [T]                                                         */
  void*          q_out;           /* bf16                                                              */
  void*          k_out;
  void*          v_out;
} gr_qk_norm_rope_params;
gr_status gr_qk_norm_rope(const gr_qk_norm_rope_params* p, void* stream);

/* ------------------------------------------------------------------------------------------------
 * A prompt cache in pages.  gr_beam_attn reads a prompt cache that is packed for one batch.  A server whose requests come and go keeps the
 * prompts in pages of a pool instead, and a prefix that all of them share (an instruction, a context) once:
 *   gr_page_map          pages are handed out of a free list for the new tokens of every request; block tables and slot map
 *   gr_page_write        K/V rows of new tokens (as prefill produced them) into their slots, in bf16 or as FP8 codes
 *   gr_page_append       the same for keys that are not yet normed and rotated, and for pages in FP4
 *   gr_page_read         rows of pages back into a packed cache
 *   gr_beam_attn_paged   the decode step's attention over such pages
 * A pool is [n_pages, page_size, Hkv, d] for K and the same for V; page_size is a power of two from 16 to 1024.  Slot s of a pool is
 * token s % page_size of page s / page_size.  Token t of request b lies in page block_table[b, t / page_size].
 * ------------------------------------------------------------------------------------------------ */
enum {
  GR_KV_BF16 = 0,
  GR_KV_FP8 = 1,                  /* OCP FP8 E4M3 codes, uint8; the value of an element is code * scale, one scale per tensor */
  GR_KV_FP4 = 2                   /* OCP MXFP4: E2M1 codes, a power of two as the scale of every 32; gr_page_append, gr_page_read, gr_beam_attn_paged */
};

/* Pools of GR_KV_FP4 are uint8 [n_pages, Hkv, gr_kv_fp4_page_bytes(page_size, d)], d a multiple of 32.  For a page and KV head they hold page_size rows of d / 2 bytes, element
 * 2 i of a token in the low half of byte i, and behind them page_size rows of d / 32 bytes: element e's value is its code's (0, 0.5, 1, 1.5, 2, 3, 4, 6 and their negatives)
 * times 2^(s - 127) with s the byte of block e / 32.  Written are s from 7 to 252, and 255 for a block that an infinite value or NaN is in: all of it is NaN. */
size_t gr_kv_fp4_page_bytes(int32_t page_size, int32_t d);       /* host only; 0 for sizes that are not supported */

/* gr_page_map - request b has seq_lens[b] tokens in its pages and gets new_lens[b] more (negative lengths count as 0).  Where its last page is full
 * (or it has none) it gets fresh pages, free_pages[0], free_pages[1], ... in the order of the requests, which are written into its row of
 * block_table from entry ceil(seq_lens[b] / page_size) on; other entries are left as they were.  A request is served whole or not at all: it is
 * not served, gets no pages and keeps its length, if it would need more than max_pages pages, if its new tokens do not fit into the slot map, or
 * if too few pages are left for it (then no request behind it that needs a page is served).
 *   lens_out  tokens after the call
 *   cu_new    exclusive sums of new_lens (they stop at 2^31 - 1); the new tokens of request b are rows cu_new[b] .. cu_new[b+1] - 1
 *   slot      slot of every new token; -1 for tokens of requests that are not served, of a page number outside [0, n_pages), and
 *             behind the last token
 *   taken     {pages taken from the free list, requests with new tokens that were not served}
 * The same inputs give the same tables, so a host that knows the lengths can follow the free list without reading anything back.  Only enqueues on
 * `stream`.  The outputs must not overlap the inputs or each other.  Supported: B <= 4096; max_pages * page_size and n_pages * page_size below 2^31,
 * total_new below 2^31 - 1024.  Errors: INVALID_ARG, UNSUPPORTED, HIP. */
typedef struct {
  int32_t B, page_size;
  int32_t max_pages;              /* entries of a row of block_table                                   */
  int32_t n_free, n_pages;        /* entries of free_pages; pages of the pool                          */
  int64_t total_new;              /* entries of slot (normally the sum of new_lens)                    */
  const int32_t* seq_lens;        /* int32 [B]                                                         */
  const int32_t* new_lens;        /* int32 [B]                                                         */
  const int32_t* free_pages;      /* int32 [n_free]                                                    */
  int32_t*       block_table;     /* int32 [B, max_pages], entries of fresh pages are written          */
  int32_t*       lens_out;        /* int32 [B]                                                         */
  int32_t*       cu_new;          /* int32 [B+1]                                                       */
  int32_t*       slot;            /* int32 [total_new]                                                 */
  int32_t*       taken;           /* int32 [2]                                                         */
} gr_page_map_params;
gr_status gr_page_map(const gr_page_map_params* p, void* stream);

/* gr_page_write - row t of k and v (Hkv * d elements, rows k_stride and v_stride elements apart: they may be parts of a fused projection's rows) goes to slot
 * slot[t] of the pools.  Rows whose slot is outside [0, n_pages * page_size) are not written; a slot that two rows have holds either's
 * elements, in parts too.  The pools do not overlap k, v or each other.  GR_KV_FP8: code = the E4M3 value nearest to x / scale (ties to even; the division is rounded to fp32 first), values beyond
 * +-448 saturate, NaN stays NaN.  Only enqueues on `stream`.  Supported: Hkv * d (at most 2^20) and the strides multiples of 8; T and
 * n_pages * page_size below 2^31.  k, v and the pools 16-byte aligned.  Errors: INVALID_ARG, UNSUPPORTED, HIP. */
typedef struct {
  int64_t T;                      /* rows                                                              */
  int32_t Hkv, d, page_size, n_pages;
  int32_t kv_type;                /* GR_KV_*: element type of the pools                                */
  float   k_scale, v_scale;       /* GR_KV_FP8: positive and finite                                    */
  int64_t k_stride, v_stride;     /* elements from a row to the next, at least Hkv * d                 */
  const void*    k;               /* bf16                                                              */
  const void*    v;               /* bf16                                                              */
  const int32_t* slot;            /* int32 [T]                                                         */
  void*          k_pages;         /* bf16 or uint8 [n_pages, page_size, Hkv, d]                        */
  void*          v_pages;
} gr_page_write_params;
gr_status gr_page_write(const gr_page_write_params* p, void* stream);

/* gr_page_append - gr_page_write for the rows of a projection: the keys are normed and rotated on the way, as gr_qk_norm_rope does it (k_weight NULL: not normed; rot 0: not
 * rotated), in fp32 and rounded once, to the pool's type.  Values go as they are.  Rows whose slot is outside [0, n_pages * page_size) or, with rot > 0, whose position is outside
 * [0, n_pos) are not written; a slot that two rows have holds either's elements, in parts too (GR_KV_FP4: codes of one may stand under scales of the other).  GR_KV_FP8: codes as gr_page_write makes them (of rotated or normed keys the quotient
 * may be one unit of fp32 off the division's).  GR_KV_FP4: a block's scale is the smallest power of two, from 2^-120 to 2^125, with |x| <= 7 * scale for its 32 values (no value is
 * further off than half the distance of the codes around it), and 2^125 where a finite one is above 7 * 2^125 (all of those become 6 * 2^125, up to two steps off); codes are the nearest, ties to even, to the values in fp32 (of normed or rotated keys, whose exact values may lie a few units of
 * fp32 away, on the other side of the border between two codes).  Only enqueues on `stream`.  The pools do not overlap k, v or each other.
 * Supported: d a multiple of 16 (GR_KV_FP4: 32) up to 256; rot a multiple of 16 up to d; Hkv * d at most 2^20; the strides multiples of 8; T and n_pages * page_size below
 * 2^31.  k, v, the pools, k_weight and table 16-byte aligned.  Errors: INVALID_ARG, UNSUPPORTED, HIP. */
typedef struct {
  int64_t T;                      /* rows                                                              */
  int32_t Hkv, d, page_size, n_pages;
  int32_t kv_type;                /* GR_KV_*: element type of the pools                                */
  int32_t rot, pairs, n_pos;      /* as for gr_qk_norm_rope                                            */
  float   eps;
  float   k_scale, v_scale;       /* GR_KV_FP8: positive and finite                                    */
  int64_t k_stride, v_stride;     /* elements from a row to the next, at least Hkv * d                 */
  const void*    k;               /* bf16                                                              */
  const void*    v;               /* bf16                                                              */
  const int32_t* slot;            /* int32 [T]                                                         */
  const int32_t* pos;             /* int32 [T]; may be NULL when rot == 0                              */
  const float*   table;           /* fp32 [n_pos, rot]; may be NULL when rot == 0                      */
  const float*   k_weight;        /* fp32 [d] or NULL                                                  */
  void*          k_pages;         /* as gr_page_write's, or GR_KV_FP4's                                */
  void*          v_pages;
} gr_page_append_params;
gr_status gr_page_append(const gr_page_append_params* p, void* stream);

/* gr_page_read - the rows in the slots slot[t] of the pools as bf16 rows t of k and v (k_stride and v_stride elements apart), packed as gr_beam_attn and gr_prefill_attn take them.
 * The value of a code (times its scale, in fp32) is rounded to bf16; of FP4 it is exact for the scales that are written.  Rows whose slot is outside [0, n_pages * page_size) are left
 * as they were.  k and v do not overlap the pools or each other.  Only enqueues on `stream`.  Supported: as for gr_page_append.  Errors: INVALID_ARG, UNSUPPORTED, HIP. */
typedef struct {
  int64_t T;                      /* rows                                                              */
  int32_t Hkv, d, page_size, n_pages;
  int32_t kv_type;                /* GR_KV_*: element type of the pools                                */
  float   k_scale, v_scale;       /* GR_KV_FP8: positive and finite                                    */
  int64_t k_stride, v_stride;     /* elements from a row to the next, at least Hkv * d                 */
  const void*    k_pages;
  const void*    v_pages;
  const int32_t* slot;            /* int32 [T]                                                         */
  void*          k;               /* bf16                                                              */
  void*          v;               /* bf16                                                              */
} gr_page_read_params;
gr_status gr_page_read(const gr_page_read_params* p, void* stream);

/* gr_beam_attn_paged - gr_beam_attn over a prompt cache in pages.  The keys of beam w of request b are, in this order, the prefix_L tokens that all
 * requests share (pages prefix_pages[0], prefix_pages[1], ...), the request's own seq_lens[b] tokens (pages block_table[b, 0], ...), and
 * the beam's own u tokens, as for gr_beam_attn (with `slot` as for gr_beam_attn_slots, or NULL).  Any part may be empty; a beam
 * without a single key gets out = 0 and lse = -inf.  Where a request has at most 80 rows of a KV head (W * Hq/Hkv) and the launch rule estimates that it pays, the
 * prefix is read and multiplied once for the rows of all requests; with more, each request's rows meet it by themselves.
 * What a table holds beyond a request's pages is of no effect; a page number outside [0, n_pages) is read as page 0, and a length outside [0, max_L] as the
 * nearer end.  Slots of a page behind a request's last token may hold anything.
 * GR_KV_FP8: pools of E4M3 codes, scales applied as in gr_beam_attn_fp8kv.  GR_KV_FP4: codes are widened with their blocks' scales to bf16, exactly (scale bytes 7 to 252).
 * A block with the scale byte 255 (gr_page_append made it of an infinite value or NaN) is no finite value: of a row with such a key or value any result may come, finite ones too, and not
 * always NaN; gr_page_read shows such blocks.
 * Supported: d in {64, 128}; Hq % Hkv == 0; 0 <= u <= ND; prefix_L a multiple of page_size; n_pages * page_size below 2^31, and that times
 * Hkv * d below 2^41; prefix_L + max_L below 2^30; Hkv * d <= 65536; W * Hq/Hkv < 2^22.  bf16 tensors and pools 16-byte aligned; finite values in the slots that are read; |v| * 2^8 * (number of keys) below 2^128.
 * Workspace (device, 256-byte aligned, contents unspecified before and after): partial results of segments, where a row's keys are split.
 * Errors: INVALID_ARG, UNSUPPORTED, WORKSPACE_TOO_SMALL, HIP. */
typedef struct {
  int32_t B, W, Hq, Hkv, d;
  int32_t ND, u;                  /* own-token capacity of a beam, and valid own tokens                */
  int32_t page_size, max_pages, n_pages;
  int32_t prefix_L;               /* tokens of the shared prefix                                       */
  int32_t max_L;                  /* max_b seq_lens[b] or more; at most max_pages * page_size           */
  int32_t kv_type;                /* GR_KV_*: element type of the pools                                */
  float   sm_scale;               /* positive and finite                                               */
  float   k_scale, v_scale;       /* GR_KV_FP8: positive and finite                                    */
  const void*    q;               /* bf16 [B, W, Hq, d]                                                */
  const void*    k_pages;         /* bf16 or uint8 [n_pages, page_size, Hkv, d], or GR_KV_FP4's pools  */
  const void*    v_pages;
  const int32_t* prefix_pages;    /* int32 [prefix_L / page_size]; may be NULL when prefix_L == 0      */
  const int32_t* block_table;     /* int32 [B, max_pages]; may be NULL when max_L == 0                 */
  const int32_t* seq_lens;        /* int32 [B]; may be NULL when max_L == 0                            */
  const void*    k_unshared;      /* bf16 [B, W, ND, Hkv, d]; may be NULL when u == 0                  */
  const void*    v_unshared;
  const int32_t* slot;            /* int32 [B, W, ND] or NULL                                          */
  void*          out;             /* bf16 [B, W, Hq, d]                                                */
  float*         lse_out;         /* fp32 [B, W, Hq] or NULL                                           */
} gr_attn_paged_params;

/* Bytes of workspace for these shapes; pointers, scales, u and ND are not looked at (0 is possible).  Host only.  The number is of this max_L and prefix_L and no bound for
 * smaller ones: a shorter list may be cut into more segments.  max_L may be larger than any of seq_lens, so a program with one workspace passes its
 * largest with every call (the lengths themselves are read on the GPU), or asks again for each. */
size_t gr_beam_attn_paged_workspace_bytes(const gr_attn_paged_params* p);
gr_status gr_beam_attn_paged(const gr_attn_paged_params* p, void* workspace, size_t workspace_bytes, void* stream);

/* ------------------------------------------------------------------------------------------------
 * gr_logits_adjust - penalties, biases and masks on the logits of an item step, in front of gr_beam_select.
 *
 * For every live beam w of request b (scores[b, w] > -inf; every beam where scores is NULL) and token v, with x = logits[b, w, v]:
 *     c  = number of rows h of the request's history with h[t] == prefix[b, w, t] for t < step and h[step] == v
 *          (items that the user has seen and that this token would continue; with depth = 1, step = 0: how often the token occurred)
 *     y  = c > 0 ? (x > 0 ? x / repetition[b] : x * repetition[b]) - (frequency[b] * c + presence[b]) : x
 *     y += bias[b, v]
 *     y  = -inf where the mask row of the beam has bit v clear, whatever x was
 * in fp32.  Rows of dead beams are left as they are (in a new tensor: as the memory was; gr_beam_select does not look at them).  `out` is `logits` itself (in place; rows without a bias or a mask are then changed at the counted
 * tokens alone) or does not overlap it.  Any of the parts may be absent (NULL).  repetition is positive.  History rows whose
 * token lies outside [0, V) count nothing.
 * Supported: 1 <= V <= 32768; depth <= 8; n_history < 2^28.  Only enqueues on `stream`.  Errors: INVALID_ARG, UNSUPPORTED, HIP.
 * ------------------------------------------------------------------------------------------------ */
typedef struct {
  int32_t B, W, V, depth, step;   /* 0 <= step < depth                                                 */
  int32_t n_history;              /* rows of history                                                   */
  int32_t bias_rows;              /* 1: one bias for all requests; B: one for each                     */
  int32_t n_allowed;              /* rows of allowed                                                   */
  const float*    logits;         /* fp32 [B, W, V]                                                    */
  float*          out;            /* fp32 [B, W, V]                                                    */
  const float*    scores;         /* fp32 [B, W] or NULL                                               */
  const int32_t*  prefix;         /* int32 [B, W, depth]; needed with a history when step > 0          */
  const int32_t*  history;        /* int32 [n_history, depth]                                          */
  const int32_t*  cu_history;     /* int32 [B+1]: request b owns rows cu[b] .. cu[b+1] - 1             */
  const float*    repetition;     /* fp32 [B] or NULL (1)                                              */
  const float*    frequency;      /* fp32 [B] or NULL (0)                                              */
  const float*    presence;       /* fp32 [B] or NULL (0)                                              */
  const float*    bias;           /* fp32 [bias_rows, V] or NULL                                       */
  const uint32_t* allowed;        /* [n_allowed, ceil(V / 32)] or NULL; bit v % 32 of word v / 32      */
  const int32_t*  allowed_row;    /* int32 [B, W] row of allowed for each beam (outside [0, n_allowed): nothing is forbidden), or NULL (row 0) */
} gr_logits_adjust_params;
gr_status gr_logits_adjust(const gr_logits_adjust_params* p, void* stream);

/* ------------------------------------------------------------------------------------------------
 * Diagnostics: the rates this GPU really sustains, reported by the benchmark next to the datasheet peaks
 * (the evaluation quotes achieved rates against the hardware's capability; Section 9.4).  Not part of the
 * decode path.  Both only enqueue on `stream`.
 *
 * gr_diag_stream_read: reads `bytes` (>= 1 MiB, 16-byte aligned device memory; whole 32 KiB slices are read)
 *   with 16-byte loads and discards them; `sink` is 4 writable device bytes.
 * gr_diag_mfma_loop: `workgroups` x 8 wavefronts each issue `iters` x 4 back-to-back bf16 32x32x16 MFMAs on the
 *   operands found at `operands` (16 KiB of device memory: 2 x 512 x 16 bytes of bf16); `sink` is 4 writable
 *   device bytes.  gr_diag_mfma_flops gives the floating-point operations of such a launch (host only).
 * gr_diag_attn_plan: host only, process-wide.  Makes every later gr_beam_attn / gr_beam_attn_workspace_bytes use
 *   workgroups of `rows_per_workgroup` (128 or 256) query rows and `l_segments` (1..16, lowered to the number of
 *   K/V tiles in the longest prompt) prompt segments instead of the built-in launch rule; (0, 0) restores the rule.
 *   For sweeps that refit the rule; not thread-safe against concurrent gr_beam_attn calls.
 * gr_diag_attn_paged_plan: host only.  How gr_beam_attn_paged launches a call of these shapes (of what gr_beam_attn_paged_workspace_bytes looks at), as five
 *   numbers in host memory: query rows of a workgroup that meets requests' own lists (32, 128 or 256; GR_KV_FP4 also 16), segments of the prefix where the rows of all requests
 *   meet it together (0: every row walks its whole list), segments of a list, sets of wavefronts of a workgroup (1 or 2), and 1 where workgroups look for
 *   the longest request first.  For tests that have to reach every kernel.
 * gr_diag_issue_loop: the issue test behind the attention kernel's roofline discussion.  `workgroups` x 8 wavefronts
 *   (256 workgroups = two wavefronts per SIMD, 512 = four) each run `iters` x 4 slots of { one bf16 32x32x16 MFMA if
 *   `with_mfma`, `n_fma` independent fp32 FMAs, `n_exp` v_exp_f32 }.  Built combinations (n_fma, n_exp): (0,0) (2,0)
 *   (4,0) (8,0) (12,0) (0,1) (2,1) (3,1) (4,1) (4,2) (0,4); others return UNSUPPORTED.  Operands and sink as for
 *   gr_diag_mfma_loop.
 * gr_diag_issue_loop_lds: the same test with the MFMA's first operand coming from LDS, as the attention loop's K and V
 *   operands do: `rounds` x 12 slots per wavefront; every `lds_every`-th slot (0 = never, 1, 2) uses an operand that a
 *   conflict-free ds_read_b128 fetched three slots earlier.  Built (n_fma, n_exp, lds_every): (0,0,*) (3,1,*) (5,0,0)
 *   (5,0,1) (0,2,0) (0,2,1).  Uses 64 KiB of LDS per workgroup.
 * Errors: INVALID_ARG, UNSUPPORTED, HIP.
 * ------------------------------------------------------------------------------------------------ */
gr_status gr_diag_issue_loop(const void* operands, int32_t workgroups, int32_t iters, int32_t n_fma, int32_t n_exp,
                             int32_t with_mfma, void* sink, void* stream);
gr_status gr_diag_issue_loop_lds(const void* operands, int32_t workgroups, int32_t rounds, int32_t n_fma, int32_t n_exp,
                                 int32_t lds_every, void* sink, void* stream);
gr_status gr_diag_attn_plan(int32_t rows_per_workgroup, int32_t l_segments);
gr_status gr_diag_attn_paged_plan(const gr_attn_paged_params* p, int32_t* plan);
gr_status gr_diag_stream_read(const void* src, size_t bytes, void* sink, void* stream);
gr_status gr_diag_mfma_loop(const void* operands, int32_t workgroups, int32_t iters, void* sink, void* stream);
double    gr_diag_mfma_flops(int32_t workgroups, int32_t iters);

#ifdef __cplusplus
}
#endif
#endif /* GR_H_ */

/*
 * lg_paged.h -- the paged form of the guarded cache: chunks of new tokens, and pages that sequences
 * share, copy and give back.
 *
 * lg_layer_cache (lg.h) gives every sequence of a batch the same number of slots. Here the slots of
 * a sequence lie in pages of a pool, so a batch of unequal budgets holds what its live slots need,
 * a common prompt is held once, and what a prune frees serves the next sequence. One step over a
 * batch, whose sequences each bring any number of new tokens (a prompt or a piece of it, one token
 * to decode, or none), is, on one HIP stream:
 *
 *   1. lg_page_reserve    once: slots, positions and pages for the new tokens.
 *   2. lg_rope_append     once per layer: rotary positions of the new queries and keys; the keys and
 *                         values are stored to their slots.
 *   3. lg_paged_attend    once per layer: every new token attends over its sequence's slots up to its
 *                         own; lse, suffix mass and conf as in lg_decode_attend.
 *   4. lg_detect_loop     once, as for the contiguous cache (lg.h).
 *   5. lg_prune_compact   once, with n_layers = 0, t_append = NULL and the map's pos and len: the keep
 *                         set, pos and len (the append is committed by lg_page_reserve already).
 *   6. lg_page_compact    once: the flagged sequences' rows move, their other pages are given back.
 *
 * lg_page_fork makes sequences continue others (beams, samples of one prompt) or end.
 *
 * Beside the guard. What belongs to a sequence and is not in the map is the caller's: its row of
 * lg_guard_state, of the token ring, of t, t0, budget, suffix_w and conf.
 *   - lg_page_fork leaves those rows as they are. A sequence that continues another takes the parent's with
 *     it (row b <- row parent[b]); one that begins anew starts from a zeroed state.
 *   - lg_detect_loop takes a step for every sequence of its batch. For one that brought no token in
 *     this step that is one step too many: conf is 0, so its streak ends, and stall and rep count the same
 *     tail once more. Copy its row of the state before step 4 and back behind it, and zero its decision
 *     before step 5 (the length alone then decides about a prune).
 *   - The last token of each piece of a prompt raises conf too: zero conf behind the prompt where it
 *     shall not count.
 *   - LG_POLICY_H2O is not available: lg_paged_attend forms no acc, and step 5 without layers takes all
 *     scores as 0, which keeps the newest slots alone.
 *
 * Conventions are those of lg.h: caller-owned device memory, no allocation, no synchronisation, host
 * checks before anything is enqueued, device-side values clamped into the buffers. Calls keep no
 * state but in the arrays they are given; a workspace is written before it is read in every call, so
 * it needs no initialisation, and calls that do not overlap in time may share one (captured graphs
 * too). Everything runs on the current device.
 *
 * The map. `table[b][c]` is the page of slots [c page_size, (c + 1) page_size) of sequence b, or -1.
 * `ref[p]` counts the table entries that name page p: 0 is a free page. Live slots 0..len[b]-1 hold
 * strictly increasing positions, as in lg.h, from 0 up and below 2^31 - 1; the columns below
 * ceil(len[b] / page_size) name pages and the others are -1. An empty map is table = -1, len = 0,
 * ref = 0. All calls here keep this, and ask for it: other values (a page number outside the pool,
 * say) give unspecified results for the sequences that hold them, without any access outside the
 * buffers. A caller may hold pages back by counting them once more in ref. Pages are taken in
 * ascending order of their number, for the sequences in ascending order, so every result is a
 * function of the inputs alone.
 *
 * When pages run out. A call that takes pages meets the sequences' needs in order, up to the first
 * that what is free does not cover; that sequence and every later one that needs any page is
 * refused: it stays exactly as it was, the others are served.
 */
#ifndef LG_PAGED_H
#define LG_PAGED_H

#include "lg.h"

#ifdef __cplusplus
extern "C" {
#endif

/* The sequences' view of the pool, common to all layers.
 *   table [batch][max_pages], pos [batch][max_pages * page_size], len [batch], ref [n_pages]: int32.
 * page_size is 16, 32, 64, 128 or 256 (LG_ERR_UNSUPPORTED); max_pages * page_size <= 2^30;
 * batch * max_pages < 2^31; batch <= 65535; n_pages <= 2^28 (LG_ERR_SHAPE). ref is 16-byte aligned
 * (LG_ERR_ALIGN). */
typedef struct {
  int32_t batch, max_pages, n_pages, page_size;
  int32_t *table, *pos, *len, *ref;
} lg_page_map;

/* One layer's pages: k, v [n_pages][n_kv_heads][page_size][head_dim] of dtype. Supported sizes and
 * types as in lg_layer_cache; n_pages and page_size as in the map (LG_ERR_SHAPE). lg_page_reserve and lg_page_compact
 * also take layers of LG_FP4 (lg_fp4.h). */
typedef struct {
  int32_t n_pages, page_size, n_q_heads, n_kv_heads, head_dim;
  lg_dtype dtype;
  void *k, *v;
} lg_paged_layer;

/* Workspace bytes of the lg_page_* calls on this map (0 for an invalid map); 16-byte aligned. */
size_t lg_page_workspace(const lg_page_map* map);

/* lg_page_reserve -- slots, positions and pages for a step's new tokens.
 *
 * Sequence b brings n = q_start[b + 1] - q_start[b] tokens (rows q_start[b] .. of the step's token
 * arrays), the newest at position t[b], the others just before it. When it is served,
 *   base[b] = len[b] (the slot of its first new token), pos of the new slots = t[b] - n + 1 + i,
 *   len[b] += n, and the table has a page for every new slot.
 * A last page that holds live slots, will take new ones and is shared (ref > 1) is replaced by a page
 * of its own with its live rows copied, in every layer given; the shared one loses this reference.
 * A sequence is refused when pages run out (see above) or n exceeds its columns: base[b] = -1, and
 * the calls that take base leave its rows alone. With n = 0, base[b] = len[b]. The first new position,
 * t[b] - n + 1, is the caller's to have at 0 or above and behind the last live one (see the map).
 *   layers       host array of n_layers views (0: the map alone; then the caller copies rows of pages).
 *                All have the same sizes and type (LG_ERR_SHAPE), and no pages in common.
 *   q_start      [batch + 1] int32, ascending.
 *   t            [batch] int32, newest position of each sequence after the step.
 *   base         [batch] int32 output. */
lg_status lg_page_reserve(const lg_page_map* map, int32_t n_layers, const lg_paged_layer* layers,
                          const int32_t* q_start, const int32_t* t, int32_t* base, void* workspace,
                          size_t workspace_bytes, hipStream_t stream);

/* lg_page_fork -- every sequence becomes what sequence parent[b] was before the call: len, the
 * positions of its live slots, and its pages, which both then share. parent[b] = b (or any value
 * outside [-1, batch)) leaves it as it is; -1 ends it (len = 0). References that the old contents held
 * are given back. No page is taken and no row moves. A permutation reorders the batch. */
lg_status lg_page_fork(const lg_page_map* map, const int32_t* parent, void* workspace,
                       size_t workspace_bytes, hipStream_t stream);

/* lg_page_compact -- moves the rows of pruned sequences to the front of their pages.
 *
 * For every sequence with new_len[b] >= 0 (as lg_prune_compact leaves new_len and keep_idx; it has
 * updated the map's pos and len already): rows r <- keep_idx[b][r] for r < new_len[b], in every layer
 * given, K and V; the columns from ceil(new_len[b] / page_size) on are given back. keep_idx ascends
 * (keep_idx[b][r] >= r). Pages before the first row that moves stay as they are, shared or not. Of the
 * others, a shared one (ref > 1 at the call) is replaced by a page of its own, and the rest is
 * rewritten in place.
 *   moved [batch] int32 output: 1 moved, 0 not flagged, -1 refused (the pages for its replacements
 *         are not there). A refused sequence's table, pages and references are as before while its
 *         pos and len say what they will hold: free pages and repeat the call, with new_len = -1 for
 *         the sequences that have moved, or end it (lg_page_fork), before it
 *         attends again: until then its positions name other rows than its pages hold.
 *   keep_idx [batch][max_pages * page_size], new_len [batch] int32. */
lg_status lg_page_compact(const lg_page_map* map, int32_t n_layers, const lg_paged_layer* layers,
                          const int32_t* keep_idx, const int32_t* new_len, int32_t* moved,
                          void* workspace, size_t workspace_bytes, hipStream_t stream);

/* Rotary frequencies (host): inv_freq[i], i < rot_dim / 2, for lg_rope_append, computed in double.
 * With f_i = theta^(-2 i / rot_dim):
 *   LG_ROPE_PLAIN    f_i.
 *   LG_ROPE_LINEAR   f_i / factor (positions interpolated).
 *   LG_ROPE_BASE     the base raised to theta factor^(rot_dim / (rot_dim - 2)): the slowest frequency
 *                    is divided by factor, the fastest stays (rot_dim >= 4).
 *   LG_ROPE_RAMP     f_i where a frequency turns more than fast times within original_context tokens,
 *                    f_i / factor where less than slow times, and between them linear in the index i
 *                    (its ends rounded outwards to whole indices); *scale = 1 + 0.1 ln(factor).
 *   LG_ROPE_BANDS    the same two regions, and between them linear in the number of turns.
 * *scale (1 but for LG_ROPE_RAMP) multiplies cos and sin. Returns LG_ERR_PARAM for a rot_dim that is
 * odd or outside [2, 128], theta <= 1, factor < 1, or (for the last two) original_context < 1 or
 * not 0 < slow < fast. */
enum { LG_ROPE_PLAIN = 0, LG_ROPE_LINEAR = 1, LG_ROPE_BASE = 2, LG_ROPE_RAMP = 3, LG_ROPE_BANDS = 4 };
typedef struct {
  int32_t kind, rot_dim;
  double theta, factor, original_context, slow, fast;
} lg_rope_params;
lg_status lg_rope_frequencies(const lg_rope_params* p, float* inv_freq, float* scale);

/* lg_rope_append -- rotary positions of a step's queries and keys, and the append of its keys and
 * values, for one layer.
 *
 * Token i of sequence b is row q_start[b] + i of q, k, v; its slot is base[b] + i and its position
 * p = pos[b][slot]. The first rot_dim values of every query and key head are rotated: with
 * a_j = p inv_freq[j], the pair (x, y) becomes scale (x cos a_j - y sin a_j, y cos a_j + x sin a_j),
 * the pair being values (j, j + rot_dim / 2), or (2 j, 2 j + 1) when `interleaved`. The others
 * and all values are kept. q goes to q_out, k and v to the token's row of its page. Angles are
 * reduced in double, the rotation is float32, rounded once. Rows of refused sequences (base < 0)
 * and rows from q_start[batch] on are left as they are.
 *   q, k, v      row r, head h at x + r * stride + h * head_dim, strides in elements (>= heads *
 *                head_dim: LG_ERR_SHAPE); e.g. parts of one projection's rows. k and v may both be NULL
 *                (queries only). Arrays and rows are 16-byte aligned (LG_ERR_ALIGN).
 *   q_out        [total][n_q_heads][head_dim]; may be q itself when that is dense (LG_ERR_PARAM when it
 *                is not), and overlaps none of q, k, v in any other way.
 *   inv_freq     [rot_dim / 2] float32 device array; may be NULL with rot_dim 0 (append alone).
 *   rot_dim      even, 0 <= rot_dim <= head_dim (LG_ERR_PARAM).
 *   total        rows of q, k and v, below 2^23 (LG_ERR_SHAPE); 0 enqueues nothing. */
lg_status lg_rope_append(const lg_paged_layer* layer, const lg_page_map* map, const void* q,
                         int64_t q_stride, const void* k, int64_t k_stride, const void* v,
                         int64_t v_stride, const float* inv_freq, int32_t rot_dim,
                         int32_t interleaved, float scale, void* q_out, const int32_t* q_start,
                         const int32_t* base, int32_t total, hipStream_t stream);

/* Workspace bytes of lg_paged_attend for these sizes (at least 16; 0 when they are invalid). It grows
 * with neither argument shrinking, so the size for the largest step serves every smaller one. */
size_t lg_paged_attend_workspace(const lg_paged_layer* layer, const lg_page_map* map, int32_t total,
                                 int32_t max_chunk);

/* lg_paged_attend -- attention of a step's new tokens over their sequences' pages, for one layer.
 *
 * Token i of sequence b, at slot m = base[b] + i and position p = pos[b][m], sees the slots j <= m
 * with pos_j > p - window or pos_j < n_sink (all of them with window = 0), and
 *   s_j = <q_h, k_j> / sqrt(head_dim),  alpha = softmax over the visible slots,
 *   out_h = sum alpha_j v_j,  lse_h = log sum exp(s_j),
 *   suffix_mass_h = sum of alpha_j over visible slots with pos_j > p - suffix_w[b],
 *   conf[b] = max(conf[b], max_h suffix_mass_h of the sequence's newest token).
 * The step's keys and values are in their pages already (lg_rope_append). What a slot that a token
 * does not see holds (infinities and NaN too) has no effect on that token. A token that sees no slot
 * (its pages are missing) gets out = 0, lse = -inf, suffix_mass = 0. A refused sequence
 * (base[b] < 0) with tokens has conf[b] = NaN, which lg_detect_loop reads as "attend_error"; its
 * rows, and rows from q_start[batch] on, are left as they are.
 *   q, out       [total][n_q_heads][head_dim] dtype, 16-byte aligned; out may not overlap q (LG_ERR_PARAM
 *                for out = q).
 *   max_chunk    the largest number of tokens of a sequence; one that brings more is treated as
 *                refused. total, max_chunk: >= 0; 0 total enqueues nothing. total * n_q_heads < 2^31, and the
 *                workgroups (one for every 128 query rows of a KV head, one for every sequence and KV head,
 *                times the splits) < 2^23 (LG_ERR_SHAPE).
 *   window, n_sink  >= 0 (LG_ERR_PARAM).
 *   suffix_w     [batch] int32 >= 0, or NULL: then suffix_mass and conf must be NULL too. p - suffix_w[b]
 *                and p - window saturate.
 *   lse, suffix_mass [total][n_q_heads] float32; suffix_mass may be NULL; conf [batch] or NULL.
 *   workspace    16-byte aligned (LG_ERR_ALIGN, LG_ERR_WORKSPACE).
 * bfloat16 layers: where a sequence's new tokens have at most 32 query heads of a KV head together (every
 * decode step; n * n_q_heads / n_kv_heads <= 32), alpha multiplies V as two bfloat16 terms, within 2^-16 of
 * it, as in lg_decode_attend; in longer chunks as one bfloat16 (one rounding, at most 2^-8 of it). The sums are
 * float32, and lse and suffix_mass are sums of the float32 weights. An infinity in v whose weight is below
 * 2^-100 of the row's largest gives a token that sees it that infinity or NaN. */
lg_status lg_paged_attend(const lg_paged_layer* layer, const lg_page_map* map, const void* q,
                          void* out, const int32_t* q_start, const int32_t* base, int32_t total,
                          int32_t max_chunk, int32_t window, int32_t n_sink,
                          const int32_t* suffix_w, float* lse, float* suffix_mass, float* conf,
                          void* workspace, size_t workspace_bytes, hipStream_t stream);

#ifdef __cplusplus
}
#endif
#endif /* LG_PAGED_H */

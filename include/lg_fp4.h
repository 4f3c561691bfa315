/*
 * lg_fp4.h -- the paged cache in 4 bits, and rotary positions with several axes.
 *
 * A layer of a paged cache (lg_paged.h) may hold its keys and values as 4-bit numbers: 4.25 bits a value in
 * place of 16 or 32. A step over such a batch is that of lg_paged.h, with
 *   lg_rope_append_axes     in place of lg_rope_append: it rotates, and rounds what it appends to 4 bits;
 *   lg_paged_attend_fp4     in place of lg_paged_attend.
 * lg_page_reserve and lg_page_compact take these layers as they take others (all layers of a call have one type),
 * lg_page_fork needs no layers, and the guard's calls (lg.h) see no difference: the same map and statistics.
 * lg_page_unpack_fp4 reads slots back as values. lg_rope_append and lg_paged_attend refuse these layers
 * (LG_ERR_UNSUPPORTED). lg_rope_append_axes also serves layers of the other types.
 *
 * The numbers. 32 values along a head share an exponent byte x, the unit is u = 2^(x - 127), and a value is a code of
 * four bits: sign s (the highest), two bits of exponent, one of fraction, for 0, 0.5, 1, 1.5, 2, 3, 4 and 6 units. Each is a
 * bfloat16 number exactly. Appending 32 values of largest magnitude m takes the smallest unit with m <= 6 u,
 * within 2^-125 .. 2^125 (x = 2 .. 252), and rounds each value to the nearest code, ties to the code with fraction 0;
 * what lies beyond 6 u (m > 6 2^125 alone) becomes 6 u. So a value moves by at most u / 4 where it is at most 2 u, by u / 2 up
 * to 4 u and by u up to 6 u; u is below m / 3 where m > 3 2^-125. At the ends, a value of a group with m <= 3 2^-125 moves by at
 * most 2^-126 and may become 0, and one beyond 6 2^125 moves by less than 2^126. 32 values of which one is infinite or NaN get
 * x = 255; they, and those of any x above 252, stand for NaN.
 *
 * Layout. lg_paged_layer with dtype LG_FP4: k, v [n_pages][n_kv_heads][page_size (head_dim / 2 + head_dim / 32)]
 * bytes. The block of a page and a head is page_size rows of head_dim / 2 bytes, value 2 i in the low half of byte i
 * and 2 i + 1 in the high half, and behind them page_size rows of head_dim / 32 exponent bytes.
 * n_pages * page_size < 2^32 - 1 (LG_ERR_SHAPE). Conventions, errors and what is caller-owned are as in lg_paged.h.
 */
#ifndef LG_FP4_H
#define LG_FP4_H

#include "lg_paged.h"

#ifdef __cplusplus
extern "C" {
#endif

/* Which axis each pair of a rotated head turns by (host): axis[j], j < rot_dim / 2, where sections[a] pairs
 * turn by axis a and all sections together are rot_dim / 2.
 *   LG_AXES_BLOCKS   the first sections[0] pairs by axis 0, the next by axis 1, ...
 *   LG_AXES_TURNS    the axes take turns while they have pairs left: 0, 1, 2, 0, 1, 2, ...
 * Frequencies are the caller's choice: one ladder over all pairs (lg_rope_frequencies with rot_dim), or in blocks a
 * ladder for each axis (with 2 sections[a], one after the other). Returns LG_ERR_PARAM for n_axes outside 1 .. 8,
 * another order, a negative section, or sections that do not add up to 1 .. 64 pairs. */
enum { LG_AXES_BLOCKS = 0, LG_AXES_TURNS = 1 };
lg_status lg_rope_axes(int32_t n_axes, const int32_t *sections, int32_t order, int32_t *axis);

/* lg_rope_append_axes -- rotary positions of a step's queries and keys on one axis or several, and the append of
 * its keys and values to pages of any type, for one layer.
 *
 * As lg_rope_append, but
 *   - pair j of token i of sequence b, row r = q_start[b] + i, turns by a_j = p inv_freq[j] with p =
 *     coord[axis[j]][r]: the token's place in time, height and width, say. With n_axes = 0, p = pos[b][slot] for all.
 *     Masks and windows go by pos as ever. cos and sin are formed in double, scaled and rounded once to float32; for 4-bit
 *     keys the products with them and their sum are rounded to float32 one by one.
 *   - dtype is the type of q, k, v and q_out (LG_F32 or LG_BF16). A layer of LG_FP4 takes both; keys are rounded to 4 bits
 *     from the float32 rotation, values from what they are. Any other layer takes its own type (LG_ERR_UNSUPPORTED).
 *   - keys and values alone: q and q_out may both be NULL (k and v are then given).
 * A slot is written by its token alone; the others of its page keep their bits.
 *   axis         [rot_dim / 2] int32 device array; values outside 0 .. n_axes - 1 count as the nearest of them.
 *   coord        int32 device array, coord[a] at coord + a * coord_stride, total each; any values.
 *                Both NULL with n_axes = 0 (LG_ERR_PARAM when not).
 *   coord_stride elements, >= total (LG_ERR_SHAPE) where n_axes > 1.
 *   n_axes       0 .. 8 (LG_ERR_PARAM).
 *   the others   as in lg_rope_append. */
lg_status lg_rope_append_axes(const lg_paged_layer *layer, const lg_page_map *map, lg_dtype dtype,
                              const void *q, int64_t q_stride, const void *k, int64_t k_stride,
                              const void *v, int64_t v_stride, const float *inv_freq, int32_t rot_dim,
                              int32_t interleaved, float scale, const int32_t *axis, const int32_t *coord,
                              int64_t coord_stride, int32_t n_axes, void *q_out, const int32_t *q_start,
                              const int32_t *base, int32_t total, hipStream_t stream);

/* lg_page_unpack_fp4 -- the values that slots of a layer of LG_FP4 stand for.
 *
 * Row q_start[b] + i of k_out and v_out becomes what slot base[b] + i of sequence b holds (with base = 0 and the lengths
 * added up in q_start: whole sequences). Rows whose slot lies outside the map or has no page, of sequences with
 * base[b] < 0, and from q_start[batch] on are left as they are. Values are exact in both types.
 *   dtype         LG_F32 or LG_BF16, of k_out and v_out.
 *   k_out, v_out  [total][n_kv_heads][head_dim], 16-byte aligned; one of them may be NULL.
 *   q_start       [batch + 1] int32, ascending; base [batch] int32; total as in lg_rope_append. */
lg_status lg_page_unpack_fp4(const lg_paged_layer *layer, const lg_page_map *map, lg_dtype dtype, void *k_out,
                             void *v_out, const int32_t *q_start, const int32_t *base, int32_t total,
                             hipStream_t stream);

/* Workspace bytes of lg_paged_attend_fp4 (see lg_paged_attend_workspace). */
size_t lg_paged_attend_fp4_workspace(const lg_paged_layer *layer, const lg_page_map *map, lg_dtype dtype,
                                     int32_t total, int32_t max_chunk);

/* lg_paged_attend_fp4 -- lg_paged_attend over a layer of LG_FP4: the same tokens, masks, statistics and arguments,
 * with k_j and v_j the values that the slots stand for and dtype (LG_F32 or LG_BF16) the type of q and out.
 *
 * What a slot that a token does not see holds has no effect on that token. A token that sees a slot whose keys have a
 * group that stands for NaN gets NaN for out and lse; one that sees a slot whose values have one gets NaN in
 * those 32 values of out, whatever the slot's weight.
 *
 * Keys and values are exact as bfloat16, so the matrix products are of bfloat16 numbers with float32 sums: in float32
 * calls q and alpha are sums of three bfloat16 terms each, all of their 24 bits from 2^-110 on and what is not below 2^-133 of
 * smaller ones (which count where keys or values reach 2^100). In bfloat16 calls alpha is two terms (within 2^-16
 * of it) where a sequence's new tokens have at most 32 query heads of a KV head together, and one (within 2^-8) in longer
 * chunks, as in lg_paged_attend. */
lg_status lg_paged_attend_fp4(const lg_paged_layer *layer, const lg_page_map *map, lg_dtype dtype, const void *q,
                              void *out, const int32_t *q_start, const int32_t *base, int32_t total,
                              int32_t max_chunk, int32_t window, int32_t n_sink, const int32_t *suffix_w,
                              float *lse, float *suffix_mass, float *conf, void *workspace,
                              size_t workspace_bytes, hipStream_t stream);

#ifdef __cplusplus
}
#endif
#endif /* LG_FP4_H */

/*
 * tmac_pages.h -- C ABI of a paged cache of keys and values in 8 bits: the rotation of queries and keys by their positions,
 * appending tokens (keys rotated on the way), reading them back, and attention over the pages.
 *
 * General rules are those of tmac.h and tmac_attn.h: the library allocates nothing, device entry points enqueue work on `stream` and
 * never synchronise, arguments are checked on the host before anything is launched.  Contents of device arrays (tables, lengths,
 * starts) cannot be checked there; the kernels clamp them, so that wrong ones give wrong results but no access out of range.
 * Types tmac_view, tmac_elem_t, tmac_attn_desc: tmac_attn.h.
 */
#ifndef TMAC_PAGES_H_
#define TMAC_PAGES_H_

#include "tmac_attn.h"

#ifdef __cplusplus
extern "C" {
#endif

/* --- rotary positions -------------------------------------------------------------------------------------------------------
 * A pair (a, b) of a head's elements at position p turns by p f_i:
 *   a' = a c - b s,  b' = a s + b c,  c = magnitude cos(p f_i),  s = magnitude sin(p f_i)
 * Pair i is elements (i, i + rot / 2), or (2 i, 2 i + 1) where interleaved; elements from rot on stay as they are.  Positions may be
 * negative (the turn back: with -p and 1 / magnitude the rotation's inverse, with -p and magnitude its gradient).  Angles,
 * cosines and sines are taken in 64 bits and rounded to 32, products are 32-bit, results are rounded once.
 *   freq_dev  fp64 [rot / 2], radians a position, 8-byte aligned
 *   D         a multiple of 4, at most 128; rot even, 2 <= rot <= D; magnitude finite */
typedef struct {
  const double* freq_dev;
  double  magnitude;
  int32_t D, rot;
  int32_t interleaved;  /* 0 or 1 */
  int32_t elem;         /* tmac_elem_t */
  int32_t reserved[2];  /* must be 0 */
} tmac_rope;

/* One tensor [T, H, D] by strides (token, head) and where its result goes: x itself (the same data and strides) or memory that does
 * not overlap any x of the call; rows of out do not overlap each other. */
typedef struct {
  tmac_view x, out;
  int32_t H;
  int32_t reserved; /* must be 0 */
} tmac_rope_item;

/* Turns `count` tensors (1 to TMAC_ROPE_MAX) of the same T tokens in one launch.
 *   positions_dev  int64 [T]
 * Errors: TMAC_EINVAL, TMAC_EUNSUPPORTED (D over 128; a launch of 2^32 threads), TMAC_EHIP. */
enum { TMAC_ROPE_MAX = 4 };
tmac_status tmac_rotate(const tmac_rope* rope, const tmac_rope_item* items, int32_t count, const int64_t* positions_dev, int32_t T,
                        void* stream);

/* --- pages --------------------------------------------------------------------------------------------------------------------
 * Keys and values in 8 bits.  TMAC_BLOCK_TOKENS consecutive tokens of a sequence share, for each key head, one scale for their keys
 * and one for their values; an element is its code's value times the scale.
 *   TMAC_CODE_I8    whole numbers -127..127;  the scale that values up to `most` need is most (1 / 127), in 32 bits
 *   TMAC_CODE_E4M3  4 exponent and 3 mantissa bits, up to 448;  most / 448 rounded up to a power of two
 * Scales are at least 2^-60 (a block of zeros has that); code = round to nearest even of x (1 / scale).  Infinite elements are held as
 * the block's largest value of their sign, NaN as zero; neither touches the scale. */
typedef enum { TMAC_CODE_I8 = 0, TMAC_CODE_E4M3 = 1 } tmac_code_t;
enum { TMAC_BLOCK_TOKENS = 32 };

/* Pages of `page` tokens (a power of two, 32 to 4096) of all Hkv key heads.  Unit u = (page * Hkv + head) * (page tokens / 32) + block
 * of the page.  With c = ceil(D / 16):
 *   codes_dev   unit u at byte u * 1024 c (tmac_pages_code_bytes in all, 16-byte aligned): 512 c bytes of keys, [c][32 tokens][16
 *               elements], then 512 c bytes of values: the 16 c elements in runs of 32 (the last may be 16), each run
 *               [2][elements][16 tokens], where token t is in half (t / 4) % 2, at byte 8 (t / 8 % 2) + 4 (t / 16) + t % 4.  (A wavefront
 *               finds the operands of its matrix instructions side by side.)  Elements from D on are zero.
 *   scales_dev  fp32 [units][2]: of keys, of values (tmac_pages_scale_bytes)
 * What is in a page before its first token is written does not matter.
 *   D a multiple of 4, at most 128; at most 2^40 units (more, and D over 128: TMAC_EUNSUPPORTED, and 0 bytes) */
typedef struct {
  void*   codes_dev;
  float*  scales_dev;
  int32_t pages, page, Hkv, D;
  int32_t code;         /* tmac_code_t */
  int32_t reserved[3];  /* must be 0 */
} tmac_pages;
size_t tmac_pages_code_bytes(const tmac_pages* pages);  /* 0 for a description that is refused */
size_t tmac_pages_scale_bytes(const tmac_pages* pages);

/* Sequences and the tokens that a call is about: the last ones of each.
 *   table_dev  int32 [S, width], table_stride entries from row to row: token i of sequence s is in page table[s][i / page].  A number
 *              that is no page (-1) means that there is none: its tokens are not written, nobody sees them, they read as zeros.
 *   lens_dev   int32 [S]: tokens of each sequence, those of this call included
 *   cu_dev     int32 [S + 1]: rows [cu[s], cu[s + 1]) of the call's tensors are the last cu[s + 1] - cu[s] tokens of sequence s, in order; it
 *              starts at 0, ends at T or before (rows behind its end are left as they are) and does not fall.  NULL: one row a sequence (T = S).
 *              Rows before a sequence's first token (more rows than the length) are not written, see nothing and read as zeros.
 *   most       most rows of a sequence, where the caller knows it (more are left out); 0: not known
 * Tokens from width * page on are as on pages that are not there.  Starts and lengths that cannot be give wrong results, within the call's
 * rows and the table's pages. */
typedef struct {
  const int32_t* table_dev;
  int64_t table_stride;
  const int32_t* lens_dev;
  const int32_t* cu_dev;
  int32_t S, width, T, most;
} tmac_pages_batch;

/* Writes the call's tokens into their pages, keys turned by `rope` on the way, and turns the queries of the same tokens.
 *   k, v   [T, Hkv, D] of type elem (token, head strides)
 *   rope   NULL: keys as they are (q and q_out NULL then).  D and elem as in the call
 *   positions_dev  int64 [T], or NULL: a token's place in its sequence
 *   q, q_out       [T, Hq, D], or both NULL; q_out as tmac_rope_item.out
 * A block that the call begins gets the scales that its tokens need, the rest of its codes zero.  A block that was begun before keeps the
 * larger of its scale and that; where it grows, codes that are there are multiplied by old / new and rounded again (in e4m3 nothing
 * but what falls below the scale's smallest numbers changes).  Pages that two sequences of a call share must not be written by
 * both.  Errors: TMAC_EINVAL, TMAC_EUNSUPPORTED (D over 128; T, S or width * page beyond 2^30; a launch of 2^32 threads), TMAC_EHIP. */
tmac_status tmac_pages_append(const tmac_pages* pages, const tmac_pages_batch* batch, int32_t elem, const tmac_view* k, const tmac_view* v,
                              const tmac_rope* rope, const int64_t* positions_dev, const tmac_view* q, const tmac_view* q_out, int32_t Hq,
                              void* stream);

/* The call's tokens as their pages hold them, rounded to elem: k, v [T, Hkv, D] (token, head strides).  Rows from cu[S] on stay as they
 * are.  Errors: as tmac_pages_append. */
tmac_status tmac_pages_read(const tmac_pages* pages, const tmac_pages_batch* batch, int32_t elem, const tmac_view* k, const tmac_view* v,
                            void* stream);

/* Attention of the call's tokens over what is in the pages: row i of sequence s's n rows sees the tokens j <= lens[s] - n + i that are on
 * a page.  Notation and rules of values as in tmac_attn.h; desc->causal is 1.  Products are of the queries in fp16 (a bf16 row is first scaled by
 * a power of two to its range, which is exact down to 2^-38 of its largest element) with codes, which fp16 holds exactly; scores, exponentials,
 * sums and lse are 32-bit.  Exponentials times the scale of the values' block are fp16 in the second product: as the sum of two such numbers for sequences with up to 64 rows
 * of the call a key head (its tokens times Hq / Hkv), off by at most 2^-22 of themselves or 2^-31 of the row's largest; as one for the others, off by at most 2^-11 of themselves
 * or 2^-31 of the largest.  Blocks of values may be any distance apart in size.
 *   q, out    [T, Hq, D] (token, head strides);  lse_dev  fp32 [Hq, T], or NULL
 *   workspace tmac_pages_attend_workspace_bytes(desc, pages, batch), 16-byte aligned, contents arbitrary
 * The order of the sums depends on sizes and lengths only.  Rows from cu[S] on stay as they are.
 * Errors: TMAC_EINVAL, TMAC_EUNSUPPORTED (as tmac_pages_append; T Hq beyond 2^30), TMAC_ESIZE, TMAC_EHIP. */
size_t tmac_pages_attend_workspace_bytes(const tmac_attn_desc* desc, const tmac_pages* pages, const tmac_pages_batch* batch);
tmac_status tmac_pages_attend(const tmac_attn_desc* desc, const tmac_pages* pages, const tmac_pages_batch* batch, const tmac_view* q,
                              const tmac_view* out, float* lse_dev, void* workspace_dev, size_t workspace_bytes, void* stream);

#ifdef __cplusplus
}
#endif
#endif /* TMAC_PAGES_H_ */

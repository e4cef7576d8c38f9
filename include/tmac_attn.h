/*
 * tmac_attn.h -- C ABI of the attention operators that stand between the projections of a decoder block: attention over
 * packed prompts, the attention weight that each key received, caches that keep the heaviest keys, and decode attention
 * over a prefix that a batch shares and such caches.
 *
 * General rules are those of tmac.h: the library allocates nothing, device entry points enqueue work on `stream` and never
 * synchronise, arguments are checked on the host before anything is launched.  Contents of device arrays (sequence
 * starts, lengths) cannot be checked there; the kernels clamp them to the sizes given on the host, so that wrong ones give
 * wrong results but no access out of range.
 *
 * Notation: Hq query heads, Hkv key heads, group = Hq / Hkv; query head h reads key head h / group.  D elements per head.
 *   s_ij  = scale q_i . k_j for the keys j that row i may see
 *   lse_i = log sum_j exp s_ij           (natural logarithm; -inf for a row that sees no key, or none above -inf)
 *   o_i   = sum_j exp(s_ij - lse_i) v_j  (zeros for such a row)
 * Results overlap neither each other's rows nor what a call reads (a cache's own weights apart, which a step adds to).
 * Elements that a row may not see do not touch its result, whatever they hold (NaN and infinities too).  Scores, exponentials,
 * sums and lse are 32-bit; the exponentials are rounded to the inputs' type before they are multiplied with v (an error of
 * the size of the result's own rounding; in fp16, exponentials below 2^-20 of the row's largest are instead off by up to 2^-31 of it, so a
 * row over n keys by up to n 2^-31 of the largest |v| more), o_i is rounded once.  Sums are 32-bit before they are divided by the
 * row's: |v| below 2^90 stays finite whatever the scores.
 */
#ifndef TMAC_ATTN_H_
#define TMAC_ATTN_H_

#include "tmac.h"

#ifdef __cplusplus
extern "C" {
#endif

/* Type of q, k, v and the results. */
typedef enum { TMAC_ELEM_F16 = 0, TMAC_ELEM_BF16 = 1 } tmac_elem_t;

/* Hq a multiple of Hkv; D a multiple of 4, at most 128; scale finite and above zero (usually 1 / sqrt(D)).
 * causal is read by tmac_attn_prompt and tmac_attn_weights only. */
typedef struct {
  int32_t Hq, Hkv, D;
  int32_t elem;      /* tmac_elem_t */
  float   scale;
  int32_t causal;    /* 0 or 1 */
  int32_t reserved[2]; /* must be 0 */
} tmac_attn_desc;

/* A tensor of rows of D consecutive elements, with strides in elements from sequence to sequence, token to token and head to
 * head (those that a call does not speak of are not read).  Data 8-byte aligned, strides multiples of 4 and not negative;
 * tmac_cache_fill moves rows fastest where data are 16-byte aligned and strides and D multiples of 8. */
typedef struct {
  void*   data;
  int64_t seq, token, head;
} tmac_view;

/* Attention over S sequences packed one after the other.
 *   q, out     [Tq, Hq, D] (token, head strides);  k, v  [Tk, Hkv, D]
 *   cu_q_dev, cu_k_dev  int32 [S + 1]: sequence s has queries [cu_q[s], cu_q[s + 1]) and keys [cu_k[s], cu_k[s + 1]); both
 *              start at 0, end at Tq and Tk and do not fall.  Lengths of zero are fine.
 *   causal     with nq queries and nk keys in a sequence, query i sees the keys j <= i + nk - nq (the queries are the last
 *              tokens: a chunk after nk - nq earlier keys; with nk < nq the first queries see none).  Else all nk.
 *   lse_dev    fp32 [Hq, Tq], or NULL
 *   workspace  tmac_attn_prompt_workspace_bytes(desc, S, Tq, Tk) bytes (0: none needed), 16-byte aligned, contents arbitrary
 * Errors: TMAC_EINVAL, TMAC_EUNSUPPORTED (D over 128; Tq Hq beyond 2^31; S, Tq or Tk beyond 2^30; a stride of 128 rows beyond 2^30
 * bytes; a launch of 2^32 threads, which 2^24 short sequences, times key heads, come to), TMAC_ESIZE, TMAC_EHIP. */
size_t tmac_attn_prompt_workspace_bytes(const tmac_attn_desc* desc, int32_t S, int32_t Tq, int32_t Tk);
tmac_status tmac_attn_prompt(const tmac_attn_desc* desc, const tmac_view* q, const tmac_view* k, const tmac_view* v, int32_t S,
                             int32_t Tq, int32_t Tk, const int32_t* cu_q_dev, const int32_t* cu_k_dev, const tmac_view* out,
                             float* lse_dev, void* workspace_dev, size_t workspace_bytes, void* stream);

/* Attention weight that every key of such sequences received, summed over the queries that see it and the query heads of its group:
 *   weight[h, j] = sum over i and the heads of group h of exp(s_ij - lse_i); rows whose lse is -inf give nothing.
 *   lse_dev     fp32 [Hq, Tq] as tmac_attn_prompt writes it (or that of tmac_attn_decode over one shared prefix, transposed)
 *   weight_dev  fp32 [Hkv, Tk], overwritten
 *   workspace   tmac_attn_weights_workspace_bytes(desc, S, Tq, Tk)
 * The order of the sums depends on the sizes only.  Errors: as tmac_attn_prompt's, of q and k. */
size_t tmac_attn_weights_workspace_bytes(const tmac_attn_desc* desc, int32_t S, int32_t Tq, int32_t Tk);
tmac_status tmac_attn_weights(const tmac_attn_desc* desc, const tmac_view* q, const tmac_view* k, const float* lse_dev, int32_t S,
                              int32_t Tq, int32_t Tk, const int32_t* cu_q_dev, const int32_t* cu_k_dev, float* weight_dev,
                              void* workspace_dev, size_t workspace_bytes, void* stream);

/* A cache of keys and values for B sequences: every sequence and key head has `capacity` slots of its own, the first lens of
 * them in use, in any order of their tokens (the position of a slot's token is kept beside it).
 *   k, v        [B, Hkv, capacity, D] by strides (seq, head, token)
 *   weight_dev  fp32  [B, Hkv, capacity]  attention weight that the slot's token has received so far
 *   pos_dev     int32 [B, Hkv, capacity]  its position
 *   lens_dev    int32 [B, Hkv]            slots in use
 *   seen_dev    int32 [B, Hkv]            tokens seen so far, evicted ones included: the next token's position
 *   recent      tokens of the last `recent` positions are evicted only after all others; 0 <= recent <= capacity
 * Eviction takes tokens that are not recent before recent ones, then the lightest first (NaN counts as -inf), then the lowest slot. */
typedef struct {
  tmac_view k, v;
  float*   weight_dev;
  int32_t* pos_dev;
  int32_t* lens_dev;
  int32_t* seen_dev;
  int32_t  B, Hkv, D, capacity, recent;
  int32_t  elem;        /* tmac_elem_t */
  int32_t  reserved[2]; /* must be 0 */
} tmac_cache;

/* Where tmac_cache_fill takes tokens from: packed prompts (cu_dev set, lens_dev NULL) or another cache (cu_dev NULL).
 *   k, v    (seq,) head, token strides;  weight: a view of fp32, head and token strides (and seq); pos: a view of int32 or data NULL:
 *           a token's position is its index in its sequence
 *   cu_dev  int32 [B + 1]: token i of sequence b is token cu[b] + i of the views; their seq strides are not read
 *   lens_dev  int32 [B, Hkv]: token i of sequence b and head h is slot i, i < lens[b, h]
 *   seen_dev  int32 [B, Hkv], or NULL: the number of tokens
 *   total   tokens in all (packed) or slots per sequence and head (cache); no index reaches it */
typedef struct {
  tmac_view k, v, weight, pos;
  const int32_t* cu_dev;
  const int32_t* lens_dev;
  const int32_t* seen_dev;
  int32_t total;
  int32_t reserved; /* must be 0 */
} tmac_cache_source;

/* Fills the cache: of the n tokens of each sequence and head those stay that eviction down to min(n, capacity) leaves, in the
 * order they have in the source, with their weights and positions.  lens = min(n, capacity), seen as above; slots from there on
 * keep what they hold.  The source must not overlap the cache.
 * Errors: TMAC_EINVAL, TMAC_EUNSUPPORTED (D over 128; capacity or total beyond 2^30; a launch of 2^32 threads, that is B Hkv of 2^22
 * caches or 2^24 times 64 slots of theirs; of 2^24, or 2^22 of more than 1024 slots, in tmac_cache_append), TMAC_ESIZE, TMAC_EHIP.
 * workspace: tmac_cache_fill_workspace_bytes(cache) bytes.  Weight views may have any strides that are not negative. */
size_t tmac_cache_fill_workspace_bytes(const tmac_cache* cache);
tmac_status tmac_cache_fill(const tmac_cache* cache, const tmac_cache_source* source, void* workspace_dev, size_t workspace_bytes,
                            void* stream);

/* One token for every sequence and head: into slot lens while there is room (lens grows by one), else into the slot that
 * eviction takes first (the new token counts among the recent ones).  Its position is seen, which grows by one, its weight 0.
 *   k, v  [B, Hkv, D] by strides (seq, head) */
tmac_status tmac_cache_append(const tmac_cache* cache, const tmac_view* k, const tmac_view* v, void* stream);

/* One decode step: row b of q, all heads, over the P keys of a prefix that all B sequences share (read once for all of them; P = 0:
 * none) and the slots in use of its own cache.
 *   q, out     [B, Hq, D] by strides (seq, head);  k0, v0  [P, Hkv, D] by strides (token, head), not read when P is 0
 *   cache      B, Hkv, D and elem as in desc; k, v, lens_dev are read.  capacity 0 with no pointers set: prefix only
 *   lse_dev    fp32 [B, Hq], or NULL
 *   accumulate 1: weight[b, h, j] += sum over the group's heads of exp(s - lse) for the slots in use
 *   workspace  tmac_attn_decode_workspace_bytes(desc, cache, P, accumulate), 16-byte aligned, contents arbitrary
 * Errors: TMAC_EINVAL, TMAC_EUNSUPPORTED (D over 128; P or the capacity beyond 2^30; a stride of 128 rows beyond 2^30 bytes; a launch of 2^32 threads, that is B Hq of
 * 2^26 or as many chunks of slots; accumulate with the lesser of the group and 32 times the capacity beyond 5e8), TMAC_ESIZE, TMAC_EHIP. */
size_t tmac_attn_decode_workspace_bytes(const tmac_attn_desc* desc, const tmac_cache* cache, int32_t P, int32_t accumulate);
tmac_status tmac_attn_decode(const tmac_attn_desc* desc, const tmac_view* q, const tmac_view* k0, const tmac_view* v0, int32_t P,
                             const tmac_cache* cache, int32_t accumulate, const tmac_view* out, float* lse_dev, void* workspace_dev,
                             size_t workspace_bytes, void* stream);

#ifdef __cplusplus
}
#endif
#endif /* TMAC_ATTN_H_ */

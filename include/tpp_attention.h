/*
 * tpp_attention.h -- C ABI of the attention operators of the MI355X (gfx950) TPP library: the norms
 * and the position rotation of query and key heads (forward, backward, and on the way into a cache),
 * attention of one new token per sequence over a paged key-value cache, and the eviction of cached
 * positions by their total attention weight.
 *
 * The paper (Tensor Processing Primitives, arXiv 2104.05755) builds its transformer layers from
 * BRGEMMs, reduces and elementwise TPPs (Sec. 5.1, 5.2.3); these calls are the fused forms of the
 * steps between two BRGEMM calls of such a layer when it is trained or serves tokens one by one.
 *
 * Conventions are those of tpp_brgemm.h: caller-owned DEVICE memory, element counts for strides,
 * asynchronous on `stream` (a hipStream_t as void*, NULL = the default stream), a tpp_status result
 * and tpp_last_error_message() for the detail.  Activations are column-major 2D blocks with a column
 * per token: head h of token t is the D entries at x + t * ld + h * D, as a fully-connected BRGEMM
 * layer writes its features.  Queries, keys and values may be parts of one block (x, x + q_heads * D,
 * ... with one ld).  Arithmetic is fp32; an output is rounded to its type once (to nearest even).
 * The order of every sum depends only on sizes and lists: results do not vary between runs.
 */
#ifndef TPP_ATTENTION_H
#define TPP_ATTENTION_H

#include "tpp_brgemm.h"

#ifdef __cplusplus
extern "C" {
#endif

/* ---- norms of queries and keys with the position rotation ------------------------------------- */

/* Which entries of a head the rotation turns together: i and i + rot_dim / 2, or 2 i and 2 i + 1. */
typedef enum { TPP_ROT_HALVES = 0, TPP_ROT_PAIRS = 1 } tpp_rot_form;

/* For every head x (D entries) of a token at position p, with w the D fp32 norm weights of the
 * queries (wq) or of the keys (wk):
 *     y = x / sqrt(mean(x^2) + eps) * w
 * then each pair (a, b) of y's first rot_dim entries, i < rot_dim / 2, becomes
 *     (a c_i - b s_i,  b c_i + a s_i)
 * with c_i = rot[p * rot_dim + i] and s_i = rot[p * rot_dim + rot_dim / 2 + i], a caller-made fp32
 * table of n_positions rows.  Entries from rot_dim on are not rotated; rot_dim == 0 is the norm alone
 * (rot may be NULL).  A token whose position lies outside [0, n_positions) is padding: its output
 * heads are zeros. */
typedef struct {
  int32_t head_dim;        /* D: 1 .. 512                                        */
  int32_t rot_dim;         /* even, 0 .. D                                       */
  int32_t rot_form;        /* tpp_rot_form                                       */
  int32_t q_heads, k_heads;/* >= 0; pointers of a side without heads may be NULL */
  int32_t dtype;           /* of queries, keys, values, outputs and gradients    */
  float eps;               /* finite, >= 0                                       */
  int64_t n_positions;     /* rows of the rotation table, >= 0                   */
} tpp_qk_desc;

/* Forward.  d_pos: device int64[tokens].  q_out / k_out may be q / k themselves (same ld); otherwise
 * outputs must not overlap inputs.  tokens == 0 is a no-op.
 * Errors: INVALID_ARG for a NULL desc, sizes, flags or leading dimensions (each >= heads * D) out of
 * their ranges, or a NULL pointer when there is work; UNSUPPORTED for D above 512 or more than 2^20
 * heads; HIP if a launch fails. */
tpp_status tpp_qk_norm_rope(const tpp_qk_desc* desc, int64_t tokens, const void* q, int64_t ldq,
                            const void* k, int64_t ldk, const float* wq, const float* wk,
                            const float* rot, const int64_t* d_pos, void* q_out, int64_t ldqo,
                            void* k_out, int64_t ldko, void* stream);

/* Backward: from the forward call's inputs and the gradients gq, gk of its outputs, the gradients dq,
 * dk of its inputs, and dwq, dwk (D floats each, overwritten) of the norm weights, summed over all
 * tokens and heads.  With g the gradient rotated back, xn = x / sqrt(mean(x^2) + eps), u = g * w:
 *     dx = (u - xn * mean(u * xn)) / sqrt(mean(x^2) + eps),    dw = sum g * xn.
 * Padding tokens get zeros and add nothing.  dq / dk may be gq / gk themselves (same ld).  tokens == 0
 * gives dwq = dwk = 0.
 * The weights' partial sums go to a work buffer as tpp_reduce's do (under stream capture to one of
 * the capture's own; where there is none to be had the sums run unsplit).
 * Errors: as tpp_qk_norm_rope, NO_MEMORY if the work buffer cannot be allocated. */
tpp_status tpp_qk_norm_rope_backward(const tpp_qk_desc* desc, int64_t tokens, const void* q,
                                     int64_t ldq, const void* k, int64_t ldk, const float* wq,
                                     const float* wk, const float* rot, const int64_t* d_pos,
                                     const void* gq, int64_t ldgq, const void* gk, int64_t ldgk,
                                     void* dq, int64_t lddq, void* dk, int64_t lddk, float* dwq,
                                     float* dwk, void* stream);

/* ---- the paged cache ---------------------------------------------------------------------------- */

/* Two pools of n_pages pages of page_size positions, for keys and values.  The D entries of head h at
 * place s of page p are contiguous at k (v) + p * page_stride + s * pos_stride + h * head_stride
 * (elements, >= 0), so [page][position][head][D] and [page][head][position][D] are both described.
 * The pages of a sequence are listed in a table row of its own: position t is at place t % page_size
 * of page d_pages[b * ld_pages + t / page_size] (device int64).  An entry outside [0, n_pages) is a
 * page that holds nothing: its positions are masked, and no memory outside the pools is read. */
typedef struct {
  void* k;
  void* v;
  int32_t dtype;
  int32_t head_dim;        /* D */
  int32_t kv_heads;
  int32_t page_size;
  int64_t n_pages;
  int64_t page_stride, pos_stride, head_stride;
} tpp_kv_cache;

/* tpp_qk_norm_rope with the keys written to the cache instead of k_out, and the values v (k_heads
 * heads per token) copied beside them: token t goes to slot d_slot[t] = page * page_size + place
 * (device int64).  A slot outside the pools, or a padding position, writes nothing to the cache.  No
 * two tokens may have the same slot.  D: 1 .. 512; desc and cache must agree on D, k_heads and dtype.
 * Errors: as tpp_qk_norm_rope, plus those of a malformed cache. */
tpp_status tpp_qk_norm_rope_append(const tpp_qk_desc* desc, int64_t tokens, const void* q, int64_t ldq,
                                   const void* k, int64_t ldk, const void* v, int64_t ldv,
                                   const float* wq, const float* wk, const float* rot,
                                   const int64_t* d_pos, void* q_out, int64_t ldqo,
                                   const tpp_kv_cache* cache, const int64_t* d_slot, void* stream);

/* ---- attention of one new token per sequence ---------------------------------------------------- */

/* Query head h reads key head h / (q_heads / kv_heads).  For sequence b with n = d_len[b] positions
 * (cut to [0, max_len]), over its positions t < n that are held by a page and, where window > 0, have
 * t >= n - window:
 *     s_t = scale * (q . k_t),   lse = log sum_t exp(s_t),   p_t = exp(s_t - lse),   out = sum_t p_t v_t
 * A head with no such position gives out = 0 and lse = -inf.  Nothing that is stored at other places
 * (NaN included) has any influence.  An infinity among the values counted gives its entry that infinity
 * (both signs, or a NaN: NaN), since every p_t is positive.  The sum is formed with exp(s_t - max s) and
 * divided last: it has to stay in fp32's range. */
typedef struct {
  int32_t q_heads;         /* a multiple of the cache's kv_heads                                  */
  int32_t out_type;
  float scale;
  int64_t window;          /* >= 0; 0: no window                                                  */
  int64_t max_len;         /* no sequence is longer: sets the launch's size                       */
} tpp_attn_desc;

/* q: n_seqs columns of q_heads * D entries of the cache's dtype; out: the same of out_type; lse:
 * n_seqs * q_heads floats, or NULL.
 * totals_out (NULL: not wanted): totals_out[b * ldt + t] = totals_in[b * ldt + t] + sum over the query
 * heads of p_t, for t < n (totals_in NULL counts as zeros; totals_out may be totals_in; ldt >=
 * max_len).
 * D: 8 .. 256.  n_seqs == 0 is a no-op; d_pages rows have ld_pages >= ceil(max_len / page_size)
 * entries.
 * Long caches are split over workgroups whose partial results (and, for totals, the scores) go to a
 * work buffer as tpp_reduce's do, under stream capture to one of the capture's own; where a capture
 * can have none, the launch is unsplit, and one with totals fails with NO_MEMORY.  Its size goes by
 * max_len, whatever the lengths are: 4 (D + 2) bytes for each of the n_seqs * q_heads rows and spans of
 * max_len (or window) positions, and with totals 4 bytes for each row and position of max_len.
 * Errors: INVALID_ARG as above and for a malformed desc or cache; UNSUPPORTED for other D, max_len above
 * 2^30 or a launch of 2^32 threads or more, before anything is done (256 for each span of 64 to 4096
 * positions of each key head of each sequence, and, where those are joined, for each of the q_heads *
 * n_seqs rows); NO_MEMORY; HIP if a launch fails. */
tpp_status tpp_paged_attention(const tpp_attn_desc* desc, const tpp_kv_cache* cache, int64_t n_seqs,
                               const void* q, int64_t ldq, const int64_t* d_len,
                               const int64_t* d_pages, int64_t ld_pages, void* out, int64_t ldo,
                               float* lse, const float* totals_in, float* totals_out, int64_t ldt,
                               void* stream);

/* ---- eviction by total weight --------------------------------------------------------------------- */

/* Cuts every sequence to `budget` positions: of its n = d_len[b] positions (cut to [0, max_len]) the
 * max(0, n - budget) with the least totals leave, equal totals by the lower t first (+0 and -0 are
 * equal; a NaN ranks above every number).  Positions protected by d_pos[b * ldt + t] >= d_horizon[b]
 * (both NULL: none is) never leave, so fewer may go.  Of the rest, those at t >= n', the new length,
 * move in order into the free places below n', the lowest first; everything else stays where it is.
 * Keys and values of the moved positions are copied inside the pools (all kv_heads), and for t < n'
 * totals_out and pos_out get the total and d_pos of what is at t now; len_out[b] = n'.  Entries from
 * n' on are not written.  Attention needs no order of the cached positions, so this is all an eviction
 * has to move.  A moved position whose page (old or new) holds nothing moves no keys or values.
 * Outputs may be the inputs themselves; otherwise they must not overlap them.  d_pos, d_horizon and
 * pos_out are given or NULL together.  No two sequences that lose positions may share a page.
 * Where no sequence can move more than a few rows (2048 chunks of 16 bytes of the keys: max_len - budget,
 * or half of max_len if that is less, times kv_heads times those of a row) and the totals stay in place or
 * max_len is at most 8192, one launch without work space; else work buffer and its errors as tpp_reduce
 * (a capture without one: NO_MEMORY).
 * Errors: INVALID_ARG for sizes < 0, max_len > 2^30, ldt < max_len, a malformed cache or a NULL
 * pointer when there is work; UNSUPPORTED for a launch of 2^32 threads or more (1024 for each
 * sequence, 256 for each 1024 positions of max_len where totals are not in place), or where the
 * moves of one sequence could be more than 2^30 rows (positions * kv_heads). */
tpp_status tpp_cache_evict(const tpp_kv_cache* cache, int64_t n_seqs, int64_t max_len, int64_t budget,
                           const int64_t* d_len, const int64_t* d_pages, int64_t ld_pages,
                           const float* totals, const int64_t* d_pos, const int64_t* d_horizon,
                           int64_t ldt, int64_t* len_out, float* totals_out, int64_t* pos_out,
                           void* stream);

#ifdef __cplusplus
}
#endif
#endif /* TPP_ATTENTION_H */

/*
 * tpp_q8.h -- C ABI of the 8-bit rows of the MI355X (gfx950) TPP library: activations in 8-bit integers
 * with a scale for each token or group of features, the products of such rows with 8-bit weights that
 * have a scale for each channel, and activations of training that keep their input in 8 bits for the
 * backward pass.
 *
 * The paper's TPPs (arXiv 2104.05755) name low-precision products and the conversion to and from them
 * among their uses (Sec. 2, Table 1: quantize / dequantize; Table 3); these calls are that part for the
 * fully-connected layers of Sec. 5.1.
 *
 * Conventions are those of tpp_brgemm.h: caller-owned DEVICE memory, element counts for strides,
 * asynchronous on `stream` (a hipStream_t as void*, NULL = the default stream), a tpp_status result and
 * tpp_last_error_message() for the detail.  Activations are column-major 2D blocks with a column per
 * token: feature i of token t is at z + t * ld + i.  Arithmetic is fp32; an output is rounded to its
 * type once (to nearest even).  Results do not vary between runs.
 *
 * 8-bit rows.  The entries v of a group are q * scale with
 *     scale = max|v| / 127,    q = the whole number nearest to 127 v / max|v| (ties to even)
 * exactly (scale rounded to fp32, q the rounding of the true quotient).  A group of zeros has scale 0.
 * A group with an infinity or NaN has scale NaN and q = 0, so that all that a product or the backward
 * pass of an activation makes of it is NaN (but for a product with TPP_EPI_RELU, whose x > 0 ? x : +0 is
 * 0 then, as everywhere in the library).
 * Entries of q behind a row's last feature are not written.  Outputs must not overlap inputs unless a call
 * says so.
 */
#ifndef TPP_Q8_H
#define TPP_Q8_H

#include "tpp_brgemm.h"

#ifdef __cplusplus
extern "C" {
#endif

/* act(z) = z;  z > 0 ? z : 0;  0.5 z (1 + tanh(sqrt(2/pi) (z + 0.044715 z^3)));  z / (1 + exp(-z)). */
typedef enum {
  TPP_ACT_NONE = 0,
  TPP_ACT_RELU = 1,
  TPP_ACT_GELU_TANH = 2,
  TPP_ACT_SILU = 3
} tpp_act_form;

/* An activation of `features` entries a token: h = act(z), or, gated, h_i = act(z_i) * z_{features + i}
 * with 2 * features entries of z a token. */
typedef struct {
  int32_t features;        /* 1 .. 2^20 (2^19 if gated)                                   */
  int32_t group;           /* features that share a scale, counted from the row's start:
                              0 (the whole row) or 16, 32, 64, 128, 256, 512               */
  int32_t dtype;           /* of z, h and their gradients                                 */
  int32_t act;             /* tpp_act_form                                                */
  int32_t gated;           /* 0 or 1                                                      */
} tpp_q8_desc;

/* h (as it would be rounded to dtype, but not stored) in 8-bit rows: entry i of token t at
 * q + t * ldq + i, the scale of its group at scale[t * lds + i / group] (scale[t * lds] where group is
 * 0).  tokens == 0 is a no-op.
 * Errors: INVALID_ARG for a NULL desc, unknown forms, sizes, flags or leading dimensions out of their
 * ranges, or a NULL pointer when there is work; UNSUPPORTED for other groups and more features; HIP if a
 * launch fails. */
tpp_status tpp_q8_quantize(const tpp_q8_desc* desc, int64_t tokens, const void* z, int64_t ldz, int8_t* q,
                           int64_t ldq, float* scale, int64_t lds, void* stream);

/* The activation in training: h, and z (all of its entries: 2 * features if gated) in 8-bit rows, which
 * are what the backward pass needs of it.  h may be NULL, and must not overlap z.
 * Errors: as tpp_q8_quantize. */
tpp_status tpp_q8_act(const tpp_q8_desc* desc, int64_t tokens, const void* z, int64_t ldz, void* h,
                      int64_t ldh, int8_t* q, int64_t ldq, float* scale, int64_t lds, void* stream);

/* The backward pass from z' = q * scale (in fp32, so infinite beyond its largest number) and the gradient
 * gh of h: the gradient of z,
 *     dz = gh * act'(z')      (gated, with a and u the halves of z': gh * u * act'(a) and gh * act(a))
 * the activation h2 = act(z') (for the next layer's weight gradient), and dbias = the sum of dz (not
 * rounded) over all tokens, one fp32 for each entry of z, overwritten (tokens == 0: zeros).  Each may be
 * NULL where it is not wanted; outputs must not overlap inputs, except h2, which may be gh (same ld).
 * act'(0) of RELU is 0; act and act' of a NaN are NaN, but for NONE's slope, which is 1.  dbias' partial
 * sums go to a work buffer as tpp_reduce's do, under stream capture to one of the capture's own.
 * Errors: as tpp_q8_quantize; NO_MEMORY if there is no work buffer to be had. */
tpp_status tpp_q8_act_backward(const tpp_q8_desc* desc, int64_t tokens, const int8_t* q, int64_t ldq,
                               const float* scale, int64_t lds, const void* gh, int64_t ldgh, void* dz,
                               int64_t lddz, void* h2, int64_t ldh2, float* dbias, void* stream);

/* C = act(b_scale_j * a_scale_i * sum_p A_ip B_pj + bias_i) for m channels i and n tokens j: A the 8-bit
 * weights with k contiguous, entry (i, p) at a + i * lda + p, B the 8-bit rows of the tokens, entry
 * (p, j) at b + j * ldb + p, C at c + j * ldc + i.  The sum is exact; it is multiplied with the token's
 * scale and then with the channel's, each in fp32.  Where a, b, lda and ldb are multiples of 16
 * bytes (and lda, ldb at most 8388607) whole 16-byte chunks are read, and what stands in them behind entry
 * k counts for nothing.  Other rows are right too but take 3 to 15 times as long (8192 tokens, 4096 -> 16384:
 * 7.3 ms against 0.48; 48 tokens: 61 us against 15): store weights with lda rounded up. */
typedef struct {
  int32_t m, n, k;         /* > 0, >= 0, > 0; m and n at most 2^31 - 512, k at most 131071:
                              the sum fits 32 bits                                          */
  int64_t lda, ldb, ldc;   /* >= k, k, m                                                    */
  int32_t b_type;          /* tpp_q8_linear: of the tokens' activations                     */
  int32_t c_type;
  uint32_t flags;          /* TPP_EPI_BIAS, and TPP_EPI_RELU or TPP_EPI_GELU_TANH           */
} tpp_q8_gemm_desc;

/* a_scale: m floats, b_scale: n floats, bias: m floats (NULL without TPP_EPI_BIAS).
 * Errors: INVALID_ARG for a NULL desc, sizes, types, flags or leading dimensions out of their ranges or
 * a NULL pointer when there is work; UNSUPPORTED for larger m, n or k, or a launch of 2^32 threads or
 * more; HIP if a launch fails. */
tpp_status tpp_q8_gemm(const tpp_q8_gemm_desc* desc, const int8_t* a, const float* a_scale,
                       const int8_t* b, const float* b_scale, void* c, const float* bias, void* stream);

/* The same of activations x (b_type, entry (p, j) at x + j * ldb + p), each token turned into an 8-bit
 * row first, as tpp_q8_quantize with act NONE and group 0 does it.  The rows go to a work buffer as
 * tpp_reduce's do (k bytes a token), under stream capture to one of the capture's own.  None is needed, and
 * there is one launch instead of two, where n <= 16, n * (k rounded up to a multiple of 128) <= 12288, and a
 * and lda are multiples of 16 bytes with lda <= 8388607.
 * Errors: as tpp_q8_gemm; NO_MEMORY if there is no work buffer to be had. */
tpp_status tpp_q8_linear(const tpp_q8_gemm_desc* desc, const int8_t* a, const float* a_scale,
                         const void* x, void* c, const float* bias, void* stream);

#ifdef __cplusplus
}
#endif
#endif /* TPP_Q8_H */

/*
 * tpp_residual.h -- C ABI of the residual stream's norms of the MI355X (gfx950) TPP library: the norm
 * after a block, its gate and scale, the addition to the stream and the norm before the next block in
 * one pass, and the gradients of all of them.
 *
 * The paper (Tensor Processing Primitives, arXiv 2104.05755) chains its fully-connected layers with
 * elementwise and Reduce TPPs (Sec. 2.2, 4.2, 5.1); these calls are the fused form of that chain
 * between two blocks of a network that is trained or that serves tokens.
 *
 * Conventions are those of tpp_brgemm.h: caller-owned DEVICE memory, element counts for strides,
 * asynchronous on `stream` (a hipStream_t as void*, NULL = the default stream), a tpp_status result and
 * tpp_last_error_message() for the detail.  Activations are column-major 2D blocks with a column per
 * token: feature i of token t is at x + t * ld + i.  Arithmetic is fp32; an output is rounded to its
 * type once (to nearest even); the sums of squares have to stay in fp32's range.  The order of every sum depends only on sizes: results do not vary
 * between runs.
 */
#ifndef TPP_RESIDUAL_H
#define TPP_RESIDUAL_H

#include "tpp_brgemm.h"

#ifdef __cplusplus
extern "C" {
#endif

/* N(v) = v;  v / sqrt(mean(v^2) + eps) * w;  (v - mean(v)) / sqrt(var(v) + eps) * w + c  (var: the mean
 * squared distance from the mean).  w and c are fp32 vectors of `features` entries; c may be NULL (0). */
typedef enum { TPP_NORM_NONE = 0, TPP_NORM_RMS = 1, TPP_NORM_LAYER = 2 } tpp_norm_form;

/* G(g) = 1 (there is no gate);  g;  1 / (1 + exp(-g));  tanh(g). */
typedef enum {
  TPP_GATE_NONE = 0,
  TPP_GATE_IDENTITY = 1,
  TPP_GATE_SIGMOID = 2,
  TPP_GATE_TANH = 3
} tpp_gate_form;

/* For every token, with x the stream, b the block's output and g the token's gate:
 *     r = x + scale * G(g) * N_after(b),     y = N_before(r)
 * where y is made of r as it was rounded to its type.  The gate of token t is row t / gate_every of
 * `gate` (row 0 where gate_every is 0: one gate for all tokens), `features` entries, ldg apart. */
typedef struct {
  int32_t features;        /* 1 .. 2^20                                          */
  int32_t dtype;           /* of x, b, r, y and their gradients                  */
  int32_t after, before;   /* tpp_norm_form                                      */
  int32_t gate;            /* tpp_gate_form                                      */
  int32_t gate_type;       /* of the gate and its gradient                       */
  float scale;             /* finite                                             */
  float eps;               /* finite, >= 0                                       */
  int64_t gate_every;      /* >= 0                                               */
} tpp_residual_desc;

/* Forward.  y: NULL where it is not wanted.  q, q_scale: NULL, or y (as it is rounded to its type) in
 * 8-bit rows as tpp_q8_quantize makes them (tpp_q8.h), feature i of token t at q + t * ldq + i, its
 * scale at q_scale[t].  w_after / w_before may be NULL only where the norm has none, c_after / c_before
 * always (0).  r may be x itself and y may be b itself (same ld); other outputs must not overlap inputs.
 * Leading dimensions (each >= features) count only where their tensor is there.  tokens == 0 is a no-op.
 * Errors: INVALID_ARG for a NULL desc, unknown forms, sizes or leading dimensions out of their ranges,
 * q without q_scale, or a NULL pointer when there is work; UNSUPPORTED for more than 2^20 features; HIP
 * if a launch fails. */
tpp_status tpp_residual_norm(const tpp_residual_desc* desc, int64_t tokens, const void* x, int64_t ldx,
                             const void* b, int64_t ldb, const void* gate, int64_t ldg,
                             const float* w_after, const float* c_after, const float* w_before,
                             const float* c_before, void* r, int64_t ldr, void* y, int64_t ldy,
                             int8_t* q, int64_t ldq, float* q_scale, void* stream);

/* Backward: from b, the gate, the forward call's r and the gradients gr of r (what reaches r by other
 * ways than y) and gy of y (NULL: 0), the gradients
 *     dx = gr + N_before'(gy),   db = N_after'(scale * G * dx),
 *     dgate = G'(g) * sum over the gate's tokens of scale * dx * N_after(b)
 * and those of the norms' vectors (`features` fp32 each, overwritten), summed over all tokens.  dx goes
 * on unrounded.  Every output may be NULL where it is not wanted.  dgate has the gate's type and rows,
 * lddg apart, each written once.  Outputs must not overlap inputs or each other (dx or db being b, r, gr
 * or gy, and two outputs being one, are refused).  tokens == 0 gives zero vectors, and a zero dgate where
 * gate_every is 0.
 * The vectors' partial sums (and for rows of more than 8192 features 24 bytes a token) go to a work
 * buffer as tpp_reduce's do, under stream capture to one of the capture's own.
 * Errors: as tpp_residual_norm; NO_MEMORY if there is no work buffer to be had. */
tpp_status tpp_residual_norm_backward(const tpp_residual_desc* desc, int64_t tokens, const void* b,
                                      int64_t ldb, const void* gate, int64_t ldg, const float* w_after,
                                      const float* c_after, const float* w_before, const void* r,
                                      int64_t ldr, const void* gr, int64_t ldgr, const void* gy,
                                      int64_t ldgy, void* dx, int64_t lddx, void* db, int64_t lddb,
                                      void* dgate, int64_t lddg, float* dw_after, float* dc_after,
                                      float* dw_before, float* dc_before, void* stream);

#ifdef __cplusplus
}
#endif
#endif /* TPP_RESIDUAL_H */

// residual_device.h -- what the forward and the backward kernels of the residual stream's norms share: gates,
// statistics of a row, and the widest row in registers.
#pragma once

#include <hip/hip_runtime.h>

#include "internal.h"
#include "rows_device.h"

namespace tpp {
namespace rows {

constexpr int RT = 256, RW = RT / 64;   // threads and wavefronts of a workgroup

__device__ __forceinline__ float gate_value(float g, int32_t form) {
  if (form == TPP_GATE_SIGMOID) return sigmoid(g);
  // tanh g = 2 sigmoid(2 g) - 1 loses what is small: tanhf
  if (form == TPP_GATE_TANH) return tanhf(g);
  return g;
}
// G' without a difference of near values: e s^2 and 4 e s^2 with s = 1 / (1 + e).
__device__ __forceinline__ float gate_slope(float g, int32_t form) {
  if (form == TPP_GATE_IDENTITY) return 1.0f;
  const float k = form == TPP_GATE_SIGMOID ? -1.44269504f : -2.88539008f;
  const float e = __builtin_amdgcn_exp2f(k * __builtin_fabsf(g)), s = __builtin_amdgcn_rcpf(1.0f + e);
  return (form == TPP_GATE_SIGMOID ? 1.0f : 4.0f) * e * s * s;
}
__device__ __forceinline__ int64_t gate_row(const ResidualParams& p, int64_t t) {
  if (!p.gate_form || !p.gate_every) return 0;
  return ((t | p.gate_every) >> 32) == 0 ? (uint32_t)t / (uint32_t)p.gate_every : t / p.gate_every;
}

// Mean (0 for RMS) and 1 / sqrt(.. + eps) of row v.
template <bool BF16>
__device__ __forceinline__ void row_stats(const ResidualParams& p, const void* v, int64_t at, int32_t form,
                                          float* part, float& mean, float& rs) {
  mean = 0.0f;
  rs = 1.0f;
  if (form == TPP_NORM_NONE) return;
  float s = 0.0f;
  if (form == TPP_NORM_LAYER) {
    for (int32_t i = threadIdx.x; i < p.f; i += RT) s += load1<BF16>(v, at + i);
    mean = over_group<Sum, RW>(s, part) / (float)p.f;
    s = 0.0f;
  }
  for (int32_t i = threadIdx.x; i < p.f; i += RT) {
    const float d = load1<BF16>(v, at + i) - mean;
    s += d * d;
  }
  __syncthreads();
  rs = 1.0f / sqrtf(over_group<Sum, RW>(s, part) / (float)p.f + p.eps);
  __syncthreads();
}
__device__ __forceinline__ float normed(float v, int32_t form, float mean, float rs, const float* w,
                                        const float* c, int32_t i) {
  if (form == TPP_NORM_NONE) return v;
  v = (v - mean) * rs * gld<float>(w + i);
  return form == TPP_NORM_LAYER && c ? v + gld<float>(c + i) : v;
}

// ---- rows in registers ----------------------------------------------------------------------------
template <int C>
__device__ __forceinline__ float sum_of(const float (&v)[C][8]) {
  float s = 0.0f;
#pragma unroll
  for (int k = 0; k < C; ++k)
#pragma unroll
    for (int e = 0; e < 8; ++e) s += v[k][e];
  return s;
}
template <int C>
__device__ __forceinline__ float squares_of(const float (&v)[C][8]) {
  float s = 0.0f;
#pragma unroll
  for (int k = 0; k < C; ++k)
#pragma unroll
    for (int e = 0; e < 8; ++e) s = __builtin_fmaf(v[k][e], v[k][e], s);
  return s;
}

constexpr int32_t MOST_ROW = 16384;       // entries of a row in registers

}  // namespace rows
}  // namespace tpp

// rows_device.h -- device-side pieces shared by the kernels over rows of features (residual_kernels.hip,
// q8_kernels.hip, q8_gemm_kernels.hip): sums and maxima over lanes and workgroups, activations, and the
// rounding to 8-bit rows.
#pragma once

#include <hip/hip_runtime.h>

#include "brgemm_device.h"
#include "internal.h"
#include "tpp_q8.h"

namespace tpp {
namespace rows {

using namespace dev;

template <bool BF16>
struct Elem {
  static constexpr int ES = BF16 ? 2 : 4;
};
template <bool BF16>
__device__ __forceinline__ float load1(const void* p, int64_t at) {
  if constexpr (BF16)
    return bf16_bits_to_f32(gld<uint16_t>(static_cast<const uint16_t*>(p) + at));
  else
    return gld<float>(static_cast<const float*>(p) + at);
}
template <bool BF16>
__device__ __forceinline__ void store1(void* p, int64_t at, float v) {
  if constexpr (BF16)
    gst<uint16_t>(static_cast<uint16_t*>(p) + at, f32_to_bf16_bits(v));
  else
    gst<float>(static_cast<float*>(p) + at, v);
}
// v as its type holds it.
template <bool BF16>
__device__ __forceinline__ float rounded(float v) {
  return BF16 ? bf16_bits_to_f32(f32_to_bf16_bits(v)) : v;
}
__device__ __forceinline__ void store1(void* p, int64_t at, float v, bool bf16) {
  bf16 ? store1<true>(p, at, v) : store1<false>(p, at, v);
}
__device__ __forceinline__ float load1(const void* p, int64_t at, bool bf16) {
  return bf16 ? load1<true>(p, at) : load1<false>(p, at);
}

// ---- over lanes and workgroups ------------------------------------------------------------------
template <int CTRL>
__device__ __forceinline__ uint32_t dpp(uint32_t v) {
  return __builtin_amdgcn_update_dpp(0, v, CTRL, 0xf, 0xf, true);
}
struct Sum {
  __device__ static float join(float a, float b) { return a + b; }
};
// Magnitudes by their bits: of one order with the values, infinities and NaN above all.
struct Top {
  __device__ static uint32_t join(uint32_t a, uint32_t b) { return a > b ? a : b; }
};
// op over groups of LANES (a power of two, 1 .. 64) consecutive lanes, in every one of them.
template <typename OP, int LANES, typename T>
__device__ __forceinline__ T over_lanes(T v) {
  const auto with = [&](uint32_t w) { v = OP::join(v, __builtin_bit_cast(T, w)); };
  const auto bits = [&]() { return __builtin_bit_cast(uint32_t, v); };
  if constexpr (LANES >= 2) with(dpp<0xB1>(bits()));     // lane ^ 1
  if constexpr (LANES >= 4) with(dpp<0x4E>(bits()));     // lane ^ 2
  if constexpr (LANES >= 8) with(dpp<0x141>(bits()));    // the other quad of 8
  if constexpr (LANES >= 16) with(dpp<0x140>(bits()));   // the other 8 of 16
  if constexpr (LANES >= 32) {
    const auto w = __builtin_amdgcn_permlane16_swap(bits(), bits(), false, false);
    const uint32_t a = w[0], b = w[1];   // (values: a bit_cast of w[1] itself reads w[0])
    v = OP::join(__builtin_bit_cast(T, a), __builtin_bit_cast(T, b));
  }
  if constexpr (LANES >= 64) {
    const auto w = __builtin_amdgcn_permlane32_swap(bits(), bits(), false, false);
    const uint32_t a = w[0], b = w[1];   // (values: a bit_cast of w[1] itself reads w[0])
    v = OP::join(__builtin_bit_cast(T, a), __builtin_bit_cast(T, b));
  }
  return v;
}
// op over a workgroup of W wavefronts, in order, in every thread.  `part`: W words of LDS, free again
// after the next barrier that is not this one's.
template <typename OP, int W, typename T>
__device__ __forceinline__ T over_group(T v, T* part) {
  v = over_lanes<OP, 64>(v);
  if constexpr (W > 1) {
    if ((threadIdx.x & 63) == 0) part[threadIdx.x >> 6] = v;
    __syncthreads();
    v = part[0];
#pragma unroll
    for (int w = 1; w < W; ++w) v = OP::join(v, part[w]);
  }
  return v;
}

// ---- activations --------------------------------------------------------------------------------
__device__ __forceinline__ float sigmoid(float z) {   // (exp(-z) = inf gives 0)
  return __builtin_amdgcn_rcpf(1.0f + __builtin_amdgcn_exp2f(z * -1.44269504f));
}
__device__ __forceinline__ float act_value(float z, int32_t act) {
  if (act == TPP_ACT_RELU) return z > 0.0f ? z : 0.0f;
  if (act == TPP_ACT_GELU_TANH) return gelu_tanh(z);
  if (act == TPP_ACT_SILU) return z * sigmoid(z);
  return z;
}
// act(z) and act'(z) together: the exponential is shared.
__device__ __forceinline__ void act_both(float z, int32_t act, float& value, float& slope) {
  if (act == TPP_ACT_RELU) {
    value = z > 0.0f ? z : 0.0f;
    slope = z > 0.0f ? 1.0f : 0.0f;
  } else if (act == TPP_ACT_GELU_TANH) {
    value = gelu_tanh(z);
    slope = gelu_tanh_grad(z);
    slope = z != z ? z : slope;   // (its clamp would drop a NaN)
  } else if (act == TPP_ACT_SILU) {
    const float e = __builtin_amdgcn_exp2f(fminf(z * -1.44269504f, 126.0f));   // 1 - s = e s, finite
    const float s = __builtin_amdgcn_rcpf(1.0f + e);
    value = z * s;
    slope = s + z * (e * s) * s;
    slope = z != z ? z : slope;
  } else {
    value = z;
    slope = 1.0f;
  }
}

// ---- 8-bit rows -----------------------------------------------------------------------------------
__device__ __forceinline__ uint32_t magnitude(float v) { return __float_as_uint(v) & 0x7fffffffu; }

// What a group's largest magnitude says of its entries' rounding.
struct Q8Group {
  float top, pre, inv, scale;
};
__device__ __forceinline__ Q8Group q8_group(uint32_t top_bits) {
  Q8Group g;
  const float top = __uint_as_float(top_bits);
  if (top_bits >= 0x7f800000u) {   // an infinity or NaN: q = 0, scale NaN
    g.top = g.pre = g.inv = 0.0f;
    g.scale = __uint_as_float(0x7fc00000u);
    return g;
  }
  g.top = top;
  g.pre = top < 0x1p-60f ? 0x1p100f : 1.0f;   // so that 127 / max|v| stays finite
  g.inv = top > 0.0f ? 127.0f / (top * g.pre) : 0.0f;
  g.scale = top / 127.0f;
  return g;
}
// The whole number nearest to 127 v / top, ties to even.  t = v * (127 / top) is off by less than 3e-5
// (|t| <= 127, two roundings of 2^-24): only a t that near to k + 1/2 can round to the wrong side, and
// there 127 |v| is compared with (k + 1/2) top, both exact in 64 bits.
__device__ __forceinline__ int32_t q8_round(float v, const Q8Group& g) {
  const float t = v * g.pre * g.inv;
  float k = __builtin_rintf(t);
  const float d = t - k;
  if (__builtin_fabsf(d) > 0.5f - 3e-5f) {
    const float half = __builtin_fabsf(k + (d > 0.0f ? 0.5f : -0.5f)), low = half - 0.5f;
    const double a = 127.0 * (double)__builtin_fabsf(v), b = (double)half * (double)g.top;
    const float even = ((int32_t)low & 1) ? low + 1.0f : low;
    const float m = a < b ? low : a > b ? low + 1.0f : even;
    k = v < 0.0f ? -m : m;
  }
  return k == k ? (int32_t)k : 0;   // (NaN: an entry of a group without a scale)
}

}  // namespace rows
}  // namespace tpp

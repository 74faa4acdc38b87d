// rows_device.h -- device-side pieces shared by the kernels over rows of features (residual_kernels.hip,
// q8_kernels.hip, q8_gemm_kernels.hip): sums and maxima over lanes and workgroups, activations, the
// rounding to 8-bit rows, and what their launches choose by.
#pragma once

#include <hip/hip_runtime.h>

#include <type_traits>

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
// The same for a number of lanes that only the launch knows.
template <typename OP, typename T>
__device__ __forceinline__ T over_lanes(T v, int32_t lanes) {
  switch (lanes) {
    case 2: return over_lanes<OP, 2>(v);
    case 4: return over_lanes<OP, 4>(v);
    case 8: return over_lanes<OP, 8>(v);
    case 16: return over_lanes<OP, 16>(v);
    case 32: return over_lanes<OP, 32>(v);
  }
  return over_lanes<OP, 64>(v);
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

// 1 / sqrt(v): the instruction's unit in the last place is enough, but it takes no numbers below the normal
// ones.
__device__ __forceinline__ float rsqrt_of(float v) {
  return v < 0x1p-100f ? 1.0f / sqrtf(v) : __builtin_amdgcn_rsqf(v);
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
// act(z) and act'(z) together: the exponential is shared.  A NaN, which is what a group of 8 bits without a scale
// holds, gives a NaN of both behind RELU too (z > 0 ? .. would make a zero of it).
// s = 1 / (1 + e) falls to 0 where e passes fp32's range, far left of zero, and z s with it; 1 - s = e s (no
// difference of near values) is taken of an e that stays finite, where s = 0 leaves nothing of the slope.
__device__ __forceinline__ void act_both(float z, int32_t act, float& value, float& slope) {
  constexpr float BIG = 0x1p126f;
  if (act == TPP_ACT_RELU) {
    value = z <= 0.0f ? 0.0f : z;
    slope = z <= 0.0f ? 0.0f : z != z ? z : 1.0f;
  } else if (act == TPP_ACT_GELU_TANH) {   // gelu_tanh and gelu_tanh_grad with one exponential
    const float e = __builtin_amdgcn_exp2f(z * __builtin_fmaf(-0.10294324f, z * z, -2.3022082f));
    const float s = __builtin_amdgcn_rcpf(1.0f + e);
    const float x = __builtin_amdgcn_fmed3f(z, -9.0f, 9.0f);   // (beyond it the slope is s to within 3e-27)
    value = z * s;
    slope = s * __builtin_fmaf(1.5957691f * x * (fminf(e, BIG) * s), __builtin_fmaf(0.134145f, x * x, 1.0f), 1.0f);
  } else if (act == TPP_ACT_SILU) {
    const float e = __builtin_amdgcn_exp2f(z * -1.44269504f);
    const float s = __builtin_amdgcn_rcpf(1.0f + e);
    value = z * s;
    slope = __builtin_fmaf(z * (fminf(e, BIG) * s), s, s);
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
    g.top = g.inv = 0.0f;
    g.pre = 1.0f;
    g.scale = __uint_as_float(0x7fc00000u);
    return g;
  }
  g.top = top;
  g.pre = top < 0x1p-60f ? 0x1p100f : 1.0f;   // so that 127 / max|v| stays finite
  g.inv = top > 0.0f ? 127.0f / (top * g.pre) : 0.0f;
  g.scale = top / 127.0f;
  return g;
}
// The whole number nearest to 127 v / top, ties to even, decided exactly: 127 |v| is compared with (k + 1/2) top,
// both exact in 64 bits, for the half k + 1/2 next to t, which is off by little.
__device__ __forceinline__ int32_t q8_exact(float v, float t, const Q8Group& g) {
  const float k = __builtin_rintf(t);
  const float half = __builtin_fabsf(k + (t > k ? 0.5f : -0.5f)), low = half - 0.5f;
  const double a = 127.0 * (double)__builtin_fabsf(v), b = (double)half * (double)g.top;
  const float even = ((int32_t)low & 1) ? low + 1.0f : low;
  const float m = a < b ? low : a > b ? low + 1.0f : even;
  return (int32_t)(v < 0.0f ? -m : m);
}
// Eight entries.  t = v * (127 / top) is off by less than 3e-5 (|t| <= 127, two roundings of 2^-24): only a t
// that near to k + 1/2 can round to the wrong side.  Adding 1.5 * 2^23 rounds t and leaves the number in the
// low byte.
__device__ __forceinline__ u32x2 q8_round(const float (&v)[8], const Q8Group& g) {
  constexpr float M = 12582912.0f;
  float t[8], m[8], off = 0.0f;
#pragma unroll
  for (int e = 0; e < 8; ++e) t[e] = v[e] * g.inv;
  if (g.pre != 1.0f) {
#pragma unroll
    for (int e = 0; e < 8; ++e) t[e] = v[e] * g.pre * g.inv;
  }
#pragma unroll
  for (int e = 0; e < 8; ++e) {
    m[e] = t[e] + M;
    off = __builtin_fmaxf(off, __builtin_fabsf(t[e] - (m[e] - M)));
  }
  if (off > 0.5f - 3e-5f) {
#pragma unroll
    for (int e = 0; e < 8; ++e)
      if (__builtin_fabsf(t[e] - (m[e] - M)) > 0.5f - 3e-5f) m[e] = M + (float)q8_exact(v[e], t[e], g);
  }
  u32x2 w;
#pragma unroll
  for (int h = 0; h < 2; ++h) {
    const uint32_t lo = __builtin_amdgcn_perm(__float_as_uint(m[4 * h + 1]), __float_as_uint(m[4 * h]), 0x0c0c0400u);
    const uint32_t hi = __builtin_amdgcn_perm(__float_as_uint(m[4 * h + 3]), __float_as_uint(m[4 * h + 2]), 0x04000c0cu);
    w[h] = g.inv > 0.0f ? lo | hi : 0u;   // (a group of zeros, or without a scale)
  }
  return w;
}
__device__ __forceinline__ int32_t q8_round(float v, const Q8Group& g) {
  const float x[8] = {v, 0.0f, 0.0f, 0.0f, 0.0f, 0.0f, 0.0f, 0.0f};
  return (int8_t)(q8_round(x, g)[0] & 0xffu);
}

// ---- chunks of eight entries --------------------------------------------------------------------
// A lane has chunks of 8 consecutive entries of a row.  In a row that is no multiple of 8 the last chunk
// ends with the row, and its first entries, which another lane has, count for nothing: they are taken as
// zeros and not stored.  So there is no branch around a load, and nothing outside the row is read; the row
// has 8 entries at least.
struct Place {
  int32_t at, skip;   // first entry, entries that another lane has (8: the lane has none)
  Place() = default;
  __device__ __forceinline__ Place(int32_t chunk, int32_t f) {
    const int32_t start = chunk * 8;
    at = min(start, f - 8);
    skip = min(start - at, 8);
  }
  __device__ __forceinline__ bool none() const { return skip >= 8; }
};
// The chunks of a lane in a row that W wavefronts have, 64 consecutive ones to a wavefront at a time (W 1:
// every wavefront of the workgroup has a row of its own).
template <int W, int C>
__device__ __forceinline__ void places(int32_t f, Place (&c)[C]) {
  const int32_t lane = threadIdx.x & 63, wave = W == 1 ? 0 : threadIdx.x >> 6;
#pragma unroll
  for (int k = 0; k < C; ++k) c[k] = Place((k * W + wave) * 64 + lane, f);
}

// How a pass goes through the caches: what is moved once only displaces what may be read again.
enum { CACHED, STREAM_OUT, STREAM };

template <bool BF16>
struct Raw {
  u32x4 w[BF16 ? 1 : 2];
};
typedef uint32_t u32x2_a1 __attribute__((ext_vector_type(2), aligned(1)));

template <bool BF16, int HOW>
__device__ __forceinline__ Raw<BF16> load_raw(const void* p, int64_t at) {
  Raw<BF16> r;
  const char* from = static_cast<const char*>(p) + at * (BF16 ? 2 : 4);
#pragma unroll
  for (int h = 0; h < (BF16 ? 1 : 2); ++h) {
    const GLOBAL_AS u32x4_a2* q = (const GLOBAL_AS u32x4_a2*)(from + 16 * h);
    r.w[h] = HOW == STREAM ? (u32x4)__builtin_nontemporal_load(q) : (u32x4)*q;
  }
  return r;
}
template <bool BF16>
__device__ __forceinline__ void widen(const Raw<BF16>& r, float (&v)[8]) {
#pragma unroll
  for (int e = 0; e < 8; ++e) {
    if constexpr (BF16)
      v[e] = __uint_as_float(e & 1 ? r.w[0][e / 2] & 0xffff0000u : r.w[0][e / 2] << 16);
    else
      v[e] = __uint_as_float(r.w[e / 4][e % 4]);
  }
}
// Zeros in the place of what another lane has: as loaded, or widened.
template <bool WHOLE, bool BF16>
__device__ __forceinline__ void mask(const Place& c, Raw<BF16>& r) {
#pragma unroll
  for (int i = 0; i < (BF16 ? 4 : 8); ++i) {
    uint32_t w = r.w[i / 4][i % 4];
    if constexpr (WHOLE)
      w = c.skip ? 0u : w;
    else if constexpr (BF16)
      w &= (2 * i >= c.skip ? 0xffffu : 0u) | (2 * i + 1 >= c.skip ? 0xffff0000u : 0u);
    else
      w = i >= c.skip ? w : 0u;
    r.w[i / 4][i % 4] = w;
  }
}
template <bool WHOLE>
__device__ __forceinline__ void mask(const Place& c, float (&v)[8]) {
#pragma unroll
  for (int e = 0; e < 8; ++e) v[e] = (WHOLE ? c.skip != 0 : e < c.skip) ? 0.0f : v[e];
}
// The largest magnitude of a chunk.
typedef uint16_t u16x2 __attribute__((ext_vector_type(2)));
template <bool BF16>
__device__ __forceinline__ uint32_t top8(const Raw<BF16>& r) {
  if constexpr (BF16) {
    u16x2 top = {0, 0};
#pragma unroll
    for (int i = 0; i < 4; ++i) top = __builtin_elementwise_max(top, __builtin_bit_cast(u16x2, r.w[0][i] & 0x7fff7fffu));
    return (uint32_t)(top.x > top.y ? top.x : top.y) << 16;
  } else {
    uint32_t top = 0;
#pragma unroll
    for (int i = 0; i < 8; ++i) top = Top::join(top, r.w[i / 4][i % 4] & 0x7fffffffu);
    return top;
  }
}
__device__ __forceinline__ void load8(const float* p, int32_t at, float (&v)[8]) {
  widen<false>(load_raw<false, CACHED>(p, at), v);
}
__device__ __forceinline__ void load8(const void* p, int64_t at, bool bf16, float (&v)[8]) {
  if (bf16)
    widen<true>(load_raw<true, CACHED>(p, at), v);
  else
    widen<false>(load_raw<false, CACHED>(p, at), v);
}
template <bool BF16>
__device__ __forceinline__ Raw<BF16> narrow(const float (&v)[8]) {
  Raw<BF16> r;
#pragma unroll
  for (int e = 0; e < (BF16 ? 4 : 8); ++e) {
    if constexpr (BF16)
      r.w[0][e] = pack_bf16x2(v[2 * e], v[2 * e + 1]);
    else
      r.w[e / 4][e % 4] = __float_as_uint(v[e]);
  }
  return r;
}
template <bool BF16, bool WHOLE, int HOW>
__device__ __forceinline__ void store_raw(void* p, int64_t row, const Place& c, const Raw<BF16>& r) {
  char* to = static_cast<char*>(p) + (row + c.at) * (BF16 ? 2 : 4);
  if (c.skip == 0) {
#pragma unroll
    for (int h = 0; h < (BF16 ? 1 : 2); ++h) {
      GLOBAL_AS u32x4_a2* q = (GLOBAL_AS u32x4_a2*)(to + 16 * h);
      if constexpr (HOW != CACHED)
        __builtin_nontemporal_store((u32x4_a2)r.w[h], q);
      else
        *q = (u32x4_a2)r.w[h];
    }
  } else if (!WHOLE && !c.none()) {
#pragma unroll
    for (int e = 1; e < 8; ++e) {
      if (e < c.skip) continue;
      if constexpr (BF16)
        gst<uint16_t>(to + 2 * e, (uint16_t)(e & 1 ? r.w[0][e / 2] >> 16 : r.w[0][e / 2]));
      else
        gst<uint32_t>(to + 4 * e, r.w[e / 4][e % 4]);
    }
  }
}
// Eight entries of an 8-bit row.
template <bool WHOLE>
__device__ __forceinline__ void store_q8(int8_t* row, const Place& c, const float (&v)[8], const Q8Group& g) {
  if (c.none()) return;
  const u32x2 w = q8_round(v, g);
  if (c.skip == 0) {
    gst<u32x2_a1>(row + c.at, (u32x2_a1){w[0], w[1]});
  } else if (!WHOLE) {
#pragma unroll
    for (int e = 1; e < 8; ++e)
      if (e >= c.skip) gst<uint8_t>(row + c.at + e, (uint8_t)(w[e / 4] >> (8 * (e % 4))));
  }
}

// ---- launches -------------------------------------------------------------------------------------
constexpr int64_t MB = int64_t(1) << 20;
inline int64_t ceil_div(int64_t a, int64_t b) { return (a + b - 1) / b; }
inline int64_t min64(int64_t a, int64_t b) { return a < b ? a : b; }
// f(bf16, whether rows of `width` entries are whole chunks).
template <typename F>
void by_type(bool bf16, int32_t width, const F& f) {
  const std::true_type yes;
  const std::false_type no;
  const bool whole = width % 8 == 0;
  if (bf16) whole ? f(yes, yes) : f(yes, no);
  else whole ? f(no, yes) : f(no, no);
}

}  // namespace rows
}  // namespace tpp

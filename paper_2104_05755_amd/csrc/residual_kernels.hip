// residual_kernels.hip -- the residual stream's norms, forward, for gfx950.
//
// r = x + scale G(g) N_after(b), y = N_before(r): two norms over a token's features, about 12 operations an
// entry of 2 or 4 bytes, four of which are moved: bound by HBM.  A row stays in registers from its one reading
// to its one writing, so that a sum over it costs register permutes and, beyond one wavefront, one exchange
// through LDS; the vectors and the gate come from the caches, which all rows share.
//
// 8192 tokens of 4096 bf16: 55 us, 4.9 TB/s (a copy of as much: 52 us); 16384 of 1024 26 us; one of 1024 3.0 us
// of kernel, 5.1 from call to call.  From a workgroup to a row and a pass for every sum: 293 us.  Two chunks of
// 8 entries to a lane carried best: of 4096 entries by 1, 2, 4 or 8 wavefronts 94, 69, 55 and 58 us.
#include <hip/hip_runtime.h>

#include "residual_device.h"

namespace tpp {
namespace {

using namespace rows;

// ---- any width ------------------------------------------------------------------------------------
// Rows below 8 entries or above 16384: a workgroup to a token, which reads its row again for each sum.
template <bool BF16>
__global__ __launch_bounds__(RT) void residual_any_kernel(ResidualParams p) {
  __shared__ float part[RW];
  __shared__ uint32_t tops[RW];
  for (int64_t t = blockIdx.x; t < p.tokens; t += gridDim.x) {
    float mean, rs;
    row_stats<BF16>(p, p.b, t * p.ldb, p.after, part, mean, rs);
    const int64_t g0 = gate_row(p, t) * p.ldg;
    for (int32_t i = threadIdx.x; i < p.f; i += RT) {
      float n = normed(load1<BF16>(p.b, t * p.ldb + i), p.after, mean, rs, p.wa, p.ca, i);
      if (p.gate_form) n *= gate_value(load1(p.gate, g0 + i, p.gate_bf16), p.gate_form);
      store1<BF16>(p.r, t * p.ldr + i, load1<BF16>(p.x, t * p.ldx + i) + p.scale * n);
    }
    if (!p.y && !p.q) continue;   // (a thread reads back only what it wrote itself)
    row_stats<BF16>(p, p.r, t * p.ldr, p.before, part, mean, rs);
    uint32_t top = 0;
    const auto y = [&](int32_t i) {
      return rounded<BF16>(normed(load1<BF16>(p.r, t * p.ldr + i), p.before, mean, rs, p.wb, p.cb, i));
    };
    for (int32_t i = threadIdx.x; i < p.f; i += RT) {
      const float v = y(i);
      top = Top::join(top, magnitude(v));
      if (p.y) store1<BF16>(p.y, t * p.ldy + i, v);
    }
    if (!p.q) continue;
    const Q8Group g = q8_group(over_group<Top, RW>(top, tops));
    for (int32_t i = threadIdx.x; i < p.f; i += RT) gst<int8_t>(p.q + t * p.ldq + i, (int8_t)q8_round(y(i), g));
    if (threadIdx.x == 0) gst<float>(p.qs + t, g.scale);
    __syncthreads();
  }
}

// ---- rows in registers ----------------------------------------------------------------------------
// A row of 8 to 16384 entries belongs to W wavefronts, C chunks of 8 to a lane; a workgroup has one row, or
// four where W is 1.

// v normed but for the vectors: its mean taken off (layer norm), times 1 / sqrt(.. + eps).
template <int W, int C, bool WHOLE>
__device__ __forceinline__ void norm_row(float (&v)[C][8], const Place (&c)[C], int32_t form, float eps,
                                         float inv_f, float (&part)[2][W]) {
  if (form == TPP_NORM_NONE) return;
  if (form == TPP_NORM_LAYER) {
    const float mean = over_group<Sum, W>(sum_of(v), part[0]) * inv_f;
#pragma unroll
    for (int k = 0; k < C; ++k) {
#pragma unroll
      for (int e = 0; e < 8; ++e) v[k][e] -= mean;
      mask<WHOLE>(c[k], v[k]);
    }
  }
  const float rs = rsqrt_of(over_group<Sum, W>(squares_of(v), part[1]) * inv_f + eps);
#pragma unroll
  for (int k = 0; k < C; ++k)
#pragma unroll
    for (int e = 0; e < 8; ++e) v[k][e] *= rs;
}
__device__ __forceinline__ void with_vectors(float (&v)[8], int32_t form, const float (&w)[8], const float* c,
                                             int32_t at) {
  if (form == TPP_NORM_NONE) return;
#pragma unroll
  for (int e = 0; e < 8; ++e) v[e] *= w[e];
  if (form != TPP_NORM_LAYER || !c) return;
  float x[8];
  load8(c, at, x);
#pragma unroll
  for (int e = 0; e < 8; ++e) v[e] += x[e];
}

template <bool BF16, int W, int C, bool WHOLE, int HOW>
__global__ __launch_bounds__(W == 1 ? RT : 64 * W) void residual_row_kernel(ResidualParams p) {
  __shared__ float part[2][2][W];
  __shared__ uint32_t tops[W];
  constexpr int R = W == 1 ? RW : 1;
  const int32_t sub = W == 1 ? __builtin_amdgcn_readfirstlane(threadIdx.x >> 6) : 0;
  const float inv_f = 1.0f / (float)p.f;
  Place c[C];
  places<W, C>(p.f, c);
  for (int64_t t = (int64_t)blockIdx.x * R + sub; t < p.tokens; t += (int64_t)gridDim.x * R) {
    Raw<BF16> xr[C], br[C];
#pragma unroll
    for (int k = 0; k < C; ++k) br[k] = load_raw<BF16, HOW>(p.b, t * p.ldb + c[k].at);
#pragma unroll
    for (int k = 0; k < C; ++k) xr[k] = load_raw<BF16, HOW>(p.x, t * p.ldx + c[k].at);
    // the vectors: where the pass is no stream, under way with the rows rather than behind the sums (one token
    // of 1024 4.0 -> 3.5 us of kernel; 8192 of 4096 53 -> 57, whose registers hold more rows back)
    constexpr bool EARLY = HOW == CACHED;
    float v[C][8], wa[C][8], wb[C][8];
    const auto vector = [&](bool there, const float* w, float (&to)[C][8]) {
      if (!there) return;
#pragma unroll
      for (int k = 0; k < C; ++k) load8(w, c[k].at, to[k]);
    };
    if constexpr (EARLY) {
      vector(p.after, p.wa, wa);
      vector(p.before && (p.y || p.q), p.wb, wb);
    }
#pragma unroll
    for (int k = 0; k < C; ++k) {
      mask<WHOLE>(c[k], br[k]);
      widen<BF16>(br[k], v[k]);
    }
    norm_row<W, C, WHOLE>(v, c, p.after, p.eps, inv_f, part[0]);
    const int64_t g0 = gate_row(p, t) * p.ldg;
#pragma unroll
    for (int k = 0; k < C; ++k) {
      if (!EARLY && p.after) load8(p.wa, c[k].at, wa[k]);
      with_vectors(v[k], p.after, wa[k], p.ca, c[k].at);
      if (p.gate_form) {
        float g[8];
        load8(p.gate, g0 + c[k].at, p.gate_bf16, g);
#pragma unroll
        for (int e = 0; e < 8; ++e) v[k][e] *= gate_value(g[e], p.gate_form);
      }
      float x[8];
      widen<BF16>(xr[k], x);
#pragma unroll
      for (int e = 0; e < 8; ++e) v[k][e] = __builtin_fmaf(p.scale, v[k][e], x[e]);
      Raw<BF16> r = narrow<BF16>(v[k]);
      store_raw<BF16, WHOLE, HOW>(p.r, t * p.ldr, c[k], r);
      mask<WHOLE>(c[k], r);
      widen<BF16>(r, v[k]);
    }
    if (p.y || p.q) {
      norm_row<W, C, WHOLE>(v, c, p.before, p.eps, inv_f, part[1]);
      uint32_t top = 0;
#pragma unroll
      for (int k = 0; k < C; ++k) {
        if (!EARLY && p.before) load8(p.wb, c[k].at, wb[k]);
        with_vectors(v[k], p.before, wb[k], p.cb, c[k].at);
        Raw<BF16> y = narrow<BF16>(v[k]);
        if (p.y) store_raw<BF16, WHOLE, HOW>(p.y, t * p.ldy, c[k], y);
        mask<WHOLE>(c[k], y);
        widen<BF16>(y, v[k]);
        top = Top::join(top, top8<BF16>(y));
      }
      if (p.q) {
        const Q8Group g = q8_group(over_group<Top, W>(top, tops));
#pragma unroll
        for (int k = 0; k < C; ++k) store_q8<WHOLE>(p.q + t * p.ldq, c[k], v[k], g);
        if ((W == 1 ? threadIdx.x & 63 : threadIdx.x) == 0) gst<float>(p.qs + t, g.scale);
      }
    }
    if constexpr (W > 1) __syncthreads();   // the sums' places are free for the next row
  }
}

// f(wavefronts of a row, chunks of a lane).
template <typename F>
void by_width(const ResidualParams& p, const F& f) {
  const int32_t chunks = (p.f + 511) / 512;   // wavefronts' chunks of a row
  if (chunks <= 1) return f(IntC<1>(), IntC<1>());
  if (chunks <= 2) return f(IntC<1>(), IntC<2>());
  if (chunks <= 4) return f(IntC<2>(), IntC<2>());
  if (chunks <= 8) return f(IntC<4>(), IntC<2>());
  if (chunks <= 16) return f(IntC<8>(), IntC<2>());
  return f(IntC<16>(), IntC<2>());
}

}  // namespace

hipError_t launch_residual(const ResidualParams& p, hipStream_t stream) {
  if (p.f >= 8 && p.f <= MOST_ROW) {
    // Beyond the L2s' reach what is moved once goes past the caches' replacement, in and out: 1024 tokens of
    // 4096 bf16 (two outputs of 8 MB) 7.4 us against 10.1, 8192 55.5 against 61.0 (outputs alone: 8.2, 60.0).
    const bool stream_it = p.tokens * p.f * (p.bf16 ? 2 : 4) * (p.y ? 2 : 1) > 8 * MB;
    by_type(p.bf16, p.f, [&](auto bf16, auto whole) {
      by_width(p, [&](auto w, auto c) {
        constexpr int W = decltype(w)::value, C = decltype(c)::value, R = W == 1 ? RW : 1;
        const auto launch = [&](auto how) {
          hipLaunchKernelGGL((residual_row_kernel<decltype(bf16)::value, W, C, decltype(whole)::value,
                                                  decltype(how)::value>),
                             dim3((uint32_t)min64(ceil_div(p.tokens, R), 1 << 20)), dim3(W == 1 ? RT : 64 * W), 0,
                             stream, p);
        };
        if (stream_it) launch(IntC<STREAM>());
        else launch(IntC<CACHED>());
      });
    });
    return hipGetLastError();
  }
  const dim3 grid((uint32_t)min64(p.tokens, 1 << 20));
  if (p.bf16)
    hipLaunchKernelGGL((residual_any_kernel<true>), grid, dim3(RT), 0, stream, p);
  else
    hipLaunchKernelGGL((residual_any_kernel<false>), grid, dim3(RT), 0, stream, p);
  return hipGetLastError();
}

}  // namespace tpp

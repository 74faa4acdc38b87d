// q8_kernels.hip -- 8-bit rows of activations (gfx950): quantisation for a product, and activations of
// training that keep their input in 8 bits, with the backward pass from it.
//
// A group's entries become q = 127 v / max|v| rounded to whole numbers, scale = max|v| / 127: about 9 operations
// an entry of 1 to 4 bytes (30 with an activation): bound by HBM.
//
// 8192 tokens of 4096 bf16: a GELU with its input kept 34 us, 4.9 TB/s, its backward pass 52 us, 4.5 TB/s, and 4.7
// the fold of dbias (a copy of as much: 78 us in all); quantised for a product 33 us.  A workgroup to a row and a
// pass for the maximum: 113, 80 and 75 us.
#include <hip/hip_runtime.h>

#include <type_traits>

#include "internal.h"
#include "rows_device.h"

namespace tpp {
namespace {

using namespace rows;

constexpr int QT = 256, QW = QT / 64;   // threads and wavefronts of a workgroup

// Entry i of h.
template <bool BF16>
__device__ __forceinline__ float h_of(const Q8Params& p, int64_t at, int32_t i) {
  const float a = act_value(load1<BF16>(p.z, at + i), p.act);
  return p.gated ? a * load1<BF16>(p.z, at + p.f + i) : a;
}

// ---- any layout -----------------------------------------------------------------------------------
// A workgroup to a token; a group of 16 to 512 entries to a wavefront, a whole row to the workgroup.

// The 8-bit row of width entries value(i).
template <typename F>
__device__ __forceinline__ void quantize_row(const Q8Params& p, int64_t t, int32_t width, uint32_t* tops,
                                             const F& value) {
  int8_t* q = p.q + t * p.ldq;
  float* s = p.s + t * p.lds;
  if (p.group == 0) {
    uint32_t top = 0;
    for (int32_t i = threadIdx.x; i < width; i += QT) top = Top::join(top, magnitude(value(i)));
    const Q8Group g = q8_group(over_group<Top, QW>(top, tops));
    for (int32_t i = threadIdx.x; i < width; i += QT) gst<int8_t>(q + i, (int8_t)q8_round(value(i), g));
    if (threadIdx.x == 0) gst<float>(s, g.scale);
    __syncthreads();
    return;
  }
  const int32_t wave = threadIdx.x >> 6, lane = threadIdx.x & 63;
  for (int32_t j = wave; j * p.group < width; j += QW) {
    const int32_t end = min(width, (j + 1) * p.group);
    uint32_t top = 0;
    for (int32_t i = j * p.group + lane; i < end; i += 64) top = Top::join(top, magnitude(value(i)));
    const Q8Group g = q8_group(over_lanes<Top, 64>(top));
    for (int32_t i = j * p.group + lane; i < end; i += 64) gst<int8_t>(q + i, (int8_t)q8_round(value(i), g));
    if (lane == 0) gst<float>(s + j, g.scale);
  }
}

template <bool BF16>
__global__ __launch_bounds__(QT) void q8_quantize_any_kernel(Q8Params p) {
  __shared__ uint32_t tops[QW];
  for (int64_t t = blockIdx.x; t < p.tokens; t += gridDim.x)
    quantize_row(p, t, p.f, tops, [&](int32_t i) { return rounded<BF16>(h_of<BF16>(p, t * p.ldz, i)); });
}

template <bool BF16>
__global__ __launch_bounds__(QT) void q8_act_any_kernel(Q8Params p) {
  __shared__ uint32_t tops[QW];
  for (int64_t t = blockIdx.x; t < p.tokens; t += gridDim.x) {
    if (p.h)
      for (int32_t i = threadIdx.x; i < p.f; i += QT) store1<BF16>(p.h, t * p.ldh + i, h_of<BF16>(p, t * p.ldz, i));
    quantize_row(p, t, p.gated ? 2 * p.f : p.f, tops,
                 [&](int32_t i) { return load1<BF16>(p.z, t * p.ldz + i); });
  }
}

// A thread to an entry of h; a workgroup row takes `take` tokens and stores its part of dbias.
template <bool BF16>
__global__ __launch_bounds__(QT) void q8_act_backward_any_kernel(Q8Params p, int64_t take, float* part) {
  const int32_t i = blockIdx.x * QT + threadIdx.x;
  if (i >= p.f) return;
  const int32_t wide = p.gated ? 2 * p.f : p.f;
  const int32_t ga = p.group ? i / p.group : 0, gu = p.group ? (p.f + i) / p.group : 0;
  float da = 0.0f, du = 0.0f;
  const int64_t end = min((blockIdx.y + 1) * take, p.tokens);
  for (int64_t t = blockIdx.y * take; t < end; ++t) {
    const float* s = p.s + t * p.lds;
    const int8_t* q = p.q + t * p.ldq;
    const float a = (float)gld<int8_t>(q + i) * gld<float>(s + ga), g = load1<BF16>(p.gh, t * p.ldgh + i);
    const float u = p.gated ? (float)gld<int8_t>(q + p.f + i) * gld<float>(s + gu) : 1.0f;
    float value, slope;
    act_both(a, p.act, value, slope);
    const float dza = p.gated ? g * u * slope : g * slope, dzu = g * value;
    da += dza;
    du += dzu;
    if (p.dz) {
      store1<BF16>(p.dz, t * p.lddz + i, dza);
      if (p.gated) store1<BF16>(p.dz, t * p.lddz + p.f + i, dzu);
    }
    if (p.h) store1<BF16>(p.h, t * p.ldh + i, p.gated ? value * u : value);
  }
  if (!part) return;
  float* to = part + (int64_t)blockIdx.y * wide;
  gst<float>(to + i, da);
  if (p.gated) gst<float>(to + p.f + i, du);
}

// ---- rows in registers ----------------------------------------------------------------------------
// A row of 8 entries or more belongs to W wavefronts, C chunks of 8 to a lane (a workgroup has one row, or
// four where W is 1).  A group of 16 to 512 entries is 2 to 64 lanes, its maximum a few register permutes; a
// whole row's goes through LDS.

// The largest magnitudes of the groups that a lane's chunks are in (`wide`: of its row).
template <int W, int C>
__device__ __forceinline__ void tops_of(const Q8Params& p, uint32_t (&top)[C], uint32_t* part) {
  if (p.group) {
#pragma unroll
    for (int k = 0; k < C; ++k) top[k] = over_lanes<Top>(top[k], p.group / 8);
    return;
  }
  uint32_t all = top[0];
#pragma unroll
  for (int k = 1; k < C; ++k) all = Top::join(all, top[k]);
  all = over_group<Top, W>(all, part);
#pragma unroll
  for (int k = 0; k < C; ++k) top[k] = all;
}
// Chunk c in 8 bits, and its group's scale by the lane that has the group's first chunk.  The chunk is number
// `chunk` of the row, which starts `from` entries before the chunks are counted (the second half of a gated row).
template <bool WHOLE>
__device__ __forceinline__ void give8(const Q8Params& p, int64_t t, int32_t from, int32_t chunk, const Place& c,
                                      const float (&v)[8], uint32_t top) {
  const Q8Group g = q8_group(top);
  store_q8<WHOLE>(p.q + t * p.ldq + from, c, v, g);
  const int32_t start = from + chunk * 8;
  if (!c.none() && (p.group ? start % p.group == 0 : start == 0))
    gst<float>(p.s + t * p.lds + (p.group ? start / p.group : 0), g.scale);
}

// HALVES: h and both halves of a gated row go chunk by chunk together (whole chunks and groups in each half);
// SPLIT: the row in 8 bits first, then h, whose chunks lie otherwise.
enum { QUANTIZE, PLAIN, HALVES, SPLIT };
template <bool BF16, int W, int C, bool WHOLE, int HOW, int KIND>
__global__ __launch_bounds__(W == 1 ? QT : 64 * W) void q8_row_kernel(Q8Params p) {
  constexpr int R = W == 1 ? QW : 1;
  constexpr int IN = HOW == STREAM && KIND != SPLIT ? STREAM : CACHED, OUT = KIND == QUANTIZE ? CACHED : HOW;
  __shared__ uint32_t part[W];
  const int32_t sub = W == 1 ? __builtin_amdgcn_readfirstlane(threadIdx.x >> 6) : 0;
  const int32_t lane = threadIdx.x & 63, wave = W == 1 ? 0 : threadIdx.x >> 6;
  const bool two = KIND == HALVES || (KIND == QUANTIZE && p.gated);
  Place c[C];
  places<W, C>(KIND == SPLIT ? 2 * p.f : p.f, c);
  for (int64_t t = (int64_t)blockIdx.x * R + sub; t < p.tokens; t += (int64_t)gridDim.x * R) {
    Raw<BF16> ar[C], ur[C];
#pragma unroll
    for (int k = 0; k < C; ++k) ar[k] = load_raw<BF16, IN>(p.z, t * p.ldz + c[k].at);
    if (two) {
#pragma unroll
      for (int k = 0; k < C; ++k) ur[k] = load_raw<BF16, IN>(p.z, t * p.ldz + p.f + c[k].at);
    }
    float v[C][8], u[C][8];
    uint32_t top[C], top_u[C];
#pragma unroll
    for (int k = 0; k < C; ++k) {
      mask<WHOLE>(c[k], ar[k]);
      widen<BF16>(ar[k], v[k]);
      if (two) {
        mask<WHOLE>(c[k], ur[k]);
        widen<BF16>(ur[k], u[k]);
      }
      if (KIND == QUANTIZE || ((KIND == PLAIN || KIND == HALVES) && p.h)) {
        float h[8];
#pragma unroll
        for (int e = 0; e < 8; ++e) {
          h[e] = act_value(v[k][e], p.act);
          if (two) h[e] *= u[k][e];
        }
        const Raw<BF16> r = narrow<BF16>(h);
        if constexpr (KIND == QUANTIZE) {
          ar[k] = r;
          widen<BF16>(r, v[k]);
        } else {
          store_raw<BF16, WHOLE, OUT>(p.h, t * p.ldh, c[k], r);
        }
      }
      top[k] = top8<BF16>(ar[k]);
      if (KIND == HALVES) top_u[k] = top8<BF16>(ur[k]);
    }
    if (KIND == HALVES && !p.group) {
#pragma unroll
      for (int k = 0; k < C; ++k) top[k] = Top::join(top[k], top_u[k]);
    }
    tops_of<W>(p, top, part);
    if (KIND == HALVES) {
#pragma unroll
      for (int k = 0; k < C; ++k) top_u[k] = p.group ? over_lanes<Top>(top_u[k], p.group / 8) : top[k];
    }
#pragma unroll
    for (int k = 0; k < C; ++k) {
      const int32_t chunk = (k * W + wave) * 64 + lane;
      give8<WHOLE>(p, t, 0, chunk, c[k], v[k], top[k]);
      if (KIND == HALVES) give8<WHOLE>(p, t, p.f, chunk, c[k], u[k], top_u[k]);
    }
    if (KIND == SPLIT && p.h) {
      for (int32_t i = (wave * 64 + lane) * 8; i < p.f; i += 8 * 64 * W) {
        const Place at(i / 8, p.f);
        float a[8], b[8];
        widen<BF16>(load_raw<BF16, CACHED>(p.z, t * p.ldz + at.at), a);
        widen<BF16>(load_raw<BF16, CACHED>(p.z, t * p.ldz + p.f + at.at), b);
#pragma unroll
        for (int e = 0; e < 8; ++e) a[e] = act_value(a[e], p.act) * b[e];
        store_raw<BF16, false, OUT>(p.h, t * p.ldh, at, narrow<BF16>(a));
      }
    }
    if constexpr (W > 1) __syncthreads();   // the maximum's places are free for the next row
  }
}

// ---- backward -----------------------------------------------------------------------------------
// No sum over a row is needed: a workgroup has 512 entries of h (and the same of the other half) of the tokens
// of its part, its four wavefronts the tokens in turn, U of them in flight, and keeps their sums of dz.
template <int N>
__device__ __forceinline__ void dequantize(const int8_t* q, const float* s, int32_t group, int32_t at, float (&v)[N]) {
  const u32x2_a1 w = gld<u32x2_a1>(q + at);
  const int32_t g0 = group ? at / group : 0, g1 = group ? (at + 7) / group : 0;
  const float s0 = gld<float>(s + g0), s1 = gld<float>(s + g1);
  const int32_t turn = group ? g1 * group - at : 8;   // entries of the first group
#pragma unroll
  for (int e = 0; e < 8; ++e)
    v[e] = (float)(int8_t)(w[e / 4] >> (8 * (e % 4))) * (e < turn || g0 == g1 ? s0 : s1);
}

template <bool BF16, bool WHOLE, int HOW, bool GATED>
__global__ __launch_bounds__(QT) void q8_backward_kernel(Q8Params p, int64_t take, float* part) {
  constexpr int U = 2;
  __shared__ float joined[QW - 1][GATED ? 16 : 8][64];
  const int32_t wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), lane = threadIdx.x & 63;
  const Place c(blockIdx.x * 64 + lane, p.f);
  float da[8] = {}, du[8] = {};
  const int64_t end = min((blockIdx.y + 1) * take, p.tokens);
  for (int64_t t0 = blockIdx.y * take + wave * U; t0 < end; t0 += QW * U) {
    Raw<BF16> gr[U];
    float a[U][8], u[U][8];
#pragma unroll
    for (int k = 0; k < U; ++k) {
      const int64_t t = min(t0 + k, end - 1);
      gr[k] = load_raw<BF16, HOW>(p.gh, t * p.ldgh + c.at);
      dequantize(p.q + t * p.ldq, p.s + t * p.lds, p.group, c.at, a[k]);
      if (GATED) dequantize(p.q + t * p.ldq, p.s + t * p.lds, p.group, p.f + c.at, u[k]);
    }
#pragma unroll
    for (int k = 0; k < U; ++k) {
      const int64_t t = t0 + k;
      if (t >= end) break;
      float g[8], z[8], h[8];
      widen<BF16>(gr[k], g);
#pragma unroll
      for (int e = 0; e < 8; ++e) {
        float value, slope;
        act_both(a[k][e], p.act, value, slope);
        const float du_e = g[e] * value;
        z[e] = (GATED ? g[e] * u[k][e] : g[e]) * slope;
        h[e] = GATED ? value * u[k][e] : value;
        da[e] += z[e];
        if (GATED) {
          du[e] += du_e;
          u[k][e] = du_e;
        }
      }
      if (p.dz) {
        store_raw<BF16, WHOLE, HOW>(p.dz, t * p.lddz, c, narrow<BF16>(z));
        if (GATED) store_raw<BF16, WHOLE, HOW>(p.dz, t * p.lddz + p.f, c, narrow<BF16>(u[k]));
      }
      if (p.h) store_raw<BF16, WHOLE, HOW>(p.h, t * p.ldh, c, narrow<BF16>(h));
    }
  }
  if (!part) return;
  if (wave > 0) {   // the four wavefronts' sums, in order
#pragma unroll
    for (int e = 0; e < 8; ++e) {
      joined[wave - 1][e][lane] = da[e];
      if (GATED) joined[wave - 1][8 + e][lane] = du[e];
    }
  }
  __syncthreads();
  if (wave > 0) return;
#pragma unroll
  for (int w = 0; w < QW - 1; ++w)
#pragma unroll
    for (int e = 0; e < 8; ++e) {
      da[e] += joined[w][e][lane];
      if (GATED) du[e] += joined[w][8 + e][lane];
    }
  const int64_t row = (int64_t)blockIdx.y * (GATED ? 2 * p.f : p.f);
  store_raw<false, WHOLE, CACHED>(part, row, c, narrow<false>(da));
  if (GATED) store_raw<false, WHOLE, CACHED>(part, row + p.f, c, narrow<false>(du));
}

// ---- launches -------------------------------------------------------------------------------------
// The backward pass' parts of dbias: `take` tokens each; 1024 workgroups, at least 8 tokens each.
struct BackPlan {
  int64_t take, parts;
  explicit BackPlan(const Q8Params& p) {
    const int64_t slabs = ceil_div(p.f, 512);
    const int64_t want = 1024 / slabs;
    take = ceil_div(p.tokens, min64(want < 64 ? 64 : want, ceil_div(p.tokens, 8)));
    parts = ceil_div(p.tokens, take);
  }
};

// How `in` and `out` bytes go through the caches: outputs beyond the L2s' reach past their replacement, and
// where all is more than half of the last-level cache inputs too (a GELU kept and its backward pass, 4096
// features bf16: 1024 tokens 21.4 us, 19.2 and 20.3; 4096 tokens 54.9, 44.2 and 49.5; 8192 tokens 95.3, 88.1
// and 86.2).
template <typename F>
void by_how(int64_t in, int64_t out, const F& f) {
  if (out <= 8 * MB) f(IntC<CACHED>());
  else if (in + out <= 128 * MB) f(IntC<STREAM_OUT>());
  else f(IntC<STREAM>());
}
// f(wavefronts of a row, chunks of a lane) for rows of `width` entries.
template <typename F>
void by_width(int32_t width, const F& f) {
  const int32_t chunks = (width + 511) / 512;
  if (chunks <= 1) return f(IntC<1>(), IntC<1>());
  if (chunks <= 2) return f(IntC<1>(), IntC<2>());
  if (chunks <= 4) return f(IntC<2>(), IntC<2>());
  if (chunks <= 8) return f(IntC<4>(), IntC<2>());
  if (chunks <= 16) return f(IntC<8>(), IntC<2>());
  if (chunks <= 32) return f(IntC<16>(), IntC<2>());
  f(IntC<16>(), IntC<4>());
}
constexpr int32_t MOST_ROW = 32768;   // entries of a row in registers

template <int KIND>
void launch_rows(const Q8Params& p, int64_t in, int64_t out, hipStream_t stream) {
  by_type(p.bf16, p.f, [&](auto bf16, auto whole) {
    const auto by_kind = [&](const auto& f) {   // (8-bit rows for a product are read next: kept)
      if constexpr (KIND == QUANTIZE) in + out > 128 * MB ? f(IntC<STREAM>()) : f(IntC<CACHED>());
      else if constexpr (KIND == SPLIT) out > 8 * MB ? f(IntC<STREAM_OUT>()) : f(IntC<CACHED>());
      else by_how(in, out, f);
    };
    by_kind([&](auto how) {
      by_width(KIND == SPLIT ? 2 * p.f : p.f, [&](auto w, auto c) {
        constexpr int W = decltype(w)::value, C = decltype(c)::value, R = W == 1 ? QW : 1;
        hipLaunchKernelGGL((q8_row_kernel<decltype(bf16)::value, W, C, KIND != SPLIT && decltype(whole)::value,
                                          decltype(how)::value, KIND>),
                           dim3((uint32_t)min64(ceil_div(p.tokens, R), 1 << 20)), dim3(W == 1 ? QT : 64 * W), 0,
                           stream, p);
      });
    });
  });
}
dim3 rows_grid(const Q8Params& p) { return dim3((uint32_t)min64(p.tokens, 1 << 20)); }

}  // namespace

hipError_t launch_q8_quantize(const Q8Params& p, hipStream_t stream) {
  const int64_t es = p.bf16 ? 2 : 4;
  if (p.f >= 8 && p.f <= MOST_ROW)
    launch_rows<QUANTIZE>(p, p.tokens * (p.f << p.gated) * es, p.tokens * p.f, stream);
  else if (p.bf16)
    hipLaunchKernelGGL((q8_quantize_any_kernel<true>), rows_grid(p), dim3(QT), 0, stream, p);
  else
    hipLaunchKernelGGL((q8_quantize_any_kernel<false>), rows_grid(p), dim3(QT), 0, stream, p);
  return hipGetLastError();
}

hipError_t launch_q8_act(const Q8Params& p, hipStream_t stream) {
  const int64_t es = p.bf16 ? 2 : 4, wide = (int64_t)p.f << p.gated;
  const int64_t in = p.tokens * wide * es, out = p.tokens * (p.f * es + wide);
  const bool halves = p.gated && p.f % 8 == 0 && (p.group == 0 || p.f % p.group == 0);
  if (p.f >= 8 && !p.gated && p.f <= MOST_ROW)
    launch_rows<PLAIN>(p, in, out, stream);
  else if (p.f >= 8 && halves && p.f <= MOST_ROW)
    launch_rows<HALVES>(p, in, out, stream);
  else if (p.f >= 8 && p.gated && 2 * p.f <= MOST_ROW)
    launch_rows<SPLIT>(p, in, out, stream);
  else if (p.bf16)
    hipLaunchKernelGGL((q8_act_any_kernel<true>), rows_grid(p), dim3(QT), 0, stream, p);
  else
    hipLaunchKernelGGL((q8_act_any_kernel<false>), rows_grid(p), dim3(QT), 0, stream, p);
  return hipGetLastError();
}

int64_t q8_backward_work_floats(const Q8Params& p) {
  return p.dbias ? BackPlan(p).parts * ((int64_t)p.f << p.gated) : 0;
}

hipError_t launch_q8_act_backward(const Q8Params& p, float* work, hipStream_t stream) {
  const BackPlan b(p);
  float* part = p.dbias ? work : nullptr;
  const int64_t es = p.bf16 ? 2 : 4, wide = (int64_t)p.f << p.gated;
  if (p.f >= 8) {
    const dim3 grid((uint32_t)ceil_div(p.f, 512), (uint32_t)b.parts);
    by_type(p.bf16, p.f, [&](auto bf16, auto whole) {
      by_how(p.tokens * (p.f * es + wide), p.tokens * (p.f + wide) * es, [&](auto how) {
        const auto launch = [&](auto gated) {
          hipLaunchKernelGGL((q8_backward_kernel<decltype(bf16)::value, decltype(whole)::value, decltype(how)::value,
                                                 decltype(gated)::value>),
                             grid, dim3(QT), 0, stream, p, b.take, part);
        };
        if (p.gated) launch(std::true_type());
        else launch(std::false_type());
      });
    });
  } else {
    const dim3 grid(1, (uint32_t)b.parts);
    if (p.bf16)
      hipLaunchKernelGGL((q8_act_backward_any_kernel<true>), grid, dim3(QT), 0, stream, p, b.take, part);
    else
      hipLaunchKernelGGL((q8_act_backward_any_kernel<false>), grid, dim3(QT), 0, stream, p, b.take, part);
  }
  if (!part) return hipGetLastError();
  FoldParams fold = {};
  fold.width = (int32_t)wide;
  fold.n = 1;
  fold.job[0] = {part, b.parts, 1, p.dbias, 0, 0, 0, nullptr, 0};
  return launch_fold(fold, stream);
}

}  // namespace tpp

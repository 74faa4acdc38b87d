// residual_kernels.hip -- the residual stream's norms, forward and backward, for gfx950.
//
// Forward: r = x + scale G(g) N_after(b), y = N_before(r): two norms over a token's features, a few
// operations an entry of 2 or 4 bytes.  Backward, with vn the normed row without its vector w, u = g w:
//     N'(g) = (u - vn mean(u vn) - mean(u)) / sqrt(..)      (mean(u): layer norm only)
// for the norm before first, whose result is dx, then for the norm after of scale G dx.
// The vectors' and the gate's gradients are sums over tokens: workgroups keep them for the tokens that
// they take and store one partial row each, which a second kernel adds in order (no atomics: the bits do
// not vary between runs).
#include <hip/hip_runtime.h>

#include "internal.h"
#include "rows_device.h"

namespace tpp {
namespace {

using namespace rows;

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
  return p.gate_every ? t / p.gate_every : 0;
}

// ---- any width ------------------------------------------------------------------------------------
// A workgroup to a token; rows are read again for each sum.

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

// Gradients of x and b, and what the sums over tokens need of a row: the means and factors of both norms,
// mean(u vn) and mean(u) of the norm before.
constexpr int STATS = 6;
template <bool BF16>
__global__ __launch_bounds__(RT) void residual_backward_any_kernel(ResidualParams p, float* stats) {
  __shared__ float part[RW];
  for (int64_t t = blockIdx.x; t < p.tokens; t += gridDim.x) {
    float mr, rr, mb, rb, uv = 0.0f, u0 = 0.0f;
    row_stats<BF16>(p, p.r, t * p.ldr, p.gy ? p.before : TPP_NORM_NONE, part, mr, rr);
    row_stats<BF16>(p, p.b, t * p.ldb, p.after, part, mb, rb);
    if (p.gy && p.before != TPP_NORM_NONE) {
      for (int32_t i = threadIdx.x; i < p.f; i += RT) {
        const float u = load1<BF16>(p.gy, t * p.ldgy + i) * gld<float>(p.wb + i);
        uv += u * (load1<BF16>(p.r, t * p.ldr + i) - mr) * rr;
        u0 += u;
      }
      uv = over_group<Sum, RW>(uv, part) / (float)p.f;
      __syncthreads();
      u0 = p.before == TPP_NORM_LAYER ? over_group<Sum, RW>(u0, part) / (float)p.f : 0.0f;
      __syncthreads();
    }
    const auto total = [&](int32_t i) {
      float g = p.gr ? load1<BF16>(p.gr, t * p.ldgr + i) : 0.0f;
      if (!p.gy) return g;
      const float y = load1<BF16>(p.gy, t * p.ldgy + i);
      if (p.before == TPP_NORM_NONE) return g + y;
      const float vn = (load1<BF16>(p.r, t * p.ldr + i) - mr) * rr;
      return g + rr * (y * gld<float>(p.wb + i) - vn * uv - u0);
    };
    const int64_t g0 = gate_row(p, t) * p.ldg;
    const auto branch = [&](int32_t i) {   // gradient of N_after(b), times its vector
      float g = p.scale * total(i);
      if (p.gate_form) g *= gate_value(load1(p.gate, g0 + i, p.gate_bf16), p.gate_form);
      return p.after == TPP_NORM_NONE ? g : g * gld<float>(p.wa + i);
    };
    float bv = 0.0f, b0 = 0.0f;
    if (p.after != TPP_NORM_NONE) {
      for (int32_t i = threadIdx.x; i < p.f; i += RT) {
        const float u = branch(i);
        bv += u * (load1<BF16>(p.b, t * p.ldb + i) - mb) * rb;
        b0 += u;
      }
      bv = over_group<Sum, RW>(bv, part) / (float)p.f;
      __syncthreads();
      b0 = p.after == TPP_NORM_LAYER ? over_group<Sum, RW>(b0, part) / (float)p.f : 0.0f;
      __syncthreads();
    }
    for (int32_t i = threadIdx.x; i < p.f; i += RT) {
      if (p.dx) store1<BF16>(p.dx, t * p.lddx + i, total(i));
      if (p.db) {
        const float vn = (load1<BF16>(p.b, t * p.ldb + i) - mb) * rb, u = branch(i);
        store1<BF16>(p.db, t * p.lddb + i, p.after == TPP_NORM_NONE ? u : rb * (u - vn * bv - b0));
      }
    }
    if (stats && threadIdx.x == 0) {
      const float s[STATS] = {mr, rr, mb, rb, uv, u0};
#pragma unroll
      for (int k = 0; k < STATS; ++k) gst<float>(stats + t * STATS + k, s[k]);
    }
  }
}

// How the sums over tokens are cut: segments of up to `rows` tokens that no gate's border crosses, `per`
// of them to a gate, `take` segments to a workgroup's partial row.
struct Cut {
  int64_t every, rows, per, segments, take, parts;
};
int64_t ceil_div(int64_t a, int64_t b) { return (a + b - 1) / b; }
Cut cut_tokens(const ResidualParams& p, int64_t most_parts) {
  Cut c;
  c.every = p.gate_every && p.gate_form ? p.gate_every : p.tokens;
  if (c.every > p.tokens) c.every = p.tokens;
  const int64_t want = ceil_div(p.tokens, most_parts);
  c.per = ceil_div(c.every, want);
  c.rows = ceil_div(c.every, c.per);
  c.segments = ceil_div(p.tokens, c.every) * c.per;
  c.take = ceil_div(c.segments, most_parts);
  c.parts = ceil_div(c.segments, c.take);
  return c;
}

// Sums over tokens, a thread to a feature: part[vector][workgroup row][feature] of the four vectors, and
// gate_part[segment][feature] (or dgate itself where a gate has one segment).
template <bool BF16>
__global__ __launch_bounds__(RT) void residual_columns_any_kernel(ResidualParams p, Cut c, const float* stats,
                                                                  float* part, float* gate_part) {
  const int32_t i = blockIdx.x * RT + threadIdx.x;
  if (i >= p.f) return;
  const float wa = p.after != TPP_NORM_NONE ? gld<float>(p.wa + i) : 1.0f;
  const float ca = p.after == TPP_NORM_LAYER && p.ca ? gld<float>(p.ca + i) : 0.0f;
  const float wb = p.gy && p.before != TPP_NORM_NONE ? gld<float>(p.wb + i) : 1.0f;
  for (int64_t row = blockIdx.y; row < c.parts; row += gridDim.y) {
    float sum[4] = {0.0f, 0.0f, 0.0f, 0.0f};
    const int64_t s_end = min((row + 1) * c.take, c.segments);
    for (int64_t s = row * c.take; s < s_end; ++s) {
      const int64_t gate = s / c.per, t0 = gate * c.every + (s - gate * c.per) * c.rows;
      const int64_t t1 = min(min(t0 + c.rows, (gate + 1) * c.every), p.tokens);
      float g = 1.0f, g_sum = 0.0f;
      const float g_in = p.gate_form ? load1(p.gate, gate * p.ldg + i, p.gate_bf16) : 0.0f;
      if (p.gate_form) g = gate_value(g_in, p.gate_form);
      for (int64_t t = t0; t < t1; ++t) {
        const float* st = stats + t * STATS;
        float d = p.gr ? load1<BF16>(p.gr, t * p.ldgr + i) : 0.0f;
        if (p.gy) {
          const float y = load1<BF16>(p.gy, t * p.ldgy + i);
          if (p.before == TPP_NORM_NONE) {
            d += y;
          } else {
            const float vn = (load1<BF16>(p.r, t * p.ldr + i) - st[0]) * st[1];
            d += st[1] * (y * wb - vn * st[4] - st[5]);
            sum[2] += y * vn;
            sum[3] += y;
          }
        }
        d *= p.scale;
        const float bn = (load1<BF16>(p.b, t * p.ldb + i) - st[2]) * st[3];
        g_sum += d * (bn * wa + ca);
        sum[0] += d * g * bn;
        sum[1] += d * g;
      }
      if (p.dgate) {
        if (gate_part) gst<float>(gate_part + s * p.f + i, g_sum);
        else
          store1(p.dgate, gate * p.lddg + i, g_sum * gate_slope(g_in, p.gate_form), p.gate_bf16);
      }
    }
    int32_t k = 0;
#pragma unroll
    for (int v = 0; v < 4; ++v)
      if (p.dv[v]) gst<float>(part + ((int64_t)k++ * c.parts + row) * p.f + i, sum[v]);
  }
}

// ---- the sums' second half --------------------------------------------------------------------------
// A workgroup has 16 columns of one output row; 16 sets of 16 lanes take every 16th part, 4 in flight,
// and meet pairwise.
constexpr int FE = 16, FS = RT / FE;
__global__ __launch_bounds__(RT) void fold_kernel(FoldParams p) {
  __shared__ float acc[FS][FE];
  const FoldJob& j = p.job[blockIdx.z];
  const int32_t set = threadIdx.x / FE, lane = threadIdx.x % FE, c = blockIdx.x * FE + lane;
  for (int64_t row = blockIdx.y; row < j.rows; row += gridDim.y) {
    const float* from = j.from + row * j.parts * p.width + c;
    float sum = 0.0f;
    for (int64_t i = set; i < j.parts; i += 4 * FS) {
      float x[4];
#pragma unroll
      for (int u = 0; u < 4; ++u)
        x[u] = c < p.width && i + u * FS < j.parts ? gld<float>(from + (i + u * FS) * p.width) : 0.0f;
#pragma unroll
      for (int u = 0; u < 4; ++u) sum += x[u];
    }
    acc[set][lane] = sum;
    __syncthreads();
#pragma unroll
    for (int h = FS / 2; h > 0; h /= 2) {
      if (set < h) acc[set][lane] += acc[set + h][lane];
      __syncthreads();
    }
    if (set == 0 && c < p.width) {
      float v = acc[0][lane];
      if (j.slope) v *= gate_slope(load1(j.gate, row * j.ldg + c, j.bf16), j.slope);
      store1(j.to, row * j.ld + c, v, j.bf16);
    }
    __syncthreads();
  }
}

__global__ __launch_bounds__(RT) void zeros_kernel(void* to, int64_t n, int32_t bf16) {
  const int64_t i = (int64_t)blockIdx.x * RT + threadIdx.x;
  if (i < n) store1(to, i, 0.0f, bf16);
}

constexpr int64_t MOST_PARTS = 256;

int vectors_of(const ResidualParams& p) {
  int n = 0;
  for (const float* v : p.dv) n += v != nullptr;
  return n;
}
bool sums_wanted(const ResidualParams& p) { return vectors_of(p) > 0 || p.dgate; }

}  // namespace

hipError_t launch_fold(const FoldParams& p, hipStream_t stream) {
  int64_t rows = 1;
  for (int k = 0; k < p.n; ++k) rows = p.job[k].rows > rows ? p.job[k].rows : rows;
  const dim3 grid((uint32_t)((p.width + FE - 1) / FE), (uint32_t)(rows < 64 ? rows : 64), (uint32_t)p.n);
  hipLaunchKernelGGL(fold_kernel, grid, dim3(RT), 0, stream, p);
  return hipGetLastError();
}

hipError_t launch_zeros(void* to, int64_t n, bool bf16, hipStream_t stream) {
  hipLaunchKernelGGL(zeros_kernel, dim3((uint32_t)ceil_div(n, RT)), dim3(RT), 0, stream, to, n, bf16);
  return hipGetLastError();
}

hipError_t launch_residual_zeros(const ResidualParams& p, hipStream_t stream) {
  for (float* to : p.dv)
    if (to)
      if (const hipError_t e = launch_zeros(to, p.f, false, stream)) return e;
  return p.dgate && p.gate_every == 0 ? launch_zeros(p.dgate, p.f, p.gate_bf16, stream) : hipSuccess;
}

hipError_t launch_residual(const ResidualParams& p, hipStream_t stream) {
  const dim3 grid((uint32_t)(p.tokens < (1 << 20) ? p.tokens : (1 << 20)));
  if (p.bf16)
    hipLaunchKernelGGL((residual_any_kernel<true>), grid, dim3(RT), 0, stream, p);
  else
    hipLaunchKernelGGL((residual_any_kernel<false>), grid, dim3(RT), 0, stream, p);
  return hipGetLastError();
}

int64_t residual_backward_work_floats(const ResidualParams& p) {
  if (!sums_wanted(p)) return 0;
  const Cut c = cut_tokens(p, MOST_PARTS);
  return p.tokens * STATS + (vectors_of(p) * c.parts + (p.dgate && c.per > 1 ? c.segments : 0)) * p.f;
}

hipError_t launch_residual_backward(const ResidualParams& p, float* work, hipStream_t stream) {
  const dim3 grid((uint32_t)(p.tokens < (1 << 20) ? p.tokens : (1 << 20)));
  float* stats = sums_wanted(p) ? work : nullptr;
  if (p.bf16)
    hipLaunchKernelGGL((residual_backward_any_kernel<true>), grid, dim3(RT), 0, stream, p, stats);
  else
    hipLaunchKernelGGL((residual_backward_any_kernel<false>), grid, dim3(RT), 0, stream, p, stats);
  if (!stats) return hipGetLastError();
  const Cut c = cut_tokens(p, MOST_PARTS);
  const int n = vectors_of(p);
  float* part = work + p.tokens * STATS;
  float* gate_part = p.dgate && c.per > 1 ? part + n * c.parts * p.f : nullptr;
  const dim3 columns((uint32_t)ceil_div(p.f, RT), (uint32_t)c.parts);
  if (p.bf16)
    hipLaunchKernelGGL((residual_columns_any_kernel<true>), columns, dim3(RT), 0, stream, p, c, stats, part, gate_part);
  else
    hipLaunchKernelGGL((residual_columns_any_kernel<false>), columns, dim3(RT), 0, stream, p, c, stats, part, gate_part);
  FoldParams fold = {};
  fold.width = p.f;
  for (float* to : p.dv) {
    if (!to) continue;
    fold.job[fold.n] = {part + (int64_t)fold.n * c.parts * p.f, c.parts, 1, to, 0, 0, 0, nullptr, 0};
    ++fold.n;
  }
  if (gate_part)
    fold.job[fold.n++] = {gate_part, c.per, ceil_div(p.tokens, c.every), p.dgate, p.lddg, p.gate_bf16,
                          p.gate_form, p.gate, p.ldg};
  if (fold.n > 0) return launch_fold(fold, stream);
  return hipGetLastError();
}

}  // namespace tpp

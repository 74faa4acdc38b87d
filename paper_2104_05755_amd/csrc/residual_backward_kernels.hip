// residual_backward_kernels.hip -- the residual stream's norms, backward, for gfx950, and the second half of
// sums over tokens, which the 8-bit activations use too.
//
// With vn the normed row without its vector w and u = g w,
//     N'(g) = (u - vn mean(u vn) - mean(u)) / sqrt(..)      (mean(u): layer norm only)
// for the norm before first, whose result is dx, then for the norm after of scale G dx: about 40 operations an
// entry of 2 or 4 bytes, six of which are moved: bound by HBM, with the arithmetic near behind.  The vectors'
// and the gate's gradients are sums over tokens: workgroups keep them for the tokens that they take and store
// one partial row each, which a second kernel adds in order (no atomics: the bits do not vary between runs).
//
// 8192 tokens of 4096 bf16: 86 to 89 us, 4.5 to 4.7 TB/s, 4.7 of them the fold (a copy of as much: 78 us).  1533 of 1001
// fp32, layer norms and a gate for every 100 tokens: 24 us, where a copy takes 7.2: a row of parts for every two
// tokens is 16 MB beside the 37 that must move; the kernel, 17 us, waits half of the time in two turns of a loop
// with three exchanges, the fold, 7, fetches 32 MB (its columns of rows of 1001 share lines).  From a workgroup to a row
// and a second reading for the sums: 707 and 40 us.  One chunk of 8 entries to a lane carried best (85 us
// against 92 with two, and 35 against 49), as did 2048 wavefronts (4096: 92 us against 84, 1024: 103 against 86); a second token's
// rows under way gained little and cost elsewhere (84.0 against 85.2, but 31 against 29).
#include <hip/hip_runtime.h>

#include "residual_device.h"

namespace tpp {
namespace {

using namespace rows;

// ---- any width ------------------------------------------------------------------------------------
// Rows below 8 entries or above 16384: a workgroup to a token, which reads its row again for each sum.

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
Cut cut_tokens(const ResidualParams& p, int64_t most_parts) {
  Cut c;
  c.every = p.gate_every && p.gate_form ? p.gate_every : p.tokens;
  if (c.every > p.tokens) c.every = p.tokens;
  const int64_t want = ceil_div(p.tokens, most_parts);
  c.per = ceil_div(c.every, want);
  c.rows = ceil_div(c.every, c.per);
  c.segments = ceil_div(p.tokens, c.every) * c.per;
  c.take = want > c.rows ? want / c.rows : 1;
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

// ---- backward with the rows in registers ------------------------------------------------------------
// W wavefronts go through the tokens of their segments with C chunks to a lane, the next token's rows
// loaded while this one's are worked on.  With b and r without their means, rb and rr their factors and
// d = dx, an entry takes
//     t = rr y,  d = gr + t wb - rr^2 along r - rr level,   dwb += t r,
//     t = rb d,  A += t b,   u = t G scale wa,   db = u - along' b - level'
// The gate is one row in a segment, so A is all that its gradient and that of wa need: scale wa A G' and
// scale G A (and B = sum d for the shifts).  At its end every workgroup stores a row of parts.
template <int W>
struct Exchange {   // sums of a row's wavefronts: places of their own for each use and turn of the loop
  float at[2][3][4][W];
};
template <int W, int N>
__device__ __forceinline__ void row_sums(float (&v)[N], float (&part)[4][W]) {
#pragma unroll
  for (int n = 0; n < N; ++n) v[n] = over_lanes<Sum, 64>(v[n]);
  if constexpr (W > 1) {
    if ((threadIdx.x & 63) == 0) {
#pragma unroll
      for (int n = 0; n < N; ++n) part[n][threadIdx.x >> 6] = v[n];
    }
    __syncthreads();
#pragma unroll
    for (int n = 0; n < N; ++n) {
      v[n] = part[n][0];
#pragma unroll
      for (int w = 1; w < W; ++w) v[n] += part[n][w];
    }
  }
}

template <bool BF16, int C>
struct BackRows {
  Raw<BF16> b[C], r[C], gr[C], gy[C];
};
template <int C>
__device__ __forceinline__ void fill(float (&v)[C][8], float x) {
#pragma unroll
  for (int k = 0; k < C; ++k)
#pragma unroll
    for (int e = 0; e < 8; ++e) v[k][e] = x;
}

// MEANS: a layer norm is among the two.  SUMS: rows of up to 8192 entries; the sums of wider ones would not
// fit the registers: what they need of a row goes to `stats`, and a kernel of their own reads the rows again.
template <bool BF16, int W, int C, bool WHOLE, int HOW, bool MEANS, bool SUMS>
__global__ __launch_bounds__(W == 1 ? RT : 64 * W) void residual_backward_row_kernel(ResidualParams p, Cut cut,
                                                                                    float* part, float* gate_part,
                                                                                    float* stats) {
  constexpr int R = W == 1 ? RW : 1;
  constexpr bool AHEAD = SUMS && (C == 1 || (BF16 && !MEANS));   // (the others' registers are full)
  __shared__ Exchange<W> sums;
  __shared__ float joined[W == 1 ? RW : 1][W == 1 ? 512 * C : 1];
  const int32_t sub = W == 1 ? __builtin_amdgcn_readfirstlane(threadIdx.x >> 6) : 0;
  const float inv_f = 1.0f / (float)p.f;
  const bool after = p.after != TPP_NORM_NONE, before = p.before != TPP_NORM_NONE && p.gy;
  const bool after_mean = MEANS && p.after == TPP_NORM_LAYER, before_mean = MEANS && before && p.before == TPP_NORM_LAYER;
  Place c[C];
  places<W, C>(p.f, c);
  // the vectors of a row team's features, or, where registers are short, loaded where they are used
  constexpr int V = SUMS ? C : 1;
  float wb[V][8], dwa[C][8], dca[C][8], dwb[C][8], dcb[C][8];
  fill(wb, 1.0f);
  fill(dwa, 0.0f);
  fill(dca, 0.0f);
  fill(dwb, 0.0f);
  fill(dcb, 0.0f);
  if (SUMS && before) {
#pragma unroll
    for (int k = 0; k < V; ++k) load8(p.wb, c[k].at, wb[k]);
  }
  const auto load = [&](BackRows<BF16, C>& x, int64_t t) {
#pragma unroll
    for (int k = 0; k < C; ++k) {
      x.b[k] = load_raw<BF16, HOW>(p.b, t * p.ldb + c[k].at);
      if (before) x.r[k] = load_raw<BF16, HOW>(p.r, t * p.ldr + c[k].at);
      if (p.gr) x.gr[k] = load_raw<BF16, HOW>(p.gr, t * p.ldgr + c[k].at);
      if (p.gy) x.gy[k] = load_raw<BF16, HOW>(p.gy, t * p.ldgy + c[k].at);
    }
  };
  const int64_t unit = (int64_t)blockIdx.x * R + sub;
  const int64_t s_end = min((unit + 1) * cut.take, cut.segments);
  int32_t turn = 0;
  for (int64_t s = unit * cut.take; s < s_end; ++s) {
    const int64_t gate = s / cut.per, t0 = gate * cut.every + (s - gate * cut.per) * cut.rows;
    const int64_t t1 = min(min(t0 + cut.rows, (gate + 1) * cut.every), p.tokens);
    BackRows<BF16, C> raw = {};
    if (AHEAD && t0 < t1) load(raw, t0);
    float gw[V][8], A[C][8], B[C][8];   // gw = scale G wa
    fill(A, 0.0f);
    fill(B, 0.0f);
    const auto branch = [&](int k, float (&to)[8]) {
      float w[8], g[8];
      if (after) load8(p.wa, c[k].at, w);
      if (p.gate_form) load8(p.gate, gate * p.ldg + c[k].at, p.gate_bf16, g);
#pragma unroll
      for (int e = 0; e < 8; ++e)
        to[e] = p.scale * (p.gate_form ? gate_value(g[e], p.gate_form) : 1.0f) * (after ? w[e] : 1.0f);
    };
    if constexpr (SUMS) {
#pragma unroll
      for (int k = 0; k < V; ++k) branch(k, gw[k]);
    }
    for (int64_t t = t0; t < t1; ++t) {
      if constexpr (!AHEAD) load(raw, t);
      float b[C][8], r[C][8], d[C][8], y[C][8];
#pragma unroll
      for (int k = 0; k < C; ++k) {   // (what there is none of is zero)
        mask<WHOLE>(c[k], raw.b[k]);
        mask<WHOLE>(c[k], raw.r[k]);
        mask<WHOLE>(c[k], raw.gr[k]);
        mask<WHOLE>(c[k], raw.gy[k]);
        widen<BF16>(raw.b[k], b[k]);
        widen<BF16>(raw.r[k], r[k]);
        widen<BF16>(raw.gr[k], d[k]);
        widen<BF16>(raw.gy[k], y[k]);
      }
      if (AHEAD && t + 1 < t1) load(raw, t + 1);
      float (&part0)[4][W] = sums.at[turn][0], (&part1)[4][W] = sums.at[turn][1], (&part2)[4][W] = sums.at[turn][2];
      turn ^= 1;
      float mb = 0.0f, mr = 0.0f;
      if constexpr (MEANS) {
        float m[2] = {sum_of(b), sum_of(r)};
        row_sums<W>(m, part0);
        mb = after_mean ? m[0] * inv_f : 0.0f;
        mr = before_mean ? m[1] * inv_f : 0.0f;
#pragma unroll
        for (int k = 0; k < C; ++k) {
#pragma unroll
          for (int e = 0; e < 8; ++e) {
            b[k][e] -= mb;
            r[k][e] -= mr;
          }
          mask<WHOLE>(c[k], b[k]);
          mask<WHOLE>(c[k], r[k]);
        }
      }
      float q[MEANS ? 4 : 3] = {squares_of(b), squares_of(r), 0.0f};
#pragma unroll
      for (int k = 0; k < C; ++k) {
        if (!SUMS && before) load8(p.wb, c[k].at, wb[0]);
#pragma unroll
        for (int e = 0; e < 8; ++e) {
          const float u = y[k][e] * wb[SUMS ? k : 0][e];
          q[2] = __builtin_fmaf(u, r[k][e], q[2]);
          if constexpr (MEANS) q[3] += u;
        }
      }
      row_sums<W>(q, part1);
      const float rb = after ? rsqrt_of(q[0] * inv_f + p.eps) : 1.0f;
      const float rr = before ? rsqrt_of(q[1] * inv_f + p.eps) : 1.0f;
      const float along_r = before ? -(q[2] * inv_f * rr * rr) * rr : 0.0f;
      const float level_r = before_mean ? q[MEANS ? 3 : 0] * inv_f * rr : 0.0f;
      if constexpr (!SUMS) {
        if (stats && threadIdx.x == 0) {
          const float st[STATS] = {mr, rr, mb, rb, before ? q[2] * inv_f * rr : 0.0f,
                                   before_mean ? q[MEANS ? 3 : 0] * inv_f : 0.0f};
#pragma unroll
          for (int k = 0; k < STATS; ++k) gst<float>(stats + t * STATS + k, st[k]);
        }
      }
      float o[MEANS ? 2 : 1] = {0.0f};
#pragma unroll
      for (int k = 0; k < C; ++k) {
        if constexpr (!SUMS) {
          if (before) load8(p.wb, c[k].at, wb[0]);
          branch(k, gw[0]);
        }
#pragma unroll
        for (int e = 0; e < 8; ++e) {
          const float ty = y[k][e] * rr;
          if constexpr (SUMS) dwb[k][e] = __builtin_fmaf(ty, r[k][e], dwb[k][e]);
          d[k][e] = __builtin_fmaf(along_r, r[k][e], __builtin_fmaf(ty, wb[SUMS ? k : 0][e], d[k][e]));
          if constexpr (MEANS) {
            if constexpr (SUMS) dcb[k][e] += y[k][e];
            d[k][e] -= level_r;
          }
        }
        if (MEANS) mask<WHOLE>(c[k], d[k]);
        if (p.dx) store_raw<BF16, WHOLE, HOW>(p.dx, t * p.lddx, c[k], narrow<BF16>(d[k]));
#pragma unroll
        for (int e = 0; e < 8; ++e) {
          if constexpr (MEANS && SUMS) B[k][e] += d[k][e];
          const float td = d[k][e] * rb;
          if constexpr (SUMS) A[k][e] = __builtin_fmaf(td, b[k][e], A[k][e]);
          d[k][e] = td * gw[SUMS ? k : 0][e];
          o[0] = __builtin_fmaf(d[k][e], b[k][e], o[0]);
          if constexpr (MEANS) o[1] += d[k][e];
        }
      }
      if (!p.db) continue;
      float along_b = 0.0f, level_b = 0.0f;
      if (after) {
        row_sums<W>(o, part2);
        along_b = -(o[0] * inv_f * rb) * rb;
        if (after_mean) level_b = o[MEANS ? 1 : 0] * inv_f;
      }
#pragma unroll
      for (int k = 0; k < C; ++k) {
#pragma unroll
        for (int e = 0; e < 8; ++e) {
          d[k][e] = __builtin_fmaf(along_b, b[k][e], d[k][e]);
          if constexpr (MEANS) d[k][e] -= level_b;
        }
        store_raw<BF16, WHOLE, HOW>(p.db, t * p.lddb, c[k], narrow<BF16>(d[k]));
      }
    }
    if constexpr (!SUMS) continue;
#pragma unroll
    for (int k = 0; k < C; ++k) {
      float g[8], w[8], ca[8];
      if (p.gate_form) load8(p.gate, gate * p.ldg + c[k].at, p.gate_bf16, g);
      if (p.dgate) {
        if (after) load8(p.wa, c[k].at, w);
        const bool shift = after_mean && p.ca;
        if (shift) load8(p.ca, c[k].at, ca);
        float v[8];
#pragma unroll
        for (int e = 0; e < 8; ++e) {
          v[e] = p.scale * (A[k][e] * (after ? w[e] : 1.0f) + (shift ? B[k][e] * ca[e] : 0.0f));
          if (!gate_part) v[e] *= gate_slope(g[e], p.gate_form);
        }
        if (gate_part)
          store_raw<false, WHOLE, CACHED>(gate_part, s * p.f, c[k], narrow<false>(v));
        else if (p.gate_bf16)
          store_raw<true, WHOLE, CACHED>(p.dgate, gate * p.lddg, c[k], narrow<true>(v));
        else
          store_raw<false, WHOLE, CACHED>(p.dgate, gate * p.lddg, c[k], narrow<false>(v));
      }
#pragma unroll
      for (int e = 0; e < 8; ++e) {
        const float gs = p.scale * (p.gate_form ? gate_value(g[e], p.gate_form) : 1.0f);
        dwa[k][e] = __builtin_fmaf(gs, A[k][e], dwa[k][e]);
        if constexpr (MEANS) dca[k][e] = __builtin_fmaf(gs, B[k][e], dca[k][e]);
      }
    }
  }
  if constexpr (!SUMS) return;
  int32_t n = 0;
  const auto give = [&](int v, const float (&sum)[C][8]) {
    if (!p.dv[v]) return;
    const int64_t row = ((int64_t)n++ * gridDim.x + blockIdx.x) * p.f;
    if constexpr (W > 1) {
#pragma unroll
      for (int k = 0; k < C; ++k) store_raw<false, WHOLE, CACHED>(part, row, c[k], narrow<false>(sum[k]));
    } else {   // the four wavefronts' sums, in order
#pragma unroll
      for (int k = 0; k < C; ++k)
#pragma unroll
        for (int e = 0; e < 8; ++e)
          if (e >= c[k].skip) joined[sub][c[k].at + e] = sum[k][e];
      __syncthreads();
      for (int32_t i = threadIdx.x; i < p.f; i += RT)
        gst<float>(part + row + i, ((joined[0][i] + joined[1][i]) + joined[2][i]) + joined[3][i]);
      __syncthreads();
    }
  };
  give(0, dwa);
  give(1, dca);
  give(2, dwb);
  give(3, dcb);
}

// The sums of wide rows: a wavefront has 512 features of the tokens of a workgroup row.
template <bool BF16, bool WHOLE, bool MEANS>
__global__ __launch_bounds__(RT) void residual_columns_kernel(ResidualParams p, Cut cut, const float* stats,
                                                              float* part, float* gate_part) {
  const int32_t wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  const Place c((blockIdx.x * RW + wave) * 64 + (threadIdx.x & 63), p.f);
  if (c.none()) return;
  const bool after = p.after != TPP_NORM_NONE, before = p.before != TPP_NORM_NONE && p.gy;
  float wa[8], wb[8], ca[8], sum[4][8] = {};
#pragma unroll
  for (int e = 0; e < 8; ++e) {
    wa[e] = wb[e] = 1.0f;
    ca[e] = 0.0f;
  }
  if (after) load8(p.wa, c.at, wa);
  if (before) load8(p.wb, c.at, wb);
  if (MEANS && p.after == TPP_NORM_LAYER && p.ca) load8(p.ca, c.at, ca);
  const int64_t s_end = min((blockIdx.y + 1) * cut.take, cut.segments);
  for (int64_t s = blockIdx.y * cut.take; s < s_end; ++s) {
    const int64_t gate = s / cut.per, t0 = gate * cut.every + (s - gate * cut.per) * cut.rows;
    const int64_t t1 = min(min(t0 + cut.rows, (gate + 1) * cut.every), p.tokens);
    float A[8] = {}, B[8] = {};
#pragma unroll 2
    for (int64_t t = t0; t < t1; ++t) {
      const float* st = stats + t * STATS;
      Raw<BF16> rb_ = load_raw<BF16, CACHED>(p.b, t * p.ldb + c.at), rr_ = {}, rd = {}, ry = {};
      if (before) rr_ = load_raw<BF16, CACHED>(p.r, t * p.ldr + c.at);
      if (p.gr) rd = load_raw<BF16, CACHED>(p.gr, t * p.ldgr + c.at);
      if (p.gy) ry = load_raw<BF16, CACHED>(p.gy, t * p.ldgy + c.at);
      const float mr = st[0], rr = st[1], mb = st[2], rb = st[3], uv = st[4], u0 = st[5];
      float b[8], r[8], d[8], y[8];
      widen<BF16>(rb_, b);
      widen<BF16>(rr_, r);
      widen<BF16>(rd, d);
      widen<BF16>(ry, y);
#pragma unroll
      for (int e = 0; e < 8; ++e) {
        const float vn = (r[e] - mr) * rr;
        sum[2][e] = __builtin_fmaf(y[e], vn, sum[2][e]);
        if (MEANS) sum[3][e] += y[e];
        d[e] = __builtin_fmaf(rr, y[e] * wb[e] - vn * uv - u0, d[e]);
        A[e] = __builtin_fmaf(d[e], (b[e] - mb) * rb, A[e]);
        if (MEANS) B[e] += d[e];
      }
    }
    float g[8], v[8];
    if (p.gate_form) load8(p.gate, gate * p.ldg + c.at, p.gate_bf16, g);
#pragma unroll
    for (int e = 0; e < 8; ++e) {
      const float gs = p.scale * (p.gate_form ? gate_value(g[e], p.gate_form) : 1.0f);
      sum[0][e] = __builtin_fmaf(gs, A[e], sum[0][e]);
      if (MEANS) sum[1][e] = __builtin_fmaf(gs, B[e], sum[1][e]);
      v[e] = p.scale * (A[e] * wa[e] + B[e] * ca[e]);
      if (p.dgate && !gate_part) v[e] *= gate_slope(g[e], p.gate_form);
    }
    if (!p.dgate) continue;
    if (gate_part)
      store_raw<false, WHOLE, CACHED>(gate_part, s * p.f, c, narrow<false>(v));
    else if (p.gate_bf16)
      store_raw<true, WHOLE, CACHED>(p.dgate, gate * p.lddg, c, narrow<true>(v));
    else
      store_raw<false, WHOLE, CACHED>(p.dgate, gate * p.lddg, c, narrow<false>(v));
  }
  int32_t n = 0;
#pragma unroll
  for (int v = 0; v < 4; ++v)
    if (p.dv[v])
      store_raw<false, WHOLE, CACHED>(part, ((int64_t)n++ * gridDim.y + blockIdx.y) * p.f, c, narrow<false>(sum[v]));
}

// ---- the sums' second half --------------------------------------------------------------------------
// A workgroup has 32 columns and 32 sets of 32 lanes; `sets` of them take every sets-th part of one output
// row, 8 in flight, and meet pairwise; the others have the next rows.
constexpr int FT = 1024, FE = 32, FS = FT / FE;
__global__ __launch_bounds__(FT) void fold_kernel(FoldParams p) {
  __shared__ float acc[FS][FE];
  int32_t k = 0;
  uint32_t block = blockIdx.y;
  while (block >= p.blocks[k]) block -= p.blocks[k++];
  const FoldJob& j = p.job[k];
  const int32_t sets = p.sets[k], mine = threadIdx.x / FE, lane = threadIdx.x % FE, c = blockIdx.x * FE + lane;
  const int32_t set = mine & (sets - 1);
  const int64_t row = (int64_t)block * (FS / sets) + mine / sets;
  const bool held = row < j.rows && c < p.width;
  const float* from = j.from + row * j.parts * p.width + c;
  float sum = 0.0f;
  for (int64_t i = set; held && i < j.parts; i += 8 * sets) {
    float x[8];
#pragma unroll
    for (int u = 0; u < 8; ++u)
      x[u] = i + u * sets < j.parts ? gld<float>(from + (i + u * sets) * p.width) : 0.0f;
#pragma unroll
    for (int u = 0; u < 8; ++u) sum += x[u];
  }
  acc[mine][lane] = sum;
  __syncthreads();
  for (int32_t h = sets / 2; h > 0; h /= 2) {
    if (set < h) acc[mine][lane] += acc[mine + h][lane];
    __syncthreads();
  }
  if (set == 0 && held) {
    float v = acc[mine][lane];
    if (j.slope) v *= gate_slope(load1(j.gate, row * j.ldg + c, j.bf16), j.slope);
    store1(j.to, row * j.ld + c, v, j.bf16);
  }
}

__global__ __launch_bounds__(RT) void zeros_kernel(void* to, int64_t n, int32_t bf16) {
  const int64_t i = (int64_t)blockIdx.x * RT + threadIdx.x;
  if (i < n) store1(to, i, 0.0f, bf16);
}

constexpr int64_t MOST_PARTS = 256;

template <typename F>
void by_how(int how, const F& f) {
  if (how == STREAM) f(IntC<STREAM>());
  else if (how == STREAM_OUT) f(IntC<STREAM_OUT>());
  else f(IntC<CACHED>());
}
// Outputs beyond the L2s' reach go past the caches' replacement (2048 tokens of 4096 bf16, 33 MB, 26.9 us
// against 30.5), and where all is more than the last-level cache holds inputs do too (8192, 402 MB, 85.6 us
// against 87.9; 2048 32.4, 1024 23.5 against 19.8).  Rows that are no whole chunks share lines.
int cache_use(const ResidualParams& p) {
  const int64_t bytes = p.tokens * p.f * (p.bf16 ? 2 : 4);
  if (2 * bytes <= 8 * MB) return CACHED;
  return 6 * bytes > 256 * MB && p.f % 8 == 0 ? STREAM : STREAM_OUT;
}
template <typename F>
void back_by_width(const ResidualParams& p, const F& f) {
  const std::true_type sums;
  const int32_t chunks = (p.f + 511) / 512;
  if (chunks <= 1) return f(IntC<1>(), IntC<1>(), sums);
  if (chunks <= 2) return f(IntC<2>(), IntC<1>(), sums);
  if (chunks <= 4) return f(IntC<4>(), IntC<1>(), sums);
  if (chunks <= 8) return f(IntC<8>(), IntC<1>(), sums);
  if (chunks <= 16) return f(IntC<8>(), IntC<2>(), sums);
  if (chunks <= 24) return f(IntC<8>(), IntC<3>(), std::false_type());
  return f(IntC<8>(), IntC<4>(), std::false_type());
}

// The backward pass: whether its rows stay in registers, its sums too, how the tokens are cut, and the
// workgroups.  A row team has two tokens at least, whose parts would else be as many as the rows; few tokens
// have a team each (300 of 4096 with a gate for every 7: 15.9 us against 18.4).
constexpr int64_t BACK_WAVES = 2048, FEW_TOKENS = 256;
struct BackPlan {
  bool rows, sums;
  Cut cut;
  int64_t groups;
  explicit BackPlan(const ResidualParams& p) : rows(p.f >= 8 && p.f <= MOST_ROW), sums(rows && p.f <= 8192) {
    int w = 8;
    if (sums) back_by_width(p, [&](auto ww, auto, auto) { w = decltype(ww)::value; });
    cut = cut_tokens(p, sums ? min64(BACK_WAVES / w, p.tokens <= FEW_TOKENS ? p.tokens : ceil_div(p.tokens, 2)) : MOST_PARTS);
    groups = ceil_div(cut.parts, sums && w == 1 ? RW : 1);
  }
};

int vectors_of(const ResidualParams& p) {
  int n = 0;
  for (const float* v : p.dv) n += v != nullptr;
  return n;
}
bool sums_wanted(const ResidualParams& p) { return vectors_of(p) > 0 || p.dgate; }

}  // namespace

hipError_t launch_fold(FoldParams& p, hipStream_t stream) {
  int64_t blocks = 0;
  for (int k = 0; k < p.n; ++k) {
    int32_t sets = 1;
    while (sets < FS && 8 * sets < p.job[k].parts) sets *= 2;
    p.sets[k] = sets;
    p.blocks[k] = (uint32_t)ceil_div(p.job[k].rows, FS / sets);
    blocks += p.blocks[k];
  }
  const dim3 grid((uint32_t)((p.width + FE - 1) / FE), (uint32_t)blocks);
  hipLaunchKernelGGL(fold_kernel, grid, dim3(FT), 0, stream, p);
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

int64_t residual_backward_work_floats(const ResidualParams& p) {
  if (!sums_wanted(p)) return 0;
  const BackPlan b(p);
  return (b.sums ? 0 : p.tokens * STATS) +
         (vectors_of(p) * b.groups + (p.dgate && b.cut.per > 1 ? b.cut.segments : 0)) * p.f;
}

hipError_t launch_residual_backward(const ResidualParams& p, float* work, hipStream_t stream) {
  const BackPlan b(p);
  const Cut& c = b.cut;
  const int n = vectors_of(p);
  const bool wanted = sums_wanted(p), means = p.after == TPP_NORM_LAYER || p.before == TPP_NORM_LAYER;
  float* stats = wanted && !b.sums ? work : nullptr;
  float* part = wanted && !b.sums ? work + p.tokens * STATS : work;
  float* gate_part = p.dgate && c.per > 1 ? part + n * b.groups * p.f : nullptr;
  const auto by_means = [&](const auto& f) { means ? f(std::true_type()) : f(std::false_type()); };
  if (b.rows) {
    const int how = cache_use(p);
    // without sums a row to a workgroup, as far as a grid goes
    Cut rows = c;
    int64_t groups = b.groups;
    if (!b.sums) {
      rows = cut_tokens(p, min64(p.tokens, 1 << 20));
      groups = rows.parts;
    }
    by_type(p.bf16, p.f, [&](auto bf16, auto whole) {
      by_how(how, [&](auto h) {
        back_by_width(p, [&](auto w, auto cc, auto sums) {
          constexpr int W = decltype(w)::value, C = decltype(cc)::value;
          if constexpr (decltype(whole)::value || decltype(h)::value != STREAM) {   // (see cache_use)
            by_means([&](auto m) {
              hipLaunchKernelGGL((residual_backward_row_kernel<decltype(bf16)::value, W, C, decltype(whole)::value,
                                                               decltype(h)::value, decltype(m)::value,
                                                               decltype(sums)::value>),
                                 dim3((uint32_t)groups), dim3(W == 1 ? RT : 64 * W), 0, stream, p, rows, part,
                                 gate_part, stats);
            });
          }
        });
      });
    });
  } else {
    const dim3 grid((uint32_t)min64(p.tokens, 1 << 20));
    if (p.bf16)
      hipLaunchKernelGGL((residual_backward_any_kernel<true>), grid, dim3(RT), 0, stream, p, stats);
    else
      hipLaunchKernelGGL((residual_backward_any_kernel<false>), grid, dim3(RT), 0, stream, p, stats);
  }
  if (!wanted) return hipGetLastError();
  if (b.rows && !b.sums) {
    const dim3 columns((uint32_t)ceil_div(p.f, 8 * RT), (uint32_t)b.groups);
    by_type(p.bf16, p.f, [&](auto bf16, auto whole) {
      by_means([&](auto m) {
        hipLaunchKernelGGL((residual_columns_kernel<decltype(bf16)::value, decltype(whole)::value, decltype(m)::value>),
                           columns, dim3(RT), 0, stream, p, c, stats, part, gate_part);
      });
    });
  } else if (!b.rows) {
    const dim3 columns((uint32_t)ceil_div(p.f, RT), (uint32_t)b.groups);
    if (p.bf16)
      hipLaunchKernelGGL((residual_columns_any_kernel<true>), columns, dim3(RT), 0, stream, p, c, stats, part, gate_part);
    else
      hipLaunchKernelGGL((residual_columns_any_kernel<false>), columns, dim3(RT), 0, stream, p, c, stats, part, gate_part);
  }
  FoldParams fold = {};
  fold.width = p.f;
  for (float* to : p.dv) {
    if (!to) continue;
    fold.job[fold.n] = {part + (int64_t)fold.n * b.groups * p.f, b.groups, 1, to, 0, 0, 0, nullptr, 0};
    ++fold.n;
  }
  if (gate_part)
    fold.job[fold.n++] = {gate_part, c.per, ceil_div(p.tokens, c.every), p.dgate, p.lddg, p.gate_bf16,
                          p.gate_form, p.gate, p.ldg};
  if (fold.n > 0) return launch_fold(fold, stream);
  return hipGetLastError();
}

}  // namespace tpp

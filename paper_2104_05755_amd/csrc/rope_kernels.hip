// rope_kernels.hip -- norms of query and key heads with the position rotation, forward (also into a
// paged cache) and backward, for gfx950.
//
// A row is one head of one token: y = x r w with r = 1 / sqrt(mean(x^2) + eps), then the pairs of its
// first rot_dim entries turned by the token's angles.  Both are linear in y, so a row needs one sum
// over its entries and one pass; the backward pass turns the gradient back (the rotation's transpose),
// u = g w, and needs one more sum, of u xn.
//
// One wavefront per row: a unit is a rotated pair or an entry behind the rotated part, lane l has the
// units l, l + 64, ...
#include <hip/hip_runtime.h>

#include "brgemm_device.h"
#include "internal.h"

namespace tpp {
namespace {

using namespace dev;

constexpr int QT = 256;   // threads per workgroup: 4 wavefronts

__device__ __forceinline__ float load_elem(const void* p, int64_t at, bool bf16) {
  return bf16 ? bf16_bits_to_f32(gld<uint16_t>(static_cast<const uint16_t*>(p) + at))
              : gld<float>(static_cast<const float*>(p) + at);
}
__device__ __forceinline__ void store_elem(void* p, int64_t at, float v, bool bf16) {
  if (bf16)
    gst<uint16_t>(static_cast<uint16_t*>(p) + at, f32_to_bf16_bits(v));
  else
    gst<float>(static_cast<float*>(p) + at, v);
}

__device__ __forceinline__ float wave_sum(float v) {
#pragma unroll
  for (int h = 32; h > 0; h >>= 1) v += __shfl_xor(v, h, 64);
  return v;
}

// Entries of unit u of a row: a pair (a, b) below rot_dim / 2, else the entry a alone (b < 0).
__device__ __forceinline__ void unit_entries(const QkParams& p, int32_t u, int32_t& a, int32_t& b) {
  const int32_t half = p.rot_dim / 2;
  if (u < half) {
    a = p.pairs ? 2 * u : u;
    b = p.pairs ? 2 * u + 1 : u + half;
  } else {
    a = u + half;
    b = -1;
  }
}

// First element of head `head` of cache slot `slot` (inside the pools).
__device__ __forceinline__ int64_t slot_base(const QkParams& p, int64_t slot, int32_t head) {
  const int64_t page = p.n_slots <= 0x7fffffff ? (int64_t)fdiv((uint32_t)slot, p.page)
                                               : slot / p.page_size;
  return page * p.page_stride + (slot - page * p.page_size) * p.pos_stride + head * p.head_stride;
}

template <int NU>
__global__ __launch_bounds__(QT) void qk_row_kernel(QkParams p, int64_t rows, int32_t per_token,
                                                    FastDiv div) {
  const int lane = threadIdx.x & 63;
  const int64_t row = (int64_t)blockIdx.x * (QT / 64) + (threadIdx.x >> 6);
  if (row >= rows) return;
  const int64_t t = fdiv((uint32_t)row, div);
  int32_t head = (int32_t)(row - t * per_token);
  int side = 0;
  for (; side < 2 && head >= p.side[side].heads; ++side) head -= p.side[side].heads;
  const int64_t pos = p.pos[t];
  const bool held = pos >= 0 && pos < p.n_positions;
  int64_t to = 0;
  void* out;
  if (side > 0 && p.slot) {
    const int64_t slot = p.slot[t];
    if (!held || slot < 0 || slot >= p.n_slots) return;
    to = slot_base(p, slot, head);
    out = side == 1 ? p.kc : p.vc;
  } else {
    to = t * p.side[side].ldo + (int64_t)head * p.d;
    out = p.side[side].out;
  }
  if (side == 2) {   // a value head: copied
    for (int32_t e = lane; e < p.d; e += 64)
      store_elem(out, to + e, load_elem(p.v, t * p.ldv + (int64_t)head * p.d + e, p.bf16), p.bf16);
    return;
  }
  const QkSide& sd = p.side[side];
  const int64_t from = t * sd.ldx + (int64_t)head * p.d;
  const int32_t units = p.d - p.rot_dim / 2;
  float xa[NU], xb[NU], sum = 0.0f;
#pragma unroll
  for (int i = 0; i < NU; ++i) {
    const int32_t u = lane + 64 * i;
    xa[i] = xb[i] = 0.0f;
    if (u < units) {
      int32_t a, b;
      unit_entries(p, u, a, b);
      xa[i] = load_elem(sd.x, from + a, p.bf16);
      if (b >= 0) xb[i] = load_elem(sd.x, from + b, p.bf16);
    }
    sum += xa[i] * xa[i] + xb[i] * xb[i];
  }
  const float r = 1.0f / sqrtf(wave_sum(sum) / (float)p.d + p.eps);
#pragma unroll
  for (int i = 0; i < NU; ++i) {
    const int32_t u = lane + 64 * i;
    if (u >= units) continue;
    int32_t a, b;
    unit_entries(p, u, a, b);
    float ya = 0.0f, yb = 0.0f;
    if (held) {
      ya = xa[i] * r * gld<float>(sd.w + a);
      if (b >= 0) {
        yb = xb[i] * r * gld<float>(sd.w + b);
        const float c = gld<float>(p.rot + pos * p.rot_dim + u);
        const float s = gld<float>(p.rot + pos * p.rot_dim + p.rot_dim / 2 + u);
        const float ta = ya * c - yb * s;
        yb = yb * c + ya * s;
        ya = ta;
      }
    }
    store_elem(out, to + a, ya, p.bf16);
    if (b >= 0) store_elem(out, to + b, yb, p.bf16);
  }
}

// Backward.  Workgroup w of a side (nq of the queries, the rest of the keys) takes its rows w, w + n,
// ... and keeps its part of the weights' gradient in registers; parts go to `part` (a row of D per
// workgroup), or straight to dw where a side has one workgroup.
template <int NU>
__global__ __launch_bounds__(QT) void qk_backward_row_kernel(QkParams p, int32_t nq, float* part) {
  __shared__ float acc[QT / 64][2 * 64 * NU];
  const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
  const int side = (int32_t)blockIdx.x >= nq ? 1 : 0;
  const int32_t wg = blockIdx.x - (side ? nq : 0);
  const int32_t n_wg = side ? (int32_t)gridDim.x - nq : nq;
  const QkSide& sd = p.side[side];
  const int64_t rows = p.tokens * sd.heads;
  const int32_t units = p.d - p.rot_dim / 2;
  float wa[NU], wb[NU], da[NU], db[NU];
#pragma unroll
  for (int i = 0; i < NU; ++i) {
    const int32_t u = lane + 64 * i;
    wa[i] = wb[i] = da[i] = db[i] = 0.0f;
    if (u >= units || rows == 0) continue;   // without rows the weights may be null
    int32_t a, b;
    unit_entries(p, u, a, b);
    wa[i] = gld<float>(sd.w + a);
    if (b >= 0) wb[i] = gld<float>(sd.w + b);
  }
  for (int64_t row = (int64_t)wg * (QT / 64) + wave; row < rows; row += (int64_t)n_wg * (QT / 64)) {
    const int64_t t = row / sd.heads;
    const int32_t head = (int32_t)(row - t * sd.heads);
    const int64_t pos = p.pos[t];
    const bool held = pos >= 0 && pos < p.n_positions;
    const int64_t fx = t * sd.ldx + (int64_t)head * p.d, fg = t * sd.ldg + (int64_t)head * p.d,
                  to = t * sd.ldo + (int64_t)head * p.d;
    float xa[NU], xb[NU], ga[NU], gb[NU], xx = 0.0f, ux = 0.0f;
#pragma unroll
    for (int i = 0; i < NU; ++i) {
      const int32_t u = lane + 64 * i;
      xa[i] = xb[i] = ga[i] = gb[i] = 0.0f;
      if (u < units && held) {
        int32_t a, b;
        unit_entries(p, u, a, b);
        xa[i] = load_elem(sd.x, fx + a, p.bf16);
        ga[i] = load_elem(sd.g, fg + a, p.bf16);
        if (b >= 0) {
          xb[i] = load_elem(sd.x, fx + b, p.bf16);
          gb[i] = load_elem(sd.g, fg + b, p.bf16);
          const float c = gld<float>(p.rot + pos * p.rot_dim + u);
          const float s = gld<float>(p.rot + pos * p.rot_dim + p.rot_dim / 2 + u);
          const float ta = ga[i] * c + gb[i] * s;
          gb[i] = gb[i] * c - ga[i] * s;
          ga[i] = ta;
        }
      }
      xx += xa[i] * xa[i] + xb[i] * xb[i];
      ux += ga[i] * wa[i] * xa[i] + gb[i] * wb[i] * xb[i];
    }
    const float r = 1.0f / sqrtf(wave_sum(xx) / (float)p.d + p.eps);
    const float m = wave_sum(ux) * r / (float)p.d;   // mean(u xn)
#pragma unroll
    for (int i = 0; i < NU; ++i) {
      const int32_t u = lane + 64 * i;
      if (u >= units) continue;
      int32_t a, b;
      unit_entries(p, u, a, b);
      const float na = xa[i] * r, nb = xb[i] * r;
      if (held) {
        da[i] += ga[i] * na;
        db[i] += gb[i] * nb;
      }
      store_elem(sd.out, to + a, held ? r * (ga[i] * wa[i] - na * m) : 0.0f, p.bf16);
      if (b >= 0) store_elem(sd.out, to + b, held ? r * (gb[i] * wb[i] - nb * m) : 0.0f, p.bf16);
    }
  }
  // the four wavefronts' parts, added in order
#pragma unroll
  for (int i = 0; i < NU; ++i) {
    acc[wave][lane + 64 * i] = da[i];
    acc[wave][64 * NU + lane + 64 * i] = db[i];
  }
  __syncthreads();
  for (int32_t j = threadIdx.x; j < 2 * 64 * NU; j += QT) {
    const int32_t u = j & (64 * NU - 1);
    if (u >= units) continue;
    int32_t a, b;
    unit_entries(p, u, a, b);
    const int32_t e = j < 64 * NU ? a : b;
    if (e < 0) continue;
    const float v = ((acc[0][j] + acc[1][j]) + acc[2][j]) + acc[3][j];
    gst<float>((part ? part + (int64_t)blockIdx.x * p.d : sd.dw) + e, v);
  }
}

// dw[e] of a side: its workgroups' parts, in order.
__global__ __launch_bounds__(QT) void qk_fold_kernel(QkParams p, int32_t nq, int32_t nk,
                                                     const float* part) {
  const int side = blockIdx.y;
  const QkSide& sd = p.side[side];
  const int32_t e = blockIdx.x * QT + threadIdx.x, n = side ? nk : nq;
  if (e >= p.d || sd.heads == 0) return;
  const float* from = part + (int64_t)(side ? nq : 0) * p.d + e;
  float sum = 0.0f;
  for (int32_t i = 0; i < n; ++i) sum += gld<float>(from + (int64_t)i * p.d);
  gst<float>(sd.dw + e, sum);
}

// Workgroups of the two sides in the backward pass: 1024 in all where there are rows for them.
void backward_groups(const QkParams& p, int32_t& nq, int32_t& nk) {
  const int32_t heads = p.side[0].heads + p.side[1].heads;
  int32_t n[2];
  for (int s = 0; s < 2; ++s) {
    const int64_t full = (p.tokens * p.side[s].heads + QT / 64 - 1) / (QT / 64);
    const int64_t share = (int64_t)1024 * p.side[s].heads / heads;
    const int64_t most = full < share ? full : share;
    n[s] = p.side[s].heads == 0 ? 0 : most < 1 ? 1 : (int32_t)most;
  }
  nq = n[0];
  nk = n[1];
}

}  // namespace

hipError_t launch_qk(const QkParams& p, hipStream_t stream) {
  const int32_t per = p.side[0].heads + p.side[1].heads * (p.slot ? 2 : 1);
  if (per == 0) return hipSuccess;
  const int32_t units = p.d - p.rot_dim / 2;
  const FastDiv div(per);
  // rows count in 32 bits within a launch
  const int64_t step = 0x7ffffff0 / per;
  for (int64_t t0 = 0; t0 < p.tokens; t0 += step) {
    QkParams q = p;
    q.tokens = p.tokens - t0 < step ? p.tokens - t0 : step;
    const int64_t es = p.bf16 ? 2 : 4;
    for (int s = 0; s < 2; ++s) {
      q.side[s].x = static_cast<const char*>(p.side[s].x) + t0 * p.side[s].ldx * es;
      if (p.side[s].out) q.side[s].out = static_cast<char*>(p.side[s].out) + t0 * p.side[s].ldo * es;
    }
    if (p.slot) {
      q.v = static_cast<const char*>(p.v) + t0 * p.ldv * es;
      q.slot += t0;
    }
    q.pos += t0;
    const int64_t rows = q.tokens * per;
    const dim3 grid((uint32_t)((rows + QT / 64 - 1) / (QT / 64)));
#define TPP_QK(NU) \
  hipLaunchKernelGGL((qk_row_kernel<NU>), grid, dim3(QT), 0, stream, q, rows, per, div)
    if (units <= 64) TPP_QK(1);
    else if (units <= 128) TPP_QK(2);
    else if (units <= 256) TPP_QK(4);
    else TPP_QK(8);
#undef TPP_QK
    const hipError_t e = hipGetLastError();
    if (e != hipSuccess) return e;
  }
  return hipSuccess;
}

int64_t qk_backward_work_floats(const QkParams& p) {
  if (p.side[0].heads + p.side[1].heads == 0) return 0;
  int32_t nq, nk;
  backward_groups(p, nq, nk);
  return nq <= 1 && nk <= 1 ? 0 : (int64_t)(nq + nk) * p.d;
}

hipError_t launch_qk_backward(const QkParams& p, float* work, hipStream_t stream) {
  if (p.side[0].heads + p.side[1].heads == 0) return hipSuccess;
  int32_t nq, nk;
  backward_groups(p, nq, nk);
  if (!work) {
    nq = nq < 1 ? nq : 1;
    nk = nk < 1 ? nk : 1;
  }
  const int32_t units = p.d - p.rot_dim / 2;
#define TPP_QKB(NU)                                                                              \
  hipLaunchKernelGGL((qk_backward_row_kernel<NU>), dim3(nq + nk), dim3(QT), 0, stream, p, nq, work)
  if (units <= 64) TPP_QKB(1);
  else if (units <= 128) TPP_QKB(2);
  else if (units <= 256) TPP_QKB(4);
  else TPP_QKB(8);
#undef TPP_QKB
  if (work)
    hipLaunchKernelGGL(qk_fold_kernel, dim3((p.d + QT - 1) / QT, 2), dim3(QT), 0, stream, p, nq, nk,
                       work);
  return hipGetLastError();
}

}  // namespace tpp

// q8_kernels.hip -- 8-bit rows of activations (gfx950): quantisation for a product, and activations of
// training that keep their input in 8 bits, with the backward pass from it.
//
// A group's entries become q = 127 v / max|v| rounded to whole numbers, scale = max|v| / 127.  A few
// operations an entry of 1 to 4 bytes: bound by HBM.
#include <hip/hip_runtime.h>

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

constexpr int64_t MOST_PARTS = 256;
int64_t parts_of(const Q8Params& p, int64_t& take) {
  take = (p.tokens + MOST_PARTS - 1) / MOST_PARTS;
  return (p.tokens + take - 1) / take;
}
dim3 rows_grid(const Q8Params& p) { return dim3((uint32_t)(p.tokens < (1 << 20) ? p.tokens : (1 << 20))); }

}  // namespace

hipError_t launch_q8_quantize(const Q8Params& p, hipStream_t stream) {
  if (p.bf16)
    hipLaunchKernelGGL((q8_quantize_any_kernel<true>), rows_grid(p), dim3(QT), 0, stream, p);
  else
    hipLaunchKernelGGL((q8_quantize_any_kernel<false>), rows_grid(p), dim3(QT), 0, stream, p);
  return hipGetLastError();
}

hipError_t launch_q8_act(const Q8Params& p, hipStream_t stream) {
  if (p.bf16)
    hipLaunchKernelGGL((q8_act_any_kernel<true>), rows_grid(p), dim3(QT), 0, stream, p);
  else
    hipLaunchKernelGGL((q8_act_any_kernel<false>), rows_grid(p), dim3(QT), 0, stream, p);
  return hipGetLastError();
}

int64_t q8_backward_work_floats(const Q8Params& p) {
  int64_t take;
  return p.dbias ? parts_of(p, take) * (p.gated ? 2 * p.f : p.f) : 0;
}

hipError_t launch_q8_act_backward(const Q8Params& p, float* work, hipStream_t stream) {
  int64_t take;
  const int64_t parts = parts_of(p, take);
  const dim3 grid((uint32_t)((p.f + QT - 1) / QT), (uint32_t)parts);
  float* part = p.dbias ? work : nullptr;
  if (p.bf16)
    hipLaunchKernelGGL((q8_act_backward_any_kernel<true>), grid, dim3(QT), 0, stream, p, take, part);
  else
    hipLaunchKernelGGL((q8_act_backward_any_kernel<false>), grid, dim3(QT), 0, stream, p, take, part);
  if (!part) return hipGetLastError();
  FoldParams fold = {};
  fold.width = p.gated ? 2 * p.f : p.f;
  fold.n = 1;
  fold.job[0] = {part, parts, 1, p.dbias, 0, 0, 0, nullptr, 0};
  return launch_fold(fold, stream);
}

}  // namespace tpp

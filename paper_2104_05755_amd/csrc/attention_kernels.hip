// attention_kernels.hip -- attention of one new token per sequence over a paged key-value cache, for
// gfx950.
//
// Per sequence and query head: scores s_t = scale q . k_t over the positions that are held, their
// softmax, and the sum of the values with it.  One workgroup per sequence and query head walks the
// positions 256 at a time, a score per lane, with the running maximum and sum of the softmax: when the
// maximum grows the sums so far are scaled down, so that every position is read once.
#include <hip/hip_runtime.h>

#include "brgemm_device.h"
#include "internal.h"

namespace tpp {
namespace {

using namespace dev;

constexpr int AT = 256;

__device__ __forceinline__ float load_elem(const void* p, int64_t at, bool bf16) {
  return bf16 ? bf16_bits_to_f32(gld<uint16_t>(static_cast<const uint16_t*>(p) + at))
              : gld<float>(static_cast<const float*>(p) + at);
}

// Element offset of position t of sequence b (head 0), or -1 where no page holds it.
__device__ __forceinline__ int64_t row_of(const AttnParams& p, int64_t b, int32_t t) {
  const int32_t j = fdiv((uint32_t)t, p.page);
  const int64_t page = gld<int64_t>(p.pages + b * p.ld_pages + j);
  if (page < 0 || page >= p.n_pages) return -1;
  return page * p.page_stride + (int64_t)(t - j * p.page_size) * p.pos_stride;
}

__device__ __forceinline__ int32_t length_of(const AttnParams& p, int64_t b) {
  const int64_t n = gld<int64_t>(p.len + b);
  return (int32_t)(n < 0 ? 0 : n > p.max_len ? p.max_len : n);
}

__device__ __forceinline__ float score(const AttnParams& p, const float* q, int64_t row) {
  float s = 0.0f;
  for (int32_t e = 0; e < p.d; ++e) s += q[e] * load_elem(p.k, row + e, p.bf16);
  return s * p.scale;
}

__global__ __launch_bounds__(AT) void attn_simple_kernel(AttnParams p, float* lse) {
  __shared__ float q[256], prob[AT];
  __shared__ int64_t rows[AT];
  __shared__ float red[AT];
  const int tid = threadIdx.x;
  const int64_t b = blockIdx.x;
  const int32_t h = blockIdx.y, hk = h / (p.q_heads / p.kv_heads);
  const int32_t n = length_of(p, b);
  const int64_t lo64 = p.window > 0 && n > p.window ? n - p.window : 0;
  for (int32_t e = tid; e < p.d; e += AT) q[e] = load_elem(p.q, b * p.ldq + (int64_t)h * p.d + e, p.bf16);
  float m = -INFINITY, l = 0.0f, o = 0.0f;   // o: entry tid of the output
  for (int32_t t0 = (int32_t)lo64; t0 < n; t0 += AT) {
    __syncthreads();
    const int32_t t = t0 + tid;
    const int64_t row = t < n ? row_of(p, b, t) : -1;
    float s = -INFINITY;
    if (row >= 0) s = score(p, q, row + hk * p.head_stride);
    rows[tid] = row;
    red[tid] = s;
    __syncthreads();
    float top = m;
    for (int i = 0; i < AT; ++i) top = fmaxf(top, red[i]);
    const float base = top == -INFINITY ? 0.0f : top;
    prob[tid] = row >= 0 ? expf(s - base) : 0.0f;
    __syncthreads();
    const float down = m == -INFINITY ? 0.0f : expf(m - base);
    l *= down;
    o *= down;
    m = top;
    for (int i = 0; i < AT; ++i) {
      if (rows[i] < 0) continue;
      l += prob[i];
      if (tid < p.d) o += prob[i] * load_elem(p.v, rows[i] + hk * p.head_stride + tid, p.bf16);
    }
  }
  if (tid < p.d) {
    const float v = l > 0.0f || l != l ? o / l : 0.0f;
    const int64_t at = b * p.ldo + (int64_t)h * p.d + tid;
    if (p.out_bf16)
      gst<uint16_t>(static_cast<uint16_t*>(p.out) + at, f32_to_bf16_bits(v));
    else
      gst<float>(static_cast<float*>(p.out) + at, v);
  }
  if (tid == 0) {
    const float z = l == 0.0f ? -INFINITY : m + logf(l);
    if (p.lse) gst<float>(p.lse + b * p.q_heads + h, z);
    if (lse) gst<float>(lse + b * p.q_heads + h, z);
  }
}

__global__ __launch_bounds__(AT) void attn_totals_kernel(AttnParams p, const float* lse) {
  __shared__ float q[256];
  const int tid = threadIdx.x;
  const int64_t b = blockIdx.x;
  const int32_t n = length_of(p, b), t = blockIdx.y * AT + tid;
  const int64_t row = t < n && (p.window == 0 || t >= n - p.window) ? row_of(p, b, t) : -1;
  float sum = 0.0f;
  for (int32_t h = 0; h < p.q_heads; ++h) {
    __syncthreads();
    for (int32_t e = tid; e < p.d; e += AT)
      q[e] = load_elem(p.q, b * p.ldq + (int64_t)h * p.d + e, p.bf16);
    __syncthreads();
    if (row >= 0)
      sum += expf(score(p, q, row + h / (p.q_heads / p.kv_heads) * p.head_stride) -
                  gld<float>(lse + b * p.q_heads + h));
  }
  if (t < n) {
    const int64_t at = b * p.ldt + t;
    gst<float>(p.totals_out + at, (p.totals_in ? gld<float>(p.totals_in + at) : 0.0f) + sum);
  }
}

}  // namespace

int64_t attn_work_floats(const AttnParams& p) { return p.totals_out ? p.n_seqs * p.q_heads : 0; }

hipError_t launch_attn(const AttnParams& p, float* work, hipStream_t stream) {
  if (p.n_seqs > 0x7fffffff || p.q_heads > 65535) return hipErrorInvalidConfiguration;
  hipLaunchKernelGGL(attn_simple_kernel, dim3((uint32_t)p.n_seqs, p.q_heads), dim3(AT), 0, stream, p,
                     work);
  if (p.totals_out && p.max_len > 0)
    hipLaunchKernelGGL(attn_totals_kernel, dim3((uint32_t)p.n_seqs, (uint32_t)((p.max_len + AT - 1) / AT)),
                       dim3(AT), 0, stream, p, work);
  return hipGetLastError();
}

}  // namespace tpp

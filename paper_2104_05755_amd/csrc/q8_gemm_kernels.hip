// q8_gemm_kernels.hip -- products of 8-bit rows (gfx950): C = act(sb_j sa_i sum_p A_ip B_pj + bias_i), both
// operands with k contiguous, the sum exact in 32-bit integers.
//
// The matrix instruction v_mfma_i32_16x16x64_i8 takes 16 consecutive bytes of a row from each lane: lane l
// has row (column) l % 16 and k from 16 (l / 16) on, and leaves rows 4 (l / 16) .. + 3 of column l % 16 in
// the lane.  Weights are its A, tokens its B, so a lane ends with four consecutive channels of one token.
#include <hip/hip_runtime.h>

#include "internal.h"
#include "rows_device.h"

namespace tpp {
namespace {

using namespace rows;

typedef int32_t i32x4_t __attribute__((ext_vector_type(4)));
typedef uint32_t u32x4_a1 __attribute__((ext_vector_type(4), aligned(1)));

// 16 bytes of a row from byte kk on, those behind k zero.  ALIGNED: row and kk at multiples of 16, and the
// whole chunk is read where its first byte is in the row.
template <bool ALIGNED>
__device__ __forceinline__ i32x4_t tail16(const int8_t* row, int32_t kk, int32_t k) {
  const int32_t have = k - kk;
  u32x4 w = {0, 0, 0, 0};
  if constexpr (ALIGNED) {
    w = gld<u32x4>(row + (have > 0 ? kk : 0));
#pragma unroll
    for (int d = 0; d < 4; ++d) {
      const int32_t n = have - 4 * d;
      w[d] = n >= 4 ? w[d] : n <= 0 ? 0u : w[d] & ((1u << (8 * n)) - 1);
    }
  } else if (have >= 16) {
    w = (u32x4)gld<u32x4_a1>(row + kk);
  } else {
    for (int32_t e = 0; e < have; ++e) {
      const uint32_t v = (uint32_t)gld<uint8_t>(row + kk + e) << (8 * (e & 3));
#pragma unroll
      for (int d = 0; d < 4; ++d) w[d] |= (e >> 2) == d ? v : 0u;
    }
  }
  return __builtin_bit_cast(i32x4_t, w);
}

// Four channels of one token: scales, bias, activation, rounding and store.
__device__ __forceinline__ void finish4(const Q8GemmParams& p, i32x4_t acc, int32_t i, int32_t j) {
  if (j >= p.n || i >= p.m) return;
  const float sb = gld<float>(p.sb + j);
  float v[4];
#pragma unroll
  for (int e = 0; e < 4; ++e) {
    const int32_t row = min(i + e, p.m - 1);
    v[e] = (float)acc[e] * sb * gld<float>(p.sa + row);
    if (p.flags & TPP_EPI_BIAS) v[e] += gld<float>(p.bias + row);
    v[e] = activate(v[e], p.flags);
  }
  const int64_t at = (int64_t)j * p.ldc + i;
  if (p.c_bf16) {
    uint16_t* c = static_cast<uint16_t*>(p.c) + at;
    if (i + 4 <= p.m) {
      gst<u32x2_a2>(c, (u32x2_a2){pack_bf16x2(v[0], v[1]), pack_bf16x2(v[2], v[3])});
      return;
    }
#pragma unroll
    for (int e = 0; e < 4; ++e)
      if (i + e < p.m) gst<uint16_t>(c + e, f32_to_bf16_bits(v[e]));
  } else {
    float* c = static_cast<float*>(p.c) + at;
    if (i + 4 <= p.m) {
      gst<f32x4_a4>(c, (f32x4_a4){v[0], v[1], v[2], v[3]});
      return;
    }
#pragma unroll
    for (int e = 0; e < 4; ++e)
      if (i + e < p.m) gst<float>(c + e, v[e]);
  }
}

// ---- operands straight from memory ----------------------------------------------------------------
// A workgroup has 16 TM channels of 16 TN tokens; its NW wavefronts take a share of k each, which are added
// in LDS.
template <int TM, int TN, int NW, bool ALIGNED>
__global__ __launch_bounds__(64 * NW) void q8_gemm_direct_kernel(Q8GemmParams p) {
  __shared__ i32x4_t part[NW][TM * TN][64];
  const int32_t lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  const int32_t i0 = blockIdx.x * 16 * TM, k16 = 16 * (lane >> 4);
  const int32_t steps = (p.k + 63) / 64;
  for (int32_t j0 = blockIdx.y * 16 * TN; j0 < p.n; j0 += gridDim.y * 16 * TN) {
    const int8_t* a[TM];
    const int8_t* b[TN];
#pragma unroll
    for (int t = 0; t < TM; ++t) a[t] = p.a + (int64_t)min(i0 + 16 * t + (lane & 15), p.m - 1) * p.lda;
#pragma unroll
    for (int t = 0; t < TN; ++t) b[t] = p.b + (int64_t)min(j0 + 16 * t + (lane & 15), p.n - 1) * p.ldb;
    i32x4_t acc[TM][TN];
#pragma unroll
    for (int x = 0; x < TM; ++x)
#pragma unroll
      for (int y = 0; y < TN; ++y) acc[x][y] = (i32x4_t){0, 0, 0, 0};
    for (int32_t s = wave; s < steps; s += NW) {
      const int32_t kk = s * 64 + k16;
      i32x4_t fa[TM], fb[TN];
#pragma unroll
      for (int t = 0; t < TM; ++t) fa[t] = tail16<ALIGNED>(a[t], kk, p.k);
#pragma unroll
      for (int t = 0; t < TN; ++t) fb[t] = tail16<ALIGNED>(b[t], kk, p.k);
#pragma unroll
      for (int x = 0; x < TM; ++x)
#pragma unroll
        for (int y = 0; y < TN; ++y)
          acc[x][y] = __builtin_amdgcn_mfma_i32_16x16x64_i8(fa[x], fb[y], acc[x][y], 0, 0, 0);
    }
#pragma unroll
    for (int x = 0; x < TM; ++x)
#pragma unroll
      for (int y = 0; y < TN; ++y) part[wave][x * TN + y][lane] = acc[x][y];
    __syncthreads();
    for (int32_t t = wave; t < TM * TN; t += NW) {
      i32x4_t sum = part[0][t][lane];
#pragma unroll
      for (int w = 1; w < NW; ++w) sum += part[w][t][lane];
      finish4(p, sum, i0 + 16 * (t / TN) + 4 * (lane >> 4), j0 + 16 * (t % TN) + (lane & 15));
    }
    __syncthreads();
  }
}

}  // namespace

hipError_t launch_q8_gemm(const Q8GemmParams& p, hipStream_t stream) {
  const bool aligned = ((reinterpret_cast<uintptr_t>(p.a) | reinterpret_cast<uintptr_t>(p.b) |
                         (uint64_t)p.lda | (uint64_t)p.ldb) & 15) == 0;
  const int64_t rows = ((int64_t)p.m + 63) / 64, cols = ((int64_t)p.n + 63) / 64;
  const int64_t most = most_groups(256) / rows;   // (m below 2^31: at least 1)
  const int64_t ny = cols < most ? cols : most;
  const dim3 grid((uint32_t)rows, (uint32_t)(ny < 65535 ? ny : 65535));
  if (aligned)
    hipLaunchKernelGGL((q8_gemm_direct_kernel<4, 4, 4, true>), grid, dim3(256), 0, stream, p);
  else
    hipLaunchKernelGGL((q8_gemm_direct_kernel<4, 4, 4, false>), grid, dim3(256), 0, stream, p);
  return hipGetLastError();
}

}  // namespace tpp

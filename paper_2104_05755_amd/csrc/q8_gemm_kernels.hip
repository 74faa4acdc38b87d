// q8_gemm_kernels.hip -- products of 8-bit rows (gfx950): C = act(sb_j sa_i sum_p A_ip B_pj + bias_i), both
// operands with k contiguous, the sum exact in 32-bit integers.
//
// The matrix instructions v_mfma_i32_16x16x64_i8 and v_mfma_i32_32x32x32_i8 take 16 consecutive bytes of a row
// from each lane and leave four (times four) consecutive rows of one column in it.  Weights are A, tokens B, so a
// lane ends with consecutive channels of one token.  2 m n k operations, twice bf16's rate: many tokens are bound
// by the matrix instructions and what feeds them (the clock falls to 1.6 to 1.8 GHz under them), few tokens by
// the weights' bytes.
//
// 8192 tokens through 4096 -> 16384 with their quantisation 491 us, 2.24 POP/s, where torch's product of the rows
// alone takes 488 to 500; the MLP block's first layer (8192 through 1024 -> 4096, bias and GELU) 56 us, 45 of
// them the product; one token of 1024 through 4096 channels 4.4 us of kernel; 48 of 4096 through 16384 20 us,
// 3.4 TB/s of weights.  Fragments straight from memory for every size took 2101, 213, 12 and 25 us.
#include <hip/hip_runtime.h>

#include <type_traits>

#include "internal.h"
#include "rows_device.h"

namespace tpp {
namespace {

using namespace rows;

typedef int32_t i32x4_t __attribute__((ext_vector_type(4)));
typedef uint32_t u32x4_a1 __attribute__((ext_vector_type(4), aligned(1)));

// 16 bytes of a row from byte kk on, those from byte k on zero; nothing behind byte k is read.
__device__ __forceinline__ i32x4_t any16(const int8_t* row, int32_t kk, int32_t k) {
  const int32_t have = k - kk;
  u32x4 w = {0, 0, 0, 0};
  if (have >= 16) {
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
// The first `have` bytes of 16.
__device__ __forceinline__ i32x4_t first_bytes(i32x4_t w, int32_t have) {
#pragma unroll
  for (int d = 0; d < 4; ++d) {
    const int32_t n = have - 4 * d;
    w[d] &= n >= 4 ? ~0u : n <= 0 ? 0u : (1u << (8 * n)) - 1;
  }
  return w;
}

// Four channels of one token: scales, bias, activation, rounding and store.
__device__ __forceinline__ void finish4(const Q8GemmParams& p, i32x4_t acc, int32_t i, int32_t j, float sb) {
  if (j >= p.n || i >= p.m) return;
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

// A workgroup's wavefronts have each a share of k of its 16 TM x 16 TN tile: the sums of all, and the stores.
template <int TM, int TN, int NW, typename F>
__device__ __forceinline__ void join(const Q8GemmParams& p, i32x4_t (&part)[NW][TM * TN][64],
                                     const i32x4_t (&acc)[TM][TN], int32_t i0, int32_t j0, int32_t wave, int32_t lane,
                                     const F& scale) {
#pragma unroll
  for (int x = 0; x < TM; ++x)
#pragma unroll
    for (int y = 0; y < TN; ++y) part[wave][x * TN + y][lane] = acc[x][y];
  __syncthreads();
  for (int32_t t = wave; t < TM * TN; t += NW) {
    i32x4_t sum = part[0][t][lane];
#pragma unroll
    for (int w = 1; w < NW; ++w) sum += part[w][t][lane];
    const int32_t j = j0 + 16 * (t % TN) + (lane & 15);
    finish4(p, sum, i0 + 16 * (t / TN) + 4 * (lane >> 4), j, scale(min(j, p.n - 1)));
  }
  __syncthreads();
}
template <int TM, int TN>
__device__ __forceinline__ void zero(i32x4_t (&acc)[TM][TN]) {
#pragma unroll
  for (int x = 0; x < TM; ++x)
#pragma unroll
    for (int y = 0; y < TN; ++y) acc[x][y] = (i32x4_t){0, 0, 0, 0};
}

// ---- rows at any byte -----------------------------------------------------------------------------
// Fragments straight from memory, 16 bytes at any address of 16 rows to every 16 lanes.  Against rows at multiples
// of 16 bytes, 8192 tokens of 4096 -> 16384 7321 us and 479, 8192 of 1024 -> 4096 509 and 42, 48 of 4096 -> 16384 61
// and 15, one of 1024 -> 4096 14 and 4.
constexpr int AT = 4, AW = 4;   // 16-row tiles each way, wavefronts
__global__ __launch_bounds__(64 * AW) void q8_gemm_any_kernel(Q8GemmParams p) {
  __shared__ i32x4_t part[AW][AT * AT][64];
  const int32_t lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  const int32_t i0 = blockIdx.x * 16 * AT, steps = (p.k + 63) / 64;
  for (int64_t j0 = (int64_t)blockIdx.y * 16 * AT; j0 < p.n; j0 += (int64_t)gridDim.y * 16 * AT) {
    i32x4_t acc[AT][AT];
    zero(acc);
    for (int32_t s = wave; s < steps; s += AW) {
      const int32_t kk = s * 64 + 16 * (lane >> 4);
      i32x4_t fa[AT], fb[AT];
#pragma unroll
      for (int t = 0; t < AT; ++t) {
        fa[t] = any16(p.a + (int64_t)min(i0 + 16 * t + (lane & 15), p.m - 1) * p.lda, kk, p.k);
        fb[t] = any16(p.b + (int64_t)min((int32_t)j0 + 16 * t + (lane & 15), p.n - 1) * p.ldb, kk, p.k);
      }
#pragma unroll
      for (int x = 0; x < AT; ++x)
#pragma unroll
        for (int y = 0; y < AT; ++y)
          acc[x][y] = __builtin_amdgcn_mfma_i32_16x16x64_i8(fa[x], fb[y], acc[x][y], 0, 0, 0);
    }
    join<AT, AT, AW>(p, part, acc, i0, (int32_t)j0, wave, lane, [&](int32_t j) { return gld<float>(p.sb + j); });
  }
}

// ---- few tokens -----------------------------------------------------------------------------------
// Up to 64 tokens: the weights' bytes count.  A workgroup has 16 TM channels and all tokens (16 TN); its NW
// wavefronts take consecutive stages of k, each with SLOTS places in LDS of its own, so that there is no barrier
// before the end: copies into a place are issued when its fragments have been read, and waited for by count.
// (Fragments straight from memory are 16 rows to every 16 lanes, a look-up of a line for every 16 bytes: the chain
// of the feed-forward step of 48 tokens, 4096 hidden, took 58 us, 48 so.)
constexpr int STAGE = 128;   // bytes of k

template <int N>
__device__ __forceinline__ void copy_rows(i32x4 from, const uint32_t* at, uint32_t to) {
  if constexpr (N == 6) {
    buffer_load_lds16_block<4>(from, at, to);
    buffer_load_lds16_block<2>(from, at + 4, to + 4096);
  } else {
    buffer_load_lds16_block<N>(from, at, to);
  }
}

// OWN: the tokens are activations x, few enough (OWN_BYTES with k rounded up to whole stages) that each
// workgroup makes their 8-bit rows itself, in LDS, beside the first weights: one launch for two.
enum { ROWS8, OWN_F32, OWN_BF16 };
constexpr int OWN_BYTES = 12288;
template <int TM, int TN, int NW, int SLOTS, int FROM>
__global__ __launch_bounds__(64 * NW) void q8_gemm_few_kernel(Q8GemmParams p) {
  constexpr bool OWN = FROM != ROWS8;
  constexpr int A_LOADS = 2 * TM, B_LOADS = OWN ? 0 : 2 * TN, LOADS = A_LOADS + B_LOADS, SLOT = LOADS * 1024;
  constexpr int RING = NW * SLOTS * SLOT, JOIN = NW * TM * TN * 1024;
  static_assert(!OWN || TN == 1, "up to 16 tokens");
  static_assert(RING <= 160 * 1024 && JOIN <= 160 * 1024, "LDS");
  static_assert(SLOTS * LOADS <= 64, "vmcnt");
  __shared__ __attribute__((aligned(1024))) char lds[RING > JOIN ? RING : JOIN];
  __shared__ __attribute__((aligned(16))) char own[OWN ? OWN_BYTES : 16];
  __shared__ uint32_t tops[16];
  const int32_t lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  const int32_t i0 = blockIdx.x * 16 * TM, j0 = OWN ? 0 : blockIdx.y * 16 * TN;
  const int32_t stages = (p.k + STAGE - 1) / STAGE, share = (stages + NW - 1) / NW;
  const int32_t s0 = min(wave * share, stages), s1 = min(s0 + share, stages);
  // a lane copies one 16-byte chunk of a row; rows' chunks XOR-swizzled as in the tiles below
  const int32_t sub = lane >> 3, pos = lane & 7;
  uint32_t la[A_LOADS], lb[B_LOADS + 1], ta[A_LOADS], tb[B_LOADS + 1];   // t: in a last stage that is not whole
  const int32_t last0 = (stages - 1) * STAGE;
  const auto offset = [&](int32_t row, int64_t ld, int32_t rows, uint32_t& whole, uint32_t& tail) {
    const int32_t c = (pos ^ ((row >> 1) & 7)) * 16;
    const uint32_t at = (uint32_t)(min(row, rows) * ld);
    whole = at + c;
    tail = at + (last0 + c < p.k ? c : 0);
  };
#pragma unroll
  for (int r = 0; r < A_LOADS; ++r) offset(r * 8 + sub, p.lda, p.m - 1 - i0, la[r], ta[r]);
#pragma unroll
  for (int r = 0; r < B_LOADS; ++r) offset(r * 8 + sub, p.ldb, p.n - 1 - j0, lb[r], tb[r]);
  const int8_t* base_a = p.a + (int64_t)i0 * p.lda;
  const int8_t* base_b = OWN ? nullptr : p.b + (int64_t)j0 * p.ldb;
  const uint32_t mine = __builtin_amdgcn_readfirstlane((uint32_t)(uintptr_t)(LDS_AS char*)lds) + wave * SLOTS * SLOT;
  const bool ragged = p.k % STAGE != 0;
  const auto issue = [&](int32_t s, int slot) {
    const i32x4 ra = raw_buffer(base_a + (int64_t)s * STAGE);
    const uint32_t to = mine + slot * SLOT;
    if (ragged && s == stages - 1) copy_rows<A_LOADS>(ra, ta, to);
    else copy_rows<A_LOADS>(ra, la, to);
    if constexpr (!OWN) {
      const i32x4 rb = raw_buffer(base_b + (int64_t)s * STAGE);
      if (ragged && s == stages - 1) copy_rows<B_LOADS>(rb, tb, to + A_LOADS * 1024);
      else copy_rows<B_LOADS>(rb, lb, to + A_LOADS * 1024);
    }
  };
  i32x4_t acc[TM][TN];
  zero(acc);
  const int32_t row = lane & 15, q = lane >> 4, swz = (row >> 1) & 7;
#pragma unroll
  for (int k = 0; k < SLOTS; ++k)
    if (s0 + k < s1) issue(s0 + k, k);
  const int32_t pitch = stages * STAGE;
  if constexpr (OWN) {
    constexpr bool BF16 = FROM == OWN_BF16;
    constexpr int C = OWN_BYTES / 8 / (64 * NW);   // chunks of 8 entries of a thread
    const int32_t chunks = pitch / 8;
    float v[C][8];
    if (threadIdx.x < 16) tops[threadIdx.x] = 0;
    __syncthreads();
#pragma unroll
    for (int c = 0; c < C; ++c) {
      const int32_t at = c * 64 * NW + threadIdx.x, j = at / chunks, e0 = (at - j * chunks) * 8;
      uint32_t top = 0;
      if (j < p.n) {
        const int64_t x = (int64_t)j * p.ldb + e0;
        if (e0 + 8 <= p.k) {
          widen<BF16>(load_raw<BF16, CACHED>(p.x, x), v[c]);
        } else {
#pragma unroll
          for (int e = 0; e < 8; ++e) v[c][e] = e0 + e < p.k ? load1<BF16>(p.x, x + e) : 0.0f;
        }
        top = top8<BF16>(narrow<BF16>(v[c]));
      }
      top = over_lanes<Top, 16>(top);   // (a row's chunks are a multiple of 16)
      if ((lane & 15) == 0 && j < p.n) atomicMax(&tops[j], top);
    }
    __syncthreads();
#pragma unroll
    for (int c = 0; c < C; ++c) {
      const int32_t at = c * 64 * NW + threadIdx.x, j = at / chunks, ch = at - j * chunks;
      if (j >= p.n) continue;
      const int32_t place = ((ch >> 1) & 7) ^ ((j >> 1) & 7);
      *reinterpret_cast<u32x2*>(own + j * pitch + (ch >> 4) * STAGE + place * 16 + (ch & 1) * 8) =
          q8_round(v[c], q8_group(tops[j]));
    }
    __syncthreads();
  }
  for (int32_t s = s0; s < s1; s += SLOTS) {
#pragma unroll
    for (int k = 0; k < SLOTS; ++k) {
      if (s + k >= s1) break;
      // this stage's copies are done when at most the later ones' are under way
      if (s + k + SLOTS - 1 < s1) __builtin_amdgcn_s_waitcnt(vmcnt_imm((SLOTS - 1) * LOADS));
      else __builtin_amdgcn_s_waitcnt(vmcnt_imm(0));
      asm volatile("" ::: "memory");
      __builtin_amdgcn_sched_barrier(0);
      const char* at = lds + (wave * SLOTS + k) * SLOT;
      i32x4_t fa[2][TM], fb[2][TN];
#pragma unroll
      for (int h = 0; h < 2; ++h) {
        const int32_t c = row * STAGE + (((4 * h + q) ^ swz) << 4);
        if constexpr (OWN) {
          const int32_t j = min(row, p.n - 1);
          fb[h][0] = *reinterpret_cast<const i32x4_t*>(own + j * pitch + (s + k) * STAGE +
                                                       (((4 * h + q) ^ ((j >> 1) & 7)) << 4));
        }
#pragma unroll
        for (int t = 0; t < TM; ++t) fa[h][t] = *reinterpret_cast<const i32x4_t*>(at + t * 2048 + c);
        if constexpr (!OWN) {
#pragma unroll
          for (int t = 0; t < TN; ++t) fb[h][t] = *reinterpret_cast<const i32x4_t*>(at + A_LOADS * 1024 + t * 2048 + c);
        }
      }
      asm volatile("s_waitcnt lgkmcnt(0)" ::: "memory");
      __builtin_amdgcn_sched_barrier(0);
      if (s + k + SLOTS < s1) issue(s + k + SLOTS, k);
      if (!OWN && ragged && s + k == stages - 1) {   // (rows made here are zero behind k)
#pragma unroll
        for (int h = 0; h < 2; ++h)
#pragma unroll
          for (int t = 0; t < TN; ++t) fb[h][t] = first_bytes(fb[h][t], p.k - last0 - 64 * h - 16 * q);
      }
#pragma unroll
      for (int h = 0; h < 2; ++h)
#pragma unroll
        for (int x = 0; x < TM; ++x)
#pragma unroll
          for (int y = 0; y < TN; ++y)
            acc[x][y] = __builtin_amdgcn_mfma_i32_16x16x64_i8(fa[h][x], fb[h][y], acc[x][y], 0, 0, 0);
    }
  }
  __syncthreads();
  join<TM, TN, NW>(p, *reinterpret_cast<i32x4_t (*)[NW][TM * TN][64]>(lds), acc, i0, j0, wave, lane,
                   [&](int32_t j) { return OWN ? q8_group(tops[j]).scale : gld<float>(p.sb + j); });
}

// ---- operands through LDS -------------------------------------------------------------------------
// A workgroup has a BM x BN tile of C.  A stage is 128 bytes of k of its rows and columns, copied from
// memory straight into one of SLOTS places in LDS (buffer_load_dwordx4 .. lds, a whole line to eight lanes)
// and read as 16-byte fragments, rows' chunks XOR-swizzled so that 16 rows meet all banks.  A wavefront has
// TM x TN products of 32 x 32 x 32; the fragments of a k-step are read while the one before is multiplied,
// across the stages too: the last k-step of a stage comes after the barrier that ends its reading, beside
// the next stage's first reads and the copies of A into the place that the barrier freed; those of B come beside
// the k-step after it (all at once: 1 % more).  256 x 256 tiles have 16 wavefronts of 64 x 64: 8 of 128 x 64, with
// fewer bytes read from LDS but twice the copies to issue by each, took 551 us where these took 532.
typedef int32_t i32x16 __attribute__((ext_vector_type(16)));

struct TileGrid {
  int32_t tiles_m, tiles_n, total, run, rest;   // tiles of an XCD, XCDs that have one more
};
// Workgroups go to the 8 XCDs in turn: each gets a run of tiles, in bands of 8 tile rows, so that the 32 it
// has at once share rows and columns in its L2.
__device__ __forceinline__ void tile_of(const TileGrid& g, int32_t& tm, int32_t& tn) {
  const int32_t xcd = blockIdx.x & 7, nth = blockIdx.x >> 3;
  const int32_t t = xcd * g.run + min(xcd, g.rest) + nth;
  const int32_t band = t / (8 * g.tiles_n), in = t - band * 8 * g.tiles_n;
  const int32_t rows = min(8, g.tiles_m - band * 8);
  tn = in / rows;
  tm = band * 8 + in - tn * rows;
}

template <int BM, int BN, int WM, int WN, int SLOTS, bool TAIL>
__global__ __launch_bounds__(64 * WM * WN, 2) void q8_gemm_tile_kernel(Q8GemmParams p, TileGrid grid) {
  constexpr int NW = WM * WN, WTM = BM / WM, WTN = BN / WN, TM = WTM / 32, TN = WTN / 32;
  constexpr int A_BYTES = BM * STAGE, SLOT = A_BYTES + BN * STAGE;
  constexpr int A_LOADS = A_BYTES / 1024 / NW, B_LOADS = BN * STAGE / 1024 / NW, LOADS = A_LOADS + B_LOADS;
  constexpr int KQ = STAGE / 32;
  constexpr int SLAB = 32 * WTM * 4;   // a wavefront's 32 columns of C on their way out
  constexpr int LDS = SLOTS * SLOT > NW * SLAB ? SLOTS * SLOT : NW * SLAB;
  static_assert(LDS <= 160 * 1024 && A_LOADS >= 1 && B_LOADS >= 1, "tile");
  constexpr int THREADS = 64 * NW;
  __shared__ __attribute__((aligned(1024))) char lds[LDS];
  __shared__ __attribute__((aligned(16))) float scales[BM], biases[BM], columns[BN];
  const int32_t lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  const int32_t wm = wave % WM, wn = wave / WM;
  int32_t tm_, tn_;
  tile_of(grid, tm_, tn_);
  const int32_t i0 = tm_ * BM, j0 = tn_ * BN;
  const int32_t stages = (p.k + STAGE - 1) / STAGE;

  // copies: load r of a wavefront fills 8 rows of 128 bytes; a lane has one chunk of one row (rows behind
  // the last read the last: they reach only outputs that are not stored)
  uint32_t la[A_LOADS], lb[B_LOADS];
  const int32_t sub = lane >> 3, pos = lane & 7;
  const auto chunk_at = [&](int32_t row) { return pos ^ ((row >> 1) & 7); };
#pragma unroll
  for (int r = 0; r < A_LOADS; ++r) {
    const int32_t row = (wave * A_LOADS + r) * 8 + sub;
    la[r] = (uint32_t)((int64_t)min(row, p.m - 1 - i0) * p.lda) + chunk_at(row) * 16;
  }
#pragma unroll
  for (int r = 0; r < B_LOADS; ++r) {
    const int32_t row = (wave * B_LOADS + r) * 8 + sub;
    lb[r] = (uint32_t)((int64_t)min(row, p.n - 1 - j0) * p.ldb) + chunk_at(row) * 16;
  }
  const int8_t* base_a = p.a + (int64_t)i0 * p.lda;
  const int8_t* base_b = p.b + (int64_t)j0 * p.ldb;
  const uint32_t lds_at = __builtin_amdgcn_readfirstlane((uint32_t)(uintptr_t)(LDS_AS char*)lds);
  // its copies of stage s: of A, of B
  const auto issue_a = [&](int32_t s) {
    const int32_t k0 = s * STAGE;
    const i32x4 from = raw_buffer(base_a + k0);
    const uint32_t to = lds_at + (uint32_t)(s % SLOTS) * SLOT + wave * A_LOADS * 1024;
    if (TAIL && k0 + STAGE > p.k) {   // chunks behind k: the stage's first (the products mask them)
      uint32_t at[A_LOADS];
#pragma unroll
      for (int r = 0; r < A_LOADS; ++r) {
        const int32_t c = chunk_at((wave * A_LOADS + r) * 8 + sub) * 16;
        at[r] = k0 + c < p.k ? la[r] : la[r] - c;
      }
      buffer_load_lds16_block<A_LOADS>(from, at, to);
    } else {
      buffer_load_lds16_block<A_LOADS>(from, la, to);
    }
  };
  const auto issue_b = [&](int32_t s) {
    const int32_t k0 = s * STAGE;
    const i32x4 from = raw_buffer(base_b + k0);
    const uint32_t to = lds_at + (uint32_t)(s % SLOTS) * SLOT + A_BYTES + wave * B_LOADS * 1024;
    if (TAIL && k0 + STAGE > p.k) {
      uint32_t at[B_LOADS];
#pragma unroll
      for (int r = 0; r < B_LOADS; ++r) {
        const int32_t c = chunk_at((wave * B_LOADS + r) * 8 + sub) * 16;
        at[r] = k0 + c < p.k ? lb[r] : lb[r] - c;
      }
      buffer_load_lds16_block<B_LOADS>(from, at, to);
    } else {
      buffer_load_lds16_block<B_LOADS>(from, lb, to);
    }
  };
  // this wavefront's copies of all but the newest `later` stages are done
  const auto landed = [&](int32_t later) {
    if (SLOTS > 3 && later >= 3) __builtin_amdgcn_s_waitcnt(vmcnt_imm(3 * LOADS));
    else if (SLOTS > 2 && later >= 2) __builtin_amdgcn_s_waitcnt(vmcnt_imm(2 * LOADS));
    else if (later >= 1) __builtin_amdgcn_s_waitcnt(vmcnt_imm(LOADS));
    else __builtin_amdgcn_s_waitcnt(vmcnt_imm(0));
  };

  const int32_t half = lane >> 5, swz = ((lane & 31) >> 1) & 7;
  const int32_t frag = (lane & 31) * STAGE + ((half ^ swz) << 4);   // (wavefronts' rows start at multiples of 32)
  const auto read = [&](int32_t s, int kq, i32x4_t (&fa)[TM], i32x4_t (&fb)[TN]) {
    const char* at = lds + (s % SLOTS) * SLOT;
    const int32_t f = frag ^ (kq << 5);
#pragma unroll
    for (int t = 0; t < TM; ++t) fa[t] = *reinterpret_cast<const i32x4_t*>(at + (wm * WTM + t * 32) * STAGE + f);
#pragma unroll
    for (int t = 0; t < TN; ++t) fb[t] = *reinterpret_cast<const i32x4_t*>(at + A_BYTES + (wn * WTN + t * 32) * STAGE + f);
  };
  i32x16 acc[TM][TN];
#pragma unroll
  for (int x = 0; x < TM; ++x)
#pragma unroll
    for (int y = 0; y < TN; ++y)
#pragma unroll
      for (int v = 0; v < 16; ++v) acc[x][y][v] = 0;
  const auto multiply = [&](int32_t s, int kq, const i32x4_t (&fa)[TM], i32x4_t (&fb)[TN]) {
    if (TAIL && s == stages - 1) {
      const int32_t have = p.k - s * STAGE - 32 * kq - 16 * half;
#pragma unroll
      for (int d = 0; d < 4; ++d) {
        const int32_t n = have - 4 * d;
        const uint32_t keep = n >= 4 ? ~0u : n <= 0 ? 0u : (1u << (8 * n)) - 1;
#pragma unroll
        for (int t = 0; t < TN; ++t) fb[t][d] &= keep;
      }
    }
#pragma unroll
    for (int x = 0; x < TM; ++x)
#pragma unroll
      for (int y = 0; y < TN; ++y) acc[x][y] = __builtin_amdgcn_mfma_i32_32x32x32_i8(fa[x], fb[y], acc[x][y], 0, 0, 0);
  };

  for (int32_t s = 0; s < SLOTS && s < stages; ++s) {
    issue_a(s);
    issue_b(s);
  }
  // what the epilogue reads of the tile's channels and tokens (visible from the next barrier on)
  const bool biased = p.flags & TPP_EPI_BIAS;
  for (int32_t t = threadIdx.x; t < BM; t += THREADS) {
    scales[t] = gld<float>(p.sa + min(i0 + t, p.m - 1));
    biases[t] = biased ? gld<float>(p.bias + min(i0 + t, p.m - 1)) : 0.0f;
  }
  for (int32_t t = threadIdx.x; t < BN; t += THREADS) columns[t] = gld<float>(p.sb + min(j0 + t, p.n - 1));
  landed(min(stages, SLOTS) - 1);
  lds_barrier();
  i32x4_t fa[2][TM], fb[2][TN];
  read(0, 0, fa[0], fb[0]);
  for (int32_t s = 0; s < stages; ++s) {
#pragma unroll
    for (int kq = 0; kq + 1 < KQ; ++kq) {
      read(s, kq + 1, fa[(kq + 1) & 1], fb[(kq + 1) & 1]);
      if (kq == 0 && s > 0 && s - 1 + SLOTS < stages) issue_b(s - 1 + SLOTS);
      __builtin_amdgcn_sched_barrier(0);   // the reads stay ahead of the products
      multiply(s, kq, fa[kq & 1], fb[kq & 1]);
      __builtin_amdgcn_sched_barrier(0);
    }
    if (s + 1 < stages) {
      landed(min(stages - 2 - s, SLOTS - 2));
      lds_barrier();   // every wavefront has read all of stage s, and stage s + 1 is there
      read(s + 1, 0, fa[0], fb[0]);
      if (s + SLOTS < stages) issue_a(s + SLOTS);
      __builtin_amdgcn_sched_barrier(0);
    }
    multiply(s, KQ - 1, fa[(KQ - 1) & 1], fb[(KQ - 1) & 1]);
    __builtin_amdgcn_sched_barrier(0);
  }
  lds_barrier();

  // C: a wavefront's 32 columns at a time through LDS, so that a store takes whole lines; the large tiles' past
  // the caches' replacement (C is 26 MB or more: the MLP block's first layer 66.5 -> 63.1 us)
  char* slab = lds + wave * SLAB;
  const int32_t iw = i0 + wm * WTM, col = lane & 31;
  const auto finish = [&](auto type, auto flags) {
    constexpr bool BF16 = decltype(type)::value;
    constexpr int V = BF16 ? 8 : 4, PER = WTM / V;   // entries of a 16-byte chunk, chunks of a column
#pragma unroll
    for (int y = 0; y < TN; ++y) {
      const int32_t jw = wn * WTN + y * 32;   // first column in the tile
      const float sb = columns[jw + col];
#pragma unroll
      for (int x = 0; x < TM; ++x)
#pragma unroll
        for (int q = 0; q < 4; ++q) {
          const int32_t r = x * 32 + 8 * q + 4 * half;   // first of four rows
          const f32x4 sa = *reinterpret_cast<const f32x4*>(scales + wm * WTM + r);
          const f32x4 bias = *reinterpret_cast<const f32x4*>(biases + wm * WTM + r);
          float v[4];
#pragma unroll
          for (int e = 0; e < 4; ++e)
            v[e] = activate((float)acc[x][y][4 * q + e] * sb * sa[e] + bias[e], (uint32_t)decltype(flags)::value);
          if constexpr (BF16) {
            const int32_t ch = (x * 4 + q) ^ (col & (PER - 1));
            *reinterpret_cast<u32x2*>(slab + col * WTM * 2 + ch * 16 + half * 8) =
                (u32x2){pack_bf16x2(v[0], v[1]), pack_bf16x2(v[2], v[3])};
          } else {
            const int32_t ch = ((x * 4 + q) * 2 + half) ^ (col & (PER - 1));
            *reinterpret_cast<f32x4*>(slab + col * WTM * 4 + ch * 16) = (f32x4){v[0], v[1], v[2], v[3]};
          }
          __builtin_amdgcn_sched_barrier(0);   // (all quads' scales read at once do not fit the registers)
        }
#pragma unroll
      for (int it = 0; it < 32 * PER / 64; ++it) {
        const int32_t c = (it * 64 + lane) / PER, ch = (it * 64 + lane) % PER;
        const u32x4 w = *reinterpret_cast<const u32x4*>(slab + c * WTM * (16 / V) + ((ch ^ (c & (PER - 1))) << 4));
        const int32_t i = iw + ch * V, j = j0 + jw + c;
        if (j >= p.n || i >= p.m) continue;
        char* to = static_cast<char*>(p.c) + ((int64_t)j * p.ldc + i) * (16 / V);
        if (i + V <= p.m) {
          if constexpr (BM == 256)
            __builtin_nontemporal_store((u32x4_a2)w, (GLOBAL_AS u32x4_a2*)to);
          else
            gst<u32x4_a2>(to, (u32x4_a2)w);
        } else {
#pragma unroll
          for (int e = 0; e < V; ++e) {
            if (i + e >= p.m) continue;
            if constexpr (BF16) gst<uint16_t>(to + 2 * e, (uint16_t)(w[e >> 1] >> (16 * (e & 1))));
            else gst<uint32_t>(to + 4 * e, w[e]);
          }
        }
      }
    }
  };
  const auto by_act = [&](auto type) {
    if (p.flags & TPP_EPI_GELU_TANH) finish(type, IntC<TPP_EPI_GELU_TANH>());
    else if (p.flags & TPP_EPI_RELU) finish(type, IntC<TPP_EPI_RELU>());
    else finish(type, IntC<0>());
  };
  if (p.c_bf16) by_act(std::true_type());
  else by_act(std::false_type());
}

template <int BM, int BN, int WM, int WN, int SLOTS>
hipError_t launch_tiles(const Q8GemmParams& p, hipStream_t stream) {
  TileGrid g;
  g.tiles_m = (int32_t)(((int64_t)p.m + BM - 1) / BM);
  g.tiles_n = (int32_t)(((int64_t)p.n + BN - 1) / BN);
  const int64_t total = (int64_t)g.tiles_m * g.tiles_n;
  if (total > most_groups(64 * WM * WN)) return hipErrorInvalidConfiguration;
  g.total = (int32_t)total;
  g.run = g.total / 8;
  g.rest = g.total % 8;
  if (p.k % STAGE)
    hipLaunchKernelGGL((q8_gemm_tile_kernel<BM, BN, WM, WN, SLOTS, true>), dim3(g.total), dim3(64 * WM * WN), 0, stream, p, g);
  else
    hipLaunchKernelGGL((q8_gemm_tile_kernel<BM, BN, WM, WN, SLOTS, false>), dim3(g.total), dim3(64 * WM * WN), 0, stream, p, g);
  return hipGetLastError();
}

template <int TM, int TN, int NW, int SLOTS, int FROM = ROWS8>
hipError_t launch_few(const Q8GemmParams& p, hipStream_t stream) {
  const int64_t rows = ((int64_t)p.m + 16 * TM - 1) / (16 * TM), cols = ((int64_t)p.n + 16 * TN - 1) / (16 * TN);
  if (rows * cols > most_groups(64 * NW)) return hipErrorInvalidConfiguration;
  hipLaunchKernelGGL((q8_gemm_few_kernel<TM, TN, NW, SLOTS, FROM>), dim3((uint32_t)rows, (uint32_t)cols), dim3(64 * NW),
                     0, stream, p);
  return hipGetLastError();
}
// Channels of a workgroup, its wavefronts and their places: 32 channels where m has 192 workgroups of them
// (48 tokens, 16384 channels of 1024: 11.0 us against 12.1 with 64 and 13.4 with 16), else 16; two workgroups
// to a compute unit where the places leave room (one token, 16384 channels of 8192: 29.3 against 33.8).
template <int TN>
hipError_t launch_few(const Q8GemmParams& p, hipStream_t stream) {
  if (p.m >= 192 * 32) return launch_few<2, TN, TN <= 2 ? 4 : 8, TN <= 2 ? 2 : 1>(p, stream);
  return launch_few<1, TN, 8, 1>(p, stream);
}
template <int FROM>
hipError_t launch_own(const Q8GemmParams& p, hipStream_t stream) {
  if (p.m >= 192 * 32) return launch_few<2, 1, 8, 1, FROM>(p, stream);
  return launch_few<1, 1, 8, 2, FROM>(p, stream);
}
// Whether the kernels that copy rows into LDS can take the weights (tokens): 16-byte chunks, and offsets inside
// a tile that count in 31 bits.
bool copied(const int8_t* rows, int64_t ld) {
  return ((reinterpret_cast<uintptr_t>(rows) | (uint64_t)ld) & 15) == 0 && ld <= 0x7fffffff / 256;
}

}  // namespace

bool q8_linear_at_once(const Q8GemmParams& p) {
  return p.n <= 16 && copied(p.a, p.lda) && (int64_t)p.n * ((p.k + STAGE - 1) / STAGE * STAGE) <= OWN_BYTES;
}

hipError_t launch_q8_linear_at_once(const Q8GemmParams& p, bool bf16, hipStream_t stream) {
  return bf16 ? launch_own<OWN_BF16>(p, stream) : launch_own<OWN_F32>(p, stream);
}

hipError_t launch_q8_gemm(const Q8GemmParams& p, hipStream_t stream) {
  if (!copied(p.a, p.lda) || !copied(p.b, p.ldb)) {
    const int64_t rows = ((int64_t)p.m + 16 * AT - 1) / (16 * AT), cols = ((int64_t)p.n + 16 * AT - 1) / (16 * AT);
    const int64_t most = most_groups(64 * AW) / rows, ny = cols < most ? cols : most;
    if (most < 1) return hipErrorInvalidConfiguration;
    hipLaunchKernelGGL(q8_gemm_any_kernel, dim3((uint32_t)rows, (uint32_t)(ny < 65535 ? ny : 65535)), dim3(64 * AW), 0,
                       stream, p);
    return hipGetLastError();
  }
  if (p.n <= 16) return launch_few<1>(p, stream);
  if (p.n <= 32) return launch_few<2>(p, stream);
  if (p.n <= 48) return launch_few<3>(p, stream);
  if (p.n <= 64) return launch_few<4>(p, stream);
  // The largest tile that gives most compute units one (256 x 256: 4096 x 4096 of 1024 36.9 us against 42.6 with
  // 128 x 128, which take 51.1 against 61.5 for 2048 x 4096 of 4096, 128 large tiles); 64 x 64 where there are
  // fewer than two of 128 x 128 to a unit's two places (1533 x 777 of 1001 14.8 against 29.3 with 256 x 256);
  // wavefronts with shares of k where even those are few (538 x 192 of 1296 10.4 against 12.9, but 1533 x 777
  // 18.8 against 14.9).  64 x 64 tiles have four places, or two where there are more tiles than the units hold
  // with four (5146 x 581 of 704 20.8 against 24.1; 512 x 2048 of 8192 26.6 against 40.0 the other way).
  const auto tiles = [&](int64_t side) { return ((p.m + side - 1) / side) * ((p.n + side - 1) / side); };
  if (tiles(256) >= 200) return launch_tiles<256, 256, 4, 4, 2>(p, stream);
  if (tiles(128) >= 256) return launch_tiles<128, 128, 2, 2, 2>(p, stream);
  if (tiles(64) < 128) return launch_few<4>(p, stream);
  if (tiles(64) <= 512) return launch_tiles<64, 64, 2, 2, 4>(p, stream);
  return launch_tiles<64, 64, 2, 2, 2>(p, stream);
}

}  // namespace tpp

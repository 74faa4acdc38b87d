// attention_kernels.hip -- attention of one new token per sequence over a paged key-value cache, for
// gfx950.
//
// Per sequence and query head: scores s_t = scale q . k_t over the positions that are held, their
// softmax, and the sum of the values with it, in one pass with the running maximum m and sum l of the
// softmax (when m grows, the sums so far are scaled down).  Scores are kept times log2 e, so that the
// exponential is the hardware's exp2.
//
// A workgroup takes one key head of one sequence, up to 16 (or 32) of the query heads that read it, and
// a span of positions; its four wavefronts take the span's tiles in turn and meet at the end.  Both
// products are matrix instructions whose operands never leave registers:
//   S^T = K Q^T   A: keys as they lie in memory (a lane holds consecutive entries of one key), B: queries
//   O^T = V^T P^T B: the softmax weights where the first product left them (a lane has the weights of one
//                 query head and of the keys whose values it loads), A: values, turned within a lane.
// The order of the entries in the first product and of the keys in the second is free, which is what
// lets both operands of each fit the layouts: no lane exchanges anything but the maximum.
//   bf16: 32 keys a tile, v_mfma_f32_16x16x32_bf16; a lane loads whole chunks of V of 8 keys and turns
//         them with byte permutes.  The weights enter as three bf16 parts whose sum is the fp32 weight
//         (8 bits of its 24 each); one would cost an fp32 output 2^-9 of its value, two 2^-17.
//   fp32: 16 keys a tile, v_mfma_f32_16x16x4_f32, whose operands are single entries: nothing to turn.
// Fewer queries than 16 leave columns of the instructions idle, which costs nothing: a tile of 16 KB
// (128 entries a head) takes 512 cycles of a SIMD's matrix unit in bf16 (two parts of the weights 384, with
// the same time of every call to 2%), 2048 in fp32, and 5000 or more of its share of HBM.
//
// The rows' addresses are looked up once per span and kept in LDS.  A position that is not held gets the
// address of one that is, and a mark that sets its score to -inf: loads need no branches, and nothing
// but held positions is ever read.
//
// An infinite value has no place in the products: a weight of 0, one of a weight's parts, or a masked place
// that stands on its row would make it NaN.  Its entry's sum is known without them -- the weights are
// positive, so it is that infinity, or NaN where both signs or a NaN are held -- and comes out of the products
// as infinite or NaN in any case, so that only then the span's values of the entry are looked up again.
//
// Bound by HBM where the cache is large.  32 heads to 8 of 128 bf16: 64 sequences of 4096 180 us, 6.0 TB/s;
// 64 of 1 to 8192 191 us, 5.6 TB/s, 7 of them the join; one of 131072 96 us, 5.6 TB/s; 32 of 2049 to 4096
// with totals 92 us, 4.4 TB/s (a kernel that only reads as many bytes: 7.1 to 7.2 TB/s).  One of 100 positions
// 5.5 us from call to call, 4.6 of them the GPU's: the loads of length, page, keys and values wait for each
// other.
#include <hip/hip_runtime.h>

#include <type_traits>

#include "brgemm_device.h"
#include "internal.h"

namespace tpp {
namespace {

using namespace dev;

constexpr int AT = 256;          // threads of a workgroup: 4 wavefronts
constexpr int AW = AT / 64;
constexpr float LOG2E = 1.4426950408889634f, LN2 = 0.6931471805599453f;

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
// First position inside the window.
__device__ __forceinline__ int32_t window_start(const AttnParams& p, int32_t n) {
  return p.window > 0 && n > p.window ? (int32_t)(n - p.window) : 0;
}

// The maximum, or the sum, over the four groups of 16 lanes.
__device__ __forceinline__ float groups_max(float v) {
  auto w = __builtin_amdgcn_permlane16_swap(__float_as_uint(v), __float_as_uint(v), false, false);
  v = fmaxf(__uint_as_float(w[0]), __uint_as_float(w[1]));
  w = __builtin_amdgcn_permlane32_swap(__float_as_uint(v), __float_as_uint(v), false, false);
  return fmaxf(__uint_as_float(w[0]), __uint_as_float(w[1]));
}
__device__ __forceinline__ float groups_sum(float v) {
  auto w = __builtin_amdgcn_permlane16_swap(__float_as_uint(v), __float_as_uint(v), false, false);
  v = __uint_as_float(w[0]) + __uint_as_float(w[1]);
  w = __builtin_amdgcn_permlane32_swap(__float_as_uint(v), __float_as_uint(v), false, false);
  return __uint_as_float(w[0]) + __uint_as_float(w[1]);
}

// v moved down by d dwords (0 .. 4), zeros behind.
__device__ __forceinline__ u32x4 shift_dwords(u32x4 v, int32_t d) {
  if (d & 1) v = (u32x4){v.y, v.z, v.w, 0u};
  if (d & 2) v = (u32x4){v.z, v.w, 0u, 0u};
  if (d & 4) v = (u32x4){0u, 0u, 0u, 0u};
  return v;
}

// How much sums of maximum m count in sums of maximum top (>= m; both may be -inf, and sums may be NaN).
__device__ __forceinline__ float share(float m, float top) {
  return m == top ? 1.0f : __builtin_amdgcn_exp2f(m - top);
}

constexpr int32_t BLOCK = 1024;   // most positions whose addresses are in LDS at a time
constexpr int JOINED = 4;         // partial results that a lane of the joining kernel has in flight
constexpr int SCORES = 16;        // heads whose scores of a position a lane has in flight
constexpr int LOOK = 8;           // values in flight of an entry whose sum is not finite
constexpr int32_t MEET = 8;       // query heads whose sums are in LDS at a time

// What one launch needs beside AttnParams.
struct AttnPlan {
  int32_t span;       // positions of a workgroup
  int32_t splits;     // spans of a sequence
  int32_t group;      // query heads of a key head
  int32_t tiles;      // query-head tiles of a key head
  FastDiv div_splits, div_seqs, div_tiles;
  int32_t round;      // workgroups of 8 spans of all key heads, where those go together, or 0
  FastDiv div_round;
  // Partial results (null: the workgroup writes the outputs): sums [row][split][D], then maxima and
  // sums of weights [row][split], row = sequence * q_heads + head; scores [row][score_ld] for totals.
  float *o, *m, *l, *s;
  int64_t score_ld;   // of a row of scores: max_len in an odd number of 256-byte lines
  int32_t block;      // positions whose addresses, and with totals whose scores, are in LDS at a time
  int32_t stage_ld;   // of a head's scores in LDS
};

// The kernel's shapes by type: keys of a tile, entries of a key step and of a lane's chunk of it.
template <bool BF16>
struct Shape {
  static constexpr int KEYS = BF16 ? 32 : 16;
  static constexpr int STEP = BF16 ? 32 : 16;
  static constexpr int CH = BF16 ? 8 : 4;
  static constexpr int SUB = KEYS / 16;
  static constexpr int VKEYS = 4 * SUB;     // keys whose values a lane loads
};

// DP: entries of a head the instance covers (D <= DP); TAIL: D < DP; NT: tiles of 16 query heads; TOTALS:
// the scores are kept.
template <bool BF16, int DP, bool TAIL, int NT, bool TOTALS>
__global__ __launch_bounds__(AT) void attn_kernel(AttnParams p, AttnPlan pl) {
  using S = Shape<BF16>;
  constexpr int ES = BF16 ? 2 : 4;
  constexpr int KEYS = S::KEYS, CH = S::CH, SUB = S::SUB, VKEYS = S::VKEYS;
  constexpr int NK = DP / S::STEP;                   // steps of the first product
  constexpr int VC = BF16 && DP > 64 ? 8 : 4;        // entries of a lane's chunk of a value
  constexpr int NV = (DP + 16 * VC - 1) / (16 * VC); // chunks
  // Values are read once, whole lines by one load: past the caches' replacement (64 sequences of 4096: 198 us
  // without, 180 so; a sequence of 131072 108 and 99).  The keys' lines take two loads, which would then both
  // go to memory (64 of 1 to 8192 196 us, 205 so), and rows that are no whole lines share some with the next.
  constexpr bool STREAM = !TAIL && DP * ES % 128 == 0;
  constexpr bool OVER = TAIL || DP % (16 * VC) != 0; // lanes past the last entry take the last chunk
  typedef typename std::conditional<VC * ES == 16, u32x4, u32x2>::type vchunk;
  typedef typename std::conditional<VC * ES == 16, u32x4_a2, u32x2_a2>::type vchunk_any;

  extern __shared__ __align__(16) char lds[];
  int64_t* rows = reinterpret_cast<int64_t*>(lds);   // byte offset of each position, bit 0: masked
  float* stage = reinterpret_cast<float*>(rows + pl.block);   // scores [query head][stage_ld]
  __shared__ int32_t missing;   // 1 + the first position of the last block that lacks a page
  __shared__ int32_t first_held;
  __shared__ float wave_m[AW][NT * 16], wave_l[AW][NT * 16];

  const int tid = threadIdx.x, lane = tid & 63, wave = tid >> 6;
  const int col = lane & 15, grp = lane >> 4;
  // Spans first, those of each sequence and head from another one on, then sequences, heads last.
  // Workgroups go to the 8 XCDs in turn: with every sequence's first span on the same XCD, the others had
  // only the work of long sequences (64 of 1 to 8192: 253 us so, 213 turned by the sequence, which is as
  // uneven for each head, 196 by both).  With the heads first the interleaved rows of the heads are read at
  // once, at a lower rate (206 us; 64 of 4096 191, 180 so; 32 of 2049 to 4096 with totals 99 and 93).
  // Workgroups of two head tiles, one to a compute unit, often run all at once: those of a key head are turned
  // alike, so that a span is read by one XCD (64 heads to one: 64 sequences of 8192 102 us turned by the tile,
  // 87 so, one of 131072 37.3 and 31.4; of one tile each, 24 heads of 192 to one, 64 sequences of 1 to 4096
  // 65.2 by the tile, 68.9 alike).
  // Where rows share lines with other heads' (plan()), all heads of a span follow each other on one XCD,
  // whose L2 has what they share.
  int32_t seq, sp, y, turn;
  if (pl.round) {
    const int32_t r = fdiv(blockIdx.x, pl.div_round), in = (int32_t)blockIdx.x - r * pl.round;
    const int32_t u = r * 8 + (in & 7);
    y = in >> 3;
    seq = fdiv(u, pl.div_splits);
    sp = u - seq * pl.splits;
    if (seq >= p.n_seqs) return;   // of the last round
    turn = seq;
  } else {
    const int32_t ys = fdiv(blockIdx.x, pl.div_splits);
    sp = (int32_t)blockIdx.x - ys * pl.splits;
    y = fdiv(ys, pl.div_seqs);
    seq = ys - y * (int32_t)p.n_seqs;
    turn = seq + (NT == 2 ? fdiv(y, pl.div_tiles) : y);
  }
  const int32_t from = turn - fdiv(turn, pl.div_splits) * pl.splits;
  const int32_t split = sp + from >= pl.splits ? sp + from - pl.splits : sp + from;
  const int32_t hk = fdiv(y, pl.div_tiles), ht = y - hk * pl.tiles;
  const int64_t b = seq;
  const int32_t D = TAIL ? p.d : DP;
  if (tid == 0) missing = 0;
  const int32_t n = length_of(p, b);
  const int32_t lo = window_start(p, n);
  const int32_t c0 = lo / KEYS * KEYS + split * pl.span;   // this span: [c0, c1)
  const int32_t c1 = c0 + pl.span < n ? c0 + pl.span : n;
  const int32_t nq = pl.group - ht * 16 * NT < 16 * NT ? pl.group - ht * 16 * NT : 16 * NT;
  const int32_t h0 = hk * pl.group + ht * 16 * NT;          // first query head
  if (c0 >= n && (pl.o || split > 0)) return;               // (an unsplit launch writes its zeros)

  // ---- queries: the first product's B operand -----------------------------------------------------
  u32x4 qf[NT][NK];
  const char* qb = static_cast<const char*>(p.q) + (b * p.ldq + (int64_t)h0 * D) * ES;
#pragma unroll
  for (int q = 0; q < NT; ++q)
#pragma unroll
    for (int s = 0; s < NK; ++s) {
      const int32_t h = q * 16 + col, e = s * S::STEP + grp * CH;
      u32x4 v = {0u, 0u, 0u, 0u};
      if (h < nq && e < D) {
        const int32_t e0 = TAIL && e > D - CH ? D - CH : e;
        v = gld<u32x4_a2>(qb + ((int64_t)h * D + e0) * ES);
        if (TAIL) v = BF16 ? shift_down(v, e - e0) : shift_dwords(v, e - e0);
      }
      qf[q][s] = v;
    }

  const char* kb = static_cast<const char*>(p.k) + hk * p.head_stride * ES;
  const char* vb = static_cast<const char*>(p.v) + hk * p.head_stride * ES;
  u32x4 kf[SUB][NK];
  vchunk vf[VKEYS][NV];
  const auto load_k = [&](int32_t i0) {
#pragma unroll
    for (int u = 0; u < SUB; ++u) {
      const char* row = kb + (rows[i0 + u * 16 + col] & ~int64_t(1));
#pragma unroll
      for (int s = 0; s < NK; ++s) {
        const int32_t e = s * S::STEP + grp * CH;
        kf[u][s] = gld<u32x4_a2>(row + (TAIL && e > D - CH ? D - CH : e) * ES);
      }
    }
  };
  uint32_t masks = 0;   // bit k: key k of this lane is masked
  const auto load_v = [&](int32_t i0) {
    masks = 0;
#pragma unroll
    for (int k = 0; k < VKEYS; ++k) {
      const int64_t row = rows[i0 + (k >> 2) * 16 + grp * 4 + (k & 3)];
      masks |= (uint32_t)(row & 1) << k;
#pragma unroll
      for (int c = 0; c < NV; ++c) {
        const int32_t e = (c * 16 + col) * VC;
        const GLOBAL_AS vchunk_any* at =
            (const GLOBAL_AS vchunk_any*)(vb + (row & ~int64_t(1)) + (OVER && e > D - VC ? D - VC : e) * ES);
        vf[k][c] = STREAM ? (vchunk)__builtin_nontemporal_load(at) : (vchunk)*at;
      }
    }
  };

  f32x4 acc[NT][NV * VC];
  float m[NT], l[NT];
#pragma unroll
  for (int q = 0; q < NT; ++q) {
    m[q] = -INFINITY;
    l[q] = 0.0f;
#pragma unroll
    for (int j = 0; j < NV * VC; ++j) acc[q][j] = (f32x4){0.0f, 0.0f, 0.0f, 0.0f};
  }
  const float sl2 = p.scale * LOG2E;

  // The tile at i0 of a block, whose loads have been issued; MORE: issues the next one's, the keys'
  // as soon as the first product has read theirs, the values' after the second, so that one of the two is
  // always in flight.
  const auto tile = [&](auto more, int32_t i0, int32_t next) {
    constexpr bool MORE = decltype(more)::value;
    float sc[NT][VKEYS];
#pragma unroll
    for (int u = 0; u < SUB; ++u) {
      f32x4 st[NT];
#pragma unroll
      for (int q = 0; q < NT; ++q) st[q] = (f32x4){0.0f, 0.0f, 0.0f, 0.0f};
#pragma unroll
      for (int s = 0; s < NK; ++s) {
        u32x4 a = kf[u][s];
        if constexpr (TAIL) {
          const int32_t e = s * S::STEP + grp * CH, over = e > D - CH ? e - (D - CH) : 0;
          a = BF16 ? shift_down(a, over < 8 ? over : 8) : shift_dwords(a, over < 4 ? over : 4);
        }
#pragma unroll
        for (int q = 0; q < NT; ++q) {
          if constexpr (BF16) {
            st[q] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(__builtin_bit_cast(bf16x8, a),
                                                            __builtin_bit_cast(bf16x8, qf[q][s]),
                                                            st[q], 0, 0, 0);
          } else {
#pragma unroll
            for (int e = 0; e < 4; ++e)
              st[q] = __builtin_amdgcn_mfma_f32_16x16x4f32(__uint_as_float(a[e]),
                                                           __uint_as_float(qf[q][s][e]), st[q], 0, 0, 0);
          }
        }
      }
#pragma unroll
      for (int q = 0; q < NT; ++q)
#pragma unroll
        for (int r = 0; r < 4; ++r)
          sc[q][u * 4 + r] = (masks >> (u * 4 + r)) & 1 ? -INFINITY : st[q][r] * sl2;
    }
    if constexpr (MORE) load_k(next);   // behind the products that read the registers
    __builtin_amdgcn_sched_barrier(0);

    if constexpr (TOTALS) {   // the scores of the columns that are a query head's
#pragma unroll
      for (int q = 0; q < NT; ++q)
        if (q * 16 + col < nq)
#pragma unroll
          for (int u = 0; u < SUB; ++u)
            *reinterpret_cast<f32x4*>(stage + (q * 16 + col) * pl.stage_ld + i0 + u * 16 + grp * 4) =
                (f32x4){sc[q][4 * u], sc[q][4 * u + 1], sc[q][4 * u + 2], sc[q][4 * u + 3]};
    }
    // ---- softmax: the maximum over the tile, the sums so far scaled down to it ------------------
    u32x4 parts[3][NT];
    float pr[NT][VKEYS];
#pragma unroll
    for (int q = 0; q < NT; ++q) {
      float top = sc[q][0];
#pragma unroll
      for (int k = 1; k < VKEYS; ++k) top = fmaxf(top, sc[q][k]);
      top = fmaxf(m[q], groups_max(top));
      const float base = top == -INFINITY ? 0.0f : top;
      const float down = __builtin_amdgcn_exp2f(m[q] - base);
      m[q] = top;
      l[q] *= down;
#pragma unroll
      for (int k = 0; k < VKEYS; ++k) {
        pr[q][k] = __builtin_amdgcn_exp2f(sc[q][k] - base);
        l[q] += pr[q][k];
      }
#pragma unroll
      for (int j = 0; j < NV * VC; ++j) acc[q][j] *= down;
      if constexpr (BF16) {
#pragma unroll
        for (int k = 0; k < 4; ++k) {
          float a = pr[q][2 * k], c = pr[q][2 * k + 1];
#pragma unroll
          for (int i = 0; i < 3; ++i) {   // what a part leaves is exact
            const uint32_t w = pack_bf16x2(a, c);
            parts[i][q][k] = w;
            a -= __uint_as_float(w << 16);
            c -= __uint_as_float(w & 0xffff0000u);
          }
        }
      }
    }
    // ---- the values -----------------------------------------------------------------------------
#pragma unroll
    for (int c = 0; c < NV; ++c) {
      if constexpr (BF16) {
#pragma unroll
        for (int j = 0; j < VC; ++j) {
          // entry j of the chunks of 8 keys, two keys a dword
          u32x4 a;
#pragma unroll
          for (int k = 0; k < 4; ++k)
            a[k] = __builtin_amdgcn_perm(vf[2 * k + 1][c][j / 2], vf[2 * k][c][j / 2],
                                         j & 1 ? 0x07060302u : 0x05040100u);
#pragma unroll
          for (int q = 0; q < NT; ++q) {
            f32x4& o = acc[q][c * VC + j];
#pragma unroll
            for (int i = 0; i < 3; ++i)
              o = __builtin_amdgcn_mfma_f32_16x16x32_bf16(__builtin_bit_cast(bf16x8, a),
                                                          __builtin_bit_cast(bf16x8, parts[i][q]), o, 0, 0, 0);
          }
        }
      } else {
#pragma unroll
        for (int j = 0; j < VC; ++j)
#pragma unroll
          for (int k = 0; k < VKEYS; ++k)
#pragma unroll
            for (int q = 0; q < NT; ++q)
              acc[q][c * VC + j] = __builtin_amdgcn_mfma_f32_16x16x4f32(
                  __uint_as_float(vf[k][c][j]), pr[q][k], acc[q][c * VC + j], 0, 0, 0);
      }
    }
    if constexpr (MORE) load_v(next);
    __builtin_amdgcn_sched_barrier(0);
  };

  constexpr int32_t step = AW * KEYS, NONE = 0x7fffffff;
  for (int32_t t0 = c0; t0 < c1; t0 += pl.block) {
    // ---- addresses of the block's rows --------------------------------------------------------------
    // A position outside the span's or the window's gets the row of the nearest one inside, masked.  Where
    // pages hold nothing, the first position that is held stands in for those that are not.
    const int32_t cnt = c1 - t0 < pl.block ? (c1 - t0 + KEYS - 1) / KEYS * KEYS : pl.block;
    __syncthreads();   // the block before is done with
    for (int32_t i = tid; i < cnt; i += AT) {
      const int32_t t = t0 + i, in = t < lo ? lo : t < c1 ? t : c1 - 1;
      const int64_t row = row_of(p, b, in);
      if (row < 0) missing = t0 + 1;
      rows[i] = row < 0 ? -1 : row * ES | (in != t);
    }
    __syncthreads();
    if (missing == t0 + 1) {   // the same for the whole workgroup
      if (tid == 0) first_held = NONE;
      __syncthreads();
      int32_t mine = NONE;
      for (int32_t i = tid; i < cnt && mine == NONE; i += AT)
        if (rows[i] >= 0) mine = i;
      if (mine != NONE) atomicMin(&first_held, mine);
      __syncthreads();
      if (first_held == NONE) continue;   // the same for the whole workgroup
      const int64_t safe = rows[first_held] | 1;
      __syncthreads();
      for (int32_t i = tid; i < cnt; i += AT)
        if (rows[i] < 0) rows[i] = safe;
      __syncthreads();
    }

    // ---- its tiles ----------------------------------------------------------------------------------
    int32_t i0 = wave * KEYS;
    if (i0 < cnt) {
      load_k(i0);
      load_v(i0);
      for (; i0 + step < cnt; i0 += step) tile(std::true_type(), i0, i0 + step);
      tile(std::false_type(), i0, 0);
    }
    // ---- its scores: a query head's row to a wavefront ------------------------------------------------
    // (Stored by each tile, 64 bytes of a head at a time: 32 sequences of 2049 to 4096 103 us, 95 so.)
    if constexpr (TOTALS) {
      __syncthreads();
      for (int32_t h = wave; h < nq; h += AW) {
        float* to = pl.s + (b * p.q_heads + h0 + h) * pl.score_ld + t0;
        for (int32_t i = lane * 4; i < cnt; i += 256)
          gst<f32x4_a4>(to + i, *reinterpret_cast<const f32x4*>(stage + h * pl.stage_ld + i));
      }
    }
  }

  // The sum of entry e, o by the products, where it is not finite: by the values held in the span, LOOK of them
  // at a time.
  const auto without_products = [&](float o, int32_t e) {
    uint32_t found = 0;   // 1: +inf, 2: -inf, 3: both, or NaN
    for (int32_t t = c0 < lo ? lo : c0; t < c1 && found != 3; t += LOOK) {
      float v[LOOK];
#pragma unroll
      for (int u = 0; u < LOOK; ++u) {
        const int64_t row = row_of(p, b, t + u < c1 ? t + u : c1 - 1);
        v[u] = row < 0 ? 0.0f : load_elem(vb, row + e, BF16);
      }
#pragma unroll
      for (int u = 0; u < LOOK; ++u)
        if (v[u] - v[u] != 0.0f) found |= v[u] > 0.0f ? 1u : v[u] < 0.0f ? 2u : 3u;
    }
    return found == 0 ? o : found == 1 ? INFINITY : found == 2 ? -INFINITY : NAN;
  };

  // ---- the wavefronts meet ------------------------------------------------------------------------
#pragma unroll
  for (int q = 0; q < NT; ++q) {
    l[q] = groups_sum(l[q]);
    if (grp == 0) {
      wave_m[wave][q * 16 + col] = m[q];
      wave_l[wave][q * 16 + col] = l[q];
    }
  }
  float* part = reinterpret_cast<float*>(lds);   // [wavefront][query of the pass][D]
  for (int32_t g0 = 0; g0 < nq; g0 += MEET) {
    const int32_t ng = nq - g0 < MEET ? nq - g0 : MEET;
    __syncthreads();   // the rows' addresses, or the pass before, are done with
#pragma unroll
    for (int q = 0; q < NT; ++q) {
      const int32_t h = q * 16 + col - g0;
      if (h < 0 || h >= ng) continue;
      float top = wave_m[0][g0 + h];
#pragma unroll
      for (int w = 1; w < AW; ++w) top = fmaxf(top, wave_m[w][g0 + h]);
      const float down = share(m[q], top);
#pragma unroll
      for (int c = 0; c < NV; ++c)
#pragma unroll
        for (int r = 0; r < 4; ++r) {
          const int32_t e = (c * 16 + grp * 4 + r) * VC;
          float* to = part + (wave * ng + h) * D + (OVER && e > D - VC ? D - VC : e);
#pragma unroll
          for (int j = 0; j < VC; ++j) to[j] = acc[q][c * VC + j][r] * down;
        }
    }
    __syncthreads();
    for (int32_t i = tid; i < ng * D; i += AT) {
      const int32_t hp = i / D, h = g0 + hp, e = i - hp * D;
      float top = wave_m[0][h];
#pragma unroll
      for (int w = 1; w < AW; ++w) top = fmaxf(top, wave_m[w][h]);
      float sum = 0.0f, o = 0.0f;
#pragma unroll
      for (int w = 0; w < AW; ++w) {
        sum += wave_l[w][h] * share(wave_m[w][h], top);
        o += part[w * ng * D + i];
      }
      if (__builtin_expect(o - o != 0.0f && sum == sum, 0)) o = without_products(o, e);
      const int64_t row = b * p.q_heads + h0 + h;
      if (pl.o) {
        const int64_t at = row * pl.splits + split;
        gst<float>(pl.o + at * D + e, o);
        if (e == 0) {
          gst<float>(pl.m + at, top);
          gst<float>(pl.l + at, sum);
        }
      } else {
        store_elem(p.out, b * p.ldo + (int64_t)(h0 + h) * D + e, sum == 0.0f ? 0.0f : o / sum, p.out_bf16);
        if (e == 0 && p.lse)
          gst<float>(p.lse + row, sum == 0.0f ? -INFINITY : (top + __builtin_amdgcn_logf(sum)) * LN2);
      }
    }
  }
}

// (A join by the last workgroup to finish, with a counter per unit, saves this launch; the releases of its
// writes to the device cost every workgroup a write-back of its L2: 64 sequences of 1 to 8192 1032 us, 224
// so, one of 1024 14.3 us and 10.6.)
// The spans' partial results joined: the first `rows` workgroups a (sequence, query head) each, whose
// wavefronts take the spans in turn; the others, with totals, a position of a sequence to a thread.
// NE: entries of a lane; JW: wavefronts.
template <int NE, int JW>
__global__ __launch_bounds__(JW * 64) void attn_join_kernel(AttnParams p, AttnPlan pl, int32_t rows,
                                                       int32_t blocks, int32_t keys) {
  __shared__ float lse[JW * 64];
  __shared__ float part[JW][NE * 64];
  const int tid = threadIdx.x, lane = tid & 63, wave = tid >> 6;
  if ((int32_t)blockIdx.x < rows) {
    const int64_t row = blockIdx.x;
    const int32_t b = (int32_t)row / p.q_heads, h = (int32_t)row - b * p.q_heads;
    const int32_t n = length_of(p, b), lo = window_start(p, n) / keys * keys;
    const int32_t used = n > lo ? (n - lo + pl.span - 1) / pl.span : 0;
    const float* mm = pl.m + row * pl.splits;
    const float* ll = pl.l + row * pl.splits;
    float top = -INFINITY;
    for (int32_t s = lane; s < used; s += 64) top = fmaxf(top, gld<float>(mm + s));
#pragma unroll
    for (int d = 32; d > 0; d >>= 1) top = fmaxf(top, __shfl_xor(top, d, 64));
    float sum = 0.0f, o[NE];
#pragma unroll
    for (int i = 0; i < NE; ++i) o[i] = 0.0f;
    for (int32_t s0 = 0; s0 < used; s0 += 64) {
      const float f = s0 + lane < used ? share(gld<float>(mm + s0 + lane), top) : 0.0f;
      if (s0 + lane < used) sum += gld<float>(ll + s0 + lane) * f;
      const int32_t end = used - s0 < 64 ? used - s0 : 64;
      for (int32_t s = wave; s < end; s += JOINED * JW) {   // JOINED spans' rows in flight
        float x[JOINED][NE];
#pragma unroll
        for (int u = 0; u < JOINED; ++u)
#pragma unroll
          for (int i = 0; i < NE; ++i)
            x[u][i] = s + u * JW < end && lane + 64 * i < p.d
                          ? gld<float>(pl.o + (row * pl.splits + s0 + s + u * JW) * p.d + lane + 64 * i)
                          : 0.0f;
#pragma unroll
        for (int u = 0; u < JOINED; ++u) {
          const float fs = __shfl(f, (s + u * JW) & 63, 64);   // 0 past the last span
#pragma unroll
          for (int i = 0; i < NE; ++i) {
            const float y = x[u][i] * fs;
            o[i] += y == y ? y : x[u][i];   // an infinity is one whatever its part's share
          }
        }
      }
    }
#pragma unroll
    for (int d = 32; d > 0; d >>= 1) sum += __shfl_xor(sum, d, 64);
#pragma unroll
    for (int i = 0; i < NE; ++i) part[wave][lane + 64 * i] = o[i];
    __syncthreads();
    if (tid < p.d) {
      float v = part[0][tid];
#pragma unroll
      for (int w = 1; w < JW; ++w) v += part[w][tid];
      store_elem(p.out, b * p.ldo + (int64_t)h * p.d + tid, sum == 0.0f ? 0.0f : v / sum, p.out_bf16);
    }
    if (tid == 0 && p.lse)
      gst<float>(p.lse + row, sum == 0.0f ? -INFINITY : (top + __builtin_amdgcn_logf(sum)) * LN2);
    return;
  }
  // ---- totals: every weight from its score --------------------------------------------------------
  const int32_t w = (int32_t)blockIdx.x - rows;
  const int64_t b = w / blocks;
  const int32_t n = length_of(p, b), start = window_start(p, n), lo = start / keys * keys;
  const int32_t t = (w - (int32_t)b * blocks) * JW * 64 + tid;
  if (t - tid >= n) return;
  const int32_t used = n > lo ? (n - lo + pl.span - 1) / pl.span : 0;
  const bool held = t < n && t >= start && row_of(p, b, t) >= 0;
  const float was = t < n && p.totals_in ? gld<float>(p.totals_in + b * p.ldt + t) : 0.0f;
  float total = 0.0f;
  for (int32_t hb = 0; hb < p.q_heads; hb += JW * 64) {
    __syncthreads();
    if (hb + tid < p.q_heads) {
      const int64_t at = (b * p.q_heads + hb + tid) * pl.splits;
      float top = -INFINITY, sum = 0.0f;
      for (int32_t s = 0; s < used; ++s) {
        const float v = gld<float>(pl.m + at + s), x = gld<float>(pl.l + at + s);
        const float up = fmaxf(top, v);
        sum = sum * share(top, up) + x * share(v, up);
        top = up;
      }
      lse[tid] = top + __builtin_amdgcn_logf(sum);
    }
    __syncthreads();
    const int32_t heads = p.q_heads - hb < JW * 64 ? p.q_heads - hb : JW * 64;
    if (held)
      // (one by one: 64 heads, 22 sequences of 0 to 54 14.3 us, 13.4 so)
      for (int32_t h = 0; h < heads; h += SCORES) {
        float s[SCORES];
#pragma unroll
        for (int u = 0; u < SCORES; ++u) {
          const int32_t hu = h + u < heads ? h + u : heads - 1;
          s[u] = gld<float>(pl.s + (b * p.q_heads + hb + hu) * pl.score_ld + t) - lse[hu];
        }
#pragma unroll
        for (int u = 0; u < SCORES; ++u)
          if (h + u < heads) total += __builtin_amdgcn_exp2f(s[u]);
      }
  }
  if (t < n) gst<float>(p.totals_out + b * p.ldt + t, was + total);
}

// Positions of a sequence that can count, from a tile's first one on.
int64_t range_of(const AttnParams& p) {
  return p.window > 0 && p.window < p.max_len ? p.window + (p.bf16 ? 32 : 16) : p.max_len;
}

// Tiles of 16 query heads per workgroup.  Two read the keys and values once for twice the heads, and have
// the registers for it up to 128 entries a head, but one wavefront per SIMD: for more than 16 heads to a
// key head and 32 MB of cache on (64 heads to one, 64 sequences of 8192: 91 us, 176 with one tile; 16 of
// 4096 24.7 and 31.8; one sequence of 300, 24 heads to one 14.1 and 10.1).
int32_t head_tiles(const AttnParams& p) {
  const double bytes = (double)range_of(p) * (double)(p.n_seqs * p.kv_heads) * (p.d * (p.bf16 ? 4 : 8));
  return p.q_heads / p.kv_heads > 16 && p.d <= 128 && bytes >= 32 << 20 ? 2 : 1;
}

// Spans that give the 256 compute units two workgroups each, as many as have the registers at once (one
// of two head tiles), between a tile per wavefront and a block; `split` false: the whole sequence.  (Four
// each: 13 sequences of 0 to 1533, window 1000, 21 fp32 heads to 7 of 77 26.9 us, 21.3 so; spans of two
// blocks: 64 sequences of 1 to 8192 209 us, 196 with one, one of 131072 105 and 99.)
// Two head tiles leave twice the partial results a span, and the start of a workgroup alone on its compute
// unit is covered by nothing: up to four blocks (64 heads to one, 64 sequences of 8192 135 us with one, 91
// so; 24 to one, 256 of 2000 to 4096 126 and 88; 32 heads of 64 to one, 64 of 1 to 8192 31 and 34).
// Where blocks would make less than two rounds of workgroups, sequences of several lengths leave compute
// units idle: half a block (22 of 0 to 1760, 16 heads to 16 of 64 30.5 us with a block, 26.2 so; 52 of 0 to
// 8745, 8 heads to 2 of 32 27.3 and 27.3; of 96 54.1 and 49.3; but one of 131072 99 and 102).
AttnPlan plan(const AttnParams& p, bool split) {
  AttnPlan pl = {};
  pl.group = p.q_heads / p.kv_heads;
  const int32_t nt = head_tiles(p);
  pl.tiles = (pl.group + 16 * nt - 1) / (16 * nt);
  const int32_t keys = p.bf16 ? 32 : 16, step = AW * keys;
  const int64_t range = range_of(p);
  const int64_t units = p.n_seqs * p.kv_heads * pl.tiles;
  int64_t span = (range * units / (nt == 2 ? 256 : 512) + step - 1) / step * step;
  if (span < step) span = step;
  const int64_t most = nt == 2 ? 4 * BLOCK : p.n_seqs > 1 && range * units < 1024 * BLOCK ? BLOCK / 2 : BLOCK;
  if (span > most) span = most;
  // Few tiles to a sequence: their workgroup is done sooner than a second kernel has joined parts (one
  // sequence of 512, 8 key heads of 128 bf16: 9.8 us whole and 9.4, of 256 6.9 and 9.4; fp32 256 10.4 whole and
  // 10.2; 16 sequences of 1024 bf16 19.0 and 19.5, of 512 fp32 17.6 and 20.3).
  const bool few = range <= keys * (units >= 128 ? 32 : p.bf16 ? 16 : 8);
  if (!split || few) span = range < step ? step : (range + step - 1) / step * step;
  pl.span = (int32_t)span;
  pl.splits = range > span ? (int32_t)((range + span - 1) / span) : 1;
  pl.score_ld = ((p.max_len + 63) / 64 | 1) * 64;
  const int32_t heads = pl.group < 16 * nt ? pl.group : 16 * nt;
  // at most 34 KB of scores, so that as many workgroups have room as have registers
  pl.block = !p.totals_out || heads <= 8 ? BLOCK : heads <= 16 ? BLOCK / 2 : BLOCK / 4;
  if (pl.block > span) pl.block = (int32_t)span;
  pl.stage_ld = pl.block + 16;   // four heads' chunks at once to different banks
  pl.div_seqs = FastDiv(p.n_seqs);
  pl.div_splits = FastDiv(pl.splits);
  pl.div_tiles = FastDiv(pl.tiles);
  // Heads side by side in the cache whose rows are no whole lines: two workgroups read a line, and the bytes
  // past L2 are those of whole lines unless they do so on one XCD.  With fewer workgroups than run at once
  // all of a sequence's on one XCD would leave others idle.  (32 heads to 8, 64 sequences: of 96 bf16, 4096
  // 169 us apart, 150 together; of 77, 1 to 8192 213 and 185; 16 of 3000, of 80, 40.3 and 36.6; 13 of 0 to
  // 1533, fp32 heads of 77 as above, 22.2 and 21.3; but 16 heads to 16 of 77, 22 of 0 to 1760, 51.1 and 51.4.)
  const int64_t lines = p.head_stride % 128 * (p.bf16 ? 2 : 4) % 128, spans = p.n_seqs * pl.splits;
  const int64_t round = 8 * (int64_t)p.kv_heads * pl.tiles;
  if (lines != 0 && p.kv_heads > 1 && p.head_stride < p.pos_stride && units * pl.splits >= 512 &&
      (spans + 7) / 8 <= 0x7fffffff / round) {
    pl.round = (int32_t)round;
    pl.div_round = FastDiv(round);
  }
  return pl;
}

template <bool BF16, int DP, int NT>
void launch_tail(const AttnParams& p, const AttnPlan& pl, dim3 grid, size_t bytes, hipStream_t stream) {
#define TPP_ATTN(TAIL, TOTALS) \
  hipLaunchKernelGGL((attn_kernel<BF16, DP, TAIL, NT, TOTALS>), grid, dim3(AT), bytes, stream, p, pl)
  if (p.d < DP) {
    if (pl.s) TPP_ATTN(true, true);
    else TPP_ATTN(true, false);
  } else {
    if (pl.s) TPP_ATTN(false, true);
    else TPP_ATTN(false, false);
  }
#undef TPP_ATTN
}

template <bool BF16, int NT>
void launch_dim(const AttnParams& p, const AttnPlan& pl, dim3 grid, size_t bytes, hipStream_t stream) {
  if (p.d <= 64) launch_tail<BF16, 64, NT>(p, pl, grid, bytes, stream);
  else if (NT == 1 && p.d <= 96) launch_tail<BF16, 96, 1>(p, pl, grid, bytes, stream);
  else if (NT == 2 || p.d <= 128) launch_tail<BF16, 128, NT>(p, pl, grid, bytes, stream);
  else if (p.d <= 192) launch_tail<BF16, 192, 1>(p, pl, grid, bytes, stream);
  else launch_tail<BF16, 256, 1>(p, pl, grid, bytes, stream);
}

// Workgroups of the attention, and of the join with `threads` each.
int64_t groups(const AttnParams& p, const AttnPlan& pl) {
  return pl.round ? (p.n_seqs * pl.splits + 7) / 8 * pl.round
                  : (int64_t)pl.splits * p.kv_heads * pl.tiles * p.n_seqs;
}
int64_t joins(const AttnParams& p, int threads) {
  return p.n_seqs * p.q_heads + (p.totals_out ? (p.max_len + threads - 1) / threads * p.n_seqs : 0);
}

}  // namespace

int64_t attn_work_floats(const AttnParams& p) {
  // every grid below is in bounds before anything is multiplied further
  const int64_t most = most_groups(AT);
  if (p.n_seqs > most || p.n_seqs * p.q_heads > 0x7fffffff) return -1;
  const AttnPlan pl = plan(p, true);
  const int64_t rows = p.n_seqs * p.q_heads, units = (int64_t)p.kv_heads * pl.tiles * p.n_seqs;
  if (units > most / pl.splits || groups(p, pl) > most) return -1;
  if (pl.splits == 1 && !p.totals_out) return 0;
  if (joins(p, AT) > most) return -1;
  return rows * pl.splits * (p.d + 2) + (p.totals_out ? 64 + rows * pl.score_ld : 0);
}

hipError_t launch_attn(const AttnParams& p, float* work, hipStream_t stream) {
  if (attn_work_floats(p) < 0) return hipErrorInvalidConfiguration;
  AttnPlan pl = plan(p, work != nullptr);
  const int64_t rows = p.n_seqs * p.q_heads;
  // more wavefronts where there are many spans to join
  const int jt = pl.splits > 16 && joins(p, 1024) <= most_groups(1024) ? 1024 : AT;
  if (work) {
    pl.o = work;
    pl.m = pl.o + rows * pl.splits * p.d;
    pl.l = pl.m + rows * pl.splits;
    pl.s = p.totals_out ? work + (rows * pl.splits * (p.d + 2) + 63) / 64 * 64 : nullptr;   // whole lines
  }
  const int32_t nt = head_tiles(p), meet = pl.group < MEET ? pl.group : MEET;
  const int32_t heads = pl.group < 16 * nt ? pl.group : 16 * nt;
  const size_t block = (size_t)pl.block * 8 + (pl.s ? (size_t)heads * pl.stage_ld * 4 : 0);
  const size_t part = (size_t)AW * meet * p.d * 4, bytes = block > part ? block : part;
  const dim3 grid((uint32_t)groups(p, pl));   // (unsplit no more than split)
  if (p.bf16)
    nt == 1 ? launch_dim<true, 1>(p, pl, grid, bytes, stream)
            : launch_dim<true, 2>(p, pl, grid, bytes, stream);
  else
    nt == 1 ? launch_dim<false, 1>(p, pl, grid, bytes, stream)
            : launch_dim<false, 2>(p, pl, grid, bytes, stream);
  if (work) {
    const dim3 jgrid((uint32_t)joins(p, jt));
    const int32_t keys = p.bf16 ? 32 : 16, blocks = (int32_t)((p.max_len + jt - 1) / jt);
#define TPP_JOIN_WAVES(NE, JW)                                                                    \
  hipLaunchKernelGGL((attn_join_kernel<NE, JW>), jgrid, dim3(JW * 64), 0, stream, p, pl, (int32_t)rows, \
                     blocks, keys)
#define TPP_JOIN(NE)                          \
  if (jt == 1024) TPP_JOIN_WAVES(NE, 16);     \
  else TPP_JOIN_WAVES(NE, AW)
    if (p.d <= 64) { TPP_JOIN(1); }
    else if (p.d <= 128) { TPP_JOIN(2); }
    else { TPP_JOIN(4); }
#undef TPP_JOIN_WAVES
#undef TPP_JOIN
  }
  return hipGetLastError();
}

}  // namespace tpp

// cache_kernels.hip -- eviction of cached positions by their total attention weight, for gfx950.
//
// Per sequence: the e candidates of least total leave (ties by position), and what is kept behind the
// new length moves into the free places below it, in order.  The totals become unsigned keys of the
// same order, a radix selection (11 + 11 + 10 bits, one histogram each) finds the key T of the e-th
// smallest candidate, and how many candidates of exactly T leave.  Then the sequence is walked in
// order: each wavefront has a run of positions, counts its ties, its free places and its movers with
// ballots, and three counts per wavefront give every one its place in the lists.
//
// One workgroup of 16 wavefronts per sequence selects.  Up to 32 totals per lane stay in registers, so
// that memory is read once, with every load in flight; longer sequences are read again by each pass.
// The moved rows of keys and values, at most half a sequence, are copied by a second kernel, a 16-byte
// chunk per lane -- or, where a sequence can lose only a few, by the selecting workgroup itself, since a
// second launch would cost more than the copy.
#include <hip/hip_runtime.h>

#include "brgemm_device.h"
#include "internal.h"

namespace tpp {
namespace {

using namespace dev;

constexpr int ST = 1024;          // threads of the selection: 16 wavefronts
constexpr int SW = ST / 64;
constexpr int BINS = 2048;        // of 11 bits
constexpr int CT = 256;           // threads of the copy

// The totals' order as unsigned integers: -0 as +0, NaN above everything.
__device__ __forceinline__ uint32_t order_key(float x) {
  if (x != x) return 0xffffffffu;
  const uint32_t u = __float_as_uint(x + 0.0f);
  return (u >> 31) ? ~u : u | 0x80000000u;
}

__device__ __forceinline__ int32_t lanes_below(uint64_t mask) {
  return __builtin_amdgcn_mbcnt_hi((uint32_t)(mask >> 32),
                                   __builtin_amdgcn_mbcnt_lo((uint32_t)mask, 0u));
}

// Lists of the moves, in the work space: per sequence the number of moves, then their free places and
// their movers (cap of each).
struct MoveLists {
  int32_t* count;
  int32_t* to;
  int32_t* from;
  int64_t cap;
};

// Element offset of position t of sequence b (head 0), or -1 where no page holds it.
__device__ __forceinline__ int64_t row_of(const EvictParams& p, int64_t b, int32_t t) {
  const int32_t j = fdiv((uint32_t)t, p.page);
  const int64_t page = gld<int64_t>(p.pages + b * p.ld_pages + j);
  if (page < 0 || page >= p.n_pages) return -1;
  return page * p.page_stride + (int64_t)(t - j * p.page_size) * p.pos_stride;
}

// Copies the moved rows of sequence b: threads `at`, at + step, ... of a set that covers them.  A thread
// takes a 16-byte chunk of a head's row, of the keys and of the values; a row that is no multiple of 16
// bytes ends with the chunk that ends with it, a shorter one goes by 2-byte units.
struct CopyShape {
  FastDiv chunks, heads;   // chunks of a row; kv_heads
  int32_t n_chunks;
};
template <int U>
__device__ __forceinline__ void copy_moves(const EvictParams& p, const CopyShape& cs, int64_t b,
                                           const int32_t* to, const int32_t* from, int32_t moves,
                                           int32_t at, int32_t step) {
  const int32_t bytes = p.d * p.es, per_move = p.kv_heads * cs.n_chunks;
  const int64_t all = (int64_t)moves * per_move;
  char* kb = static_cast<char*>(p.k);
  char* vb = static_cast<char*>(p.v);
  for (int64_t i0 = at; i0 < all; i0 += (int64_t)step * U) {
    u32x4 k[U], v[U];
    int64_t dst[U];
#pragma unroll
    for (int u = 0; u < U; ++u) {
      const int64_t i = i0 + (int64_t)u * step;
      dst[u] = -1;
      if (i >= all) continue;
      // below 2^31 by the launcher
      const int32_t r = fdiv((uint32_t)i, cs.chunks), c = (int32_t)i - r * cs.n_chunks;
      const int32_t j = fdiv((uint32_t)r, cs.heads), h = r - j * p.kv_heads;
      const int64_t d = row_of(p, b, to[j]), s = row_of(p, b, from[j]);
      if (d < 0 || s < 0) continue;
      if (bytes < 16) {
#pragma unroll 1
        for (int32_t e = 0; e < bytes; e += 2) {
          const int64_t x = (s + h * p.head_stride) * p.es + e, y = (d + h * p.head_stride) * p.es + e;
          gst<uint16_t>(kb + y, gld<uint16_t>(kb + x));
          gst<uint16_t>(vb + y, gld<uint16_t>(vb + x));
        }
        continue;
      }
      const int32_t e = c * 16 + 16 <= bytes ? c * 16 : bytes - 16;
      const int64_t x = (s + h * p.head_stride) * p.es + e;
      dst[u] = (d + h * p.head_stride) * p.es + e;
      k[u] = gld<u32x4_a2>(kb + x);
      v[u] = gld<u32x4_a2>(vb + x);
    }
#pragma unroll
    for (int u = 0; u < U; ++u)
      if (dst[u] >= 0) {
        gst<u32x4_a2>(kb + dst[u], k[u]);
        gst<u32x4_a2>(vb + dst[u], v[u]);
      }
  }
}

// KPT: totals that a lane keeps (0: none, read again).  FUSED: this workgroup copies the rows too.
template <int KPT, bool FUSED>
__global__ __launch_bounds__(ST) void evict_select_kernel(EvictParams p, MoveLists ml, CopyShape cs) {
  __shared__ int32_t hist[BINS];
  __shared__ int32_t wsum[3][SW];
  __shared__ int32_t pick[2];     // digit, candidates below it
  const int tid = threadIdx.x, lane = tid & 63, wave = tid >> 6;
  const int64_t b = blockIdx.x;
  const int64_t len = gld<int64_t>(p.len + b);
  const int32_t n = (int32_t)(len < 0 ? 0 : len > p.max_len ? p.max_len : len);
  const int32_t want = n > p.budget ? (int32_t)(n - p.budget) : 0;
  const float* tot = p.totals + b * p.ldt;
  const int64_t* pos = p.pos ? p.pos + b * p.ldt : nullptr;
  const int64_t horizon = p.pos ? gld<int64_t>(p.horizon + b) : 0;
  float* tot_out = p.totals_out + b * p.ldt;
  int64_t* pos_out = p.pos ? p.pos_out + b * p.ldt : nullptr;
  const bool hand_on = p.totals_out != p.totals, hand_pos = pos && p.pos_out != p.pos;

  // ---- each wavefront's run of positions, whole sets of 64 ---------------------------------------
  const int32_t run = (((n + SW - 1) / SW) + 63) / 64 * 64;
  const int32_t t0 = wave * run < n ? wave * run : n;
  const int32_t t1 = t0 + run < n ? t0 + run : n;
  float w[KPT > 0 ? KPT : 1];
  uint32_t may = 0;               // bit i: the i-th total is a candidate's
  const auto may_go = [&](int32_t t) { return !pos || gld<int64_t>(pos + t) < horizon; };
  if constexpr (KPT > 0) {
#pragma unroll
    for (int i = 0; i < KPT; ++i) {
      const int32_t t = t0 + i * 64 + lane;
      w[i] = t < t1 ? gld<float>(tot + t) : 0.0f;
    }
    if (want > 0)
#pragma unroll
      for (int i = 0; i < KPT; ++i) {
        const int32_t t = t0 + i * 64 + lane;
        if (t < t1 && may_go(t)) may |= 1u << i;
      }
  }
  // f(t, in the run, key, candidate, total) for the run's sets in order, with all lanes
  const auto each = [&](auto&& f) {
    if constexpr (KPT > 0) {
#pragma unroll
      for (int i = 0; i < KPT; ++i) {
        const int32_t t = t0 + i * 64 + lane;
        if (t0 + i * 64 < t1) f(t, t < t1, order_key(w[i]), (may >> i & 1) != 0, w[i]);
      }
    } else {
      for (int32_t t = t0 + lane; t - lane < t1; t += 64) {
        const bool in = t < t1;
        const float x = in ? gld<float>(tot + t) : 0.0f;
        f(t, in, order_key(x), in && may_go(t), x);
      }
    }
  };

  // ---- the key of the last one to leave ----------------------------------------------------------
  uint32_t prefix = 0;            // the digits found so far
  int32_t rank = 0, gone_n = 0;   // ordinal (from 0) among the candidates with that prefix
  if (want > 0) {
    for (int pass = 0; pass < 3; ++pass) {
      const int shift = pass == 0 ? 21 : pass == 1 ? 10 : 0;
      const uint32_t mask = pass == 2 ? 1023u : 2047u;
      // the bits above the digit, which have to be those found
      const uint32_t found = pass == 0 ? 0u : pass == 1 ? 0xffe00000u : 0xfffffc00u;
      for (int i = tid; i < BINS; i += ST) hist[i] = 0;
      __syncthreads();
      each([&](int32_t, bool, uint32_t key, bool cand, float) {
        if (cand && (key & found) == prefix) atomicAdd(&hist[(key >> shift) & mask], 1);
      });
      __syncthreads();
      // running sums of the histogram: two bins per thread
      const int32_t h0 = hist[2 * tid], h1 = hist[2 * tid + 1];
      int32_t up = h0 + h1;
#pragma unroll
      for (int d = 1; d < 64; d *= 2) {
        const int32_t v = __shfl_up(up, d, 64);
        if (lane >= d) up += v;
      }
      if (lane == 63) wsum[0][wave] = up;
      __syncthreads();
      int32_t before = 0, all = 0;
#pragma unroll
      for (int x = 0; x < SW; ++x) {
        const int32_t v = wsum[0][x];
        before += x < wave ? v : 0;
        all += v;
      }
      if (pass == 0) {
        gone_n = all < want ? all : want;
        rank = gone_n - 1;
      }
      const int32_t lo = before + up - h0 - h1;   // candidates below this thread's bins
      if (gone_n > 0) {
        if (rank >= lo && rank < lo + h0) {
          pick[0] = 2 * tid;
          pick[1] = lo;
        } else if (rank >= lo + h0 && rank < lo + h0 + h1) {
          pick[0] = 2 * tid + 1;
          pick[1] = lo + h0;
        }
      }
      __syncthreads();
      if (gone_n == 0) break;
      prefix |= (uint32_t)pick[0] << shift;
      rank -= pick[1];
    }
  }
  const int32_t left = n - gone_n;
  // candidates below `prefix` leave, and of those equal to it the first rank + 1

  int32_t ties = 0;
  if (gone_n > 0)
    each([&](int32_t, bool, uint32_t key, bool cand, float) {
      ties += __popcll(__ballot(cand && key == prefix));
    });
  if (lane == 0) wsum[0][wave] = ties;
  __syncthreads();
  int32_t ties_before = 0;
  for (int x = 0; x < wave; ++x) ties_before += wsum[0][x];
  // f(t, in the run, free place, mover, total)
  const auto walk = [&](auto&& f) {
    int32_t seen = ties_before;
    each([&](int32_t t, bool in, uint32_t key, bool cand, float x) {
      const uint64_t tie = __ballot(cand && key == prefix);
      const bool goes = cand && (key < prefix || (key == prefix && seen + lanes_below(tie) <= rank));
      seen += __popcll(tie);
      f(t, in, goes && t < left, in && !goes && t >= left, x);
    });
  };
  int32_t places = 0, movers = 0;
  if (gone_n > 0)
    walk([&](int32_t, bool, bool place, bool mover, float) {
      places += __popcll(__ballot(place));
      movers += __popcll(__ballot(mover));
    });
  if (lane == 0) {
    wsum[1][wave] = places;
    wsum[2][wave] = movers;
  }
  __syncthreads();
  int32_t place_at = 0, mover_at = 0, moves = 0;
  for (int x = 0; x < SW; ++x) {
    if (x < wave) {
      place_at += wsum[1][x];
      mover_at += wsum[2][x];
    }
    moves += wsum[1][x];
  }
  int32_t* to = ml.to + b * ml.cap;
  int32_t* from = ml.from + b * ml.cap;
  // the lists, and the totals and positions of what stays where it is
  const auto stay = [&](int32_t t, float x) {
    if (hand_on) gst<float>(tot_out + t, x);
    if (hand_pos) gst<int64_t>(pos_out + t, gld<int64_t>(pos + t));
  };
  if (gone_n > 0)
    walk([&](int32_t t, bool in, bool place, bool mover, float x) {
      const uint64_t pm = __ballot(place), mm = __ballot(mover);
      if (place) gst<int32_t>(to + place_at + lanes_below(pm), t);
      else if (in && t < left) stay(t, x);
      if (mover) gst<int32_t>(from + mover_at + lanes_below(mm), t);
      place_at += __popcll(pm);
      mover_at += __popcll(mm);
    });
  else if (hand_on || hand_pos)
    each([&](int32_t t, bool in, uint32_t, bool, float x) {
      if (in) stay(t, x);
    });
  __threadfence_block();
  __syncthreads();
  for (int32_t j = tid; j < moves; j += ST) {
    const int32_t d = to[j], s = from[j];
    gst<float>(tot_out + d, gld<float>(tot + s));
    if (pos) gst<int64_t>(pos_out + d, gld<int64_t>(pos + s));
  }
  if (tid == 0) {
    ml.count[b] = moves;
    gst<int64_t>(p.len_out + b, left);
  }
  if constexpr (FUSED) copy_moves<1>(p, cs, b, to, from, moves, tid, ST);
}

// The moved rows of sequence blockIdx.x.
__global__ __launch_bounds__(CT) void evict_copy_kernel(EvictParams p, MoveLists ml, CopyShape cs) {
  const int64_t b = blockIdx.x;
  copy_moves<2>(p, cs, b, ml.to + b * ml.cap, ml.from + b * ml.cap, ml.count[b],
                blockIdx.y * CT + threadIdx.x, gridDim.y * CT);
}

// Most moves of a sequence: no more than leave, and no more than stay below the new length.
int64_t move_cap(const EvictParams& p) {
  const int64_t gone = p.max_len > p.budget ? p.max_len - p.budget : 0;
  return gone < p.max_len / 2 ? gone : p.max_len / 2;
}

}  // namespace

int64_t evict_work_floats(const EvictParams& p) { return p.n_seqs * (2 * move_cap(p) + 1); }

hipError_t launch_evict(const EvictParams& p, float* work, hipStream_t stream) {
  MoveLists ml;
  ml.cap = move_cap(p);
  ml.count = reinterpret_cast<int32_t*>(work);
  ml.to = ml.count + p.n_seqs;
  ml.from = ml.to + p.n_seqs * ml.cap;
  CopyShape cs;
  const int64_t bytes = (int64_t)p.d * p.es;
  cs.n_chunks = (int32_t)((bytes + 15) / 16);
  cs.chunks = FastDiv(cs.n_chunks);
  cs.heads = FastDiv(p.kv_heads);
  const int64_t chunks = ml.cap * p.kv_heads * cs.n_chunks;   // of a sequence's moves
  if (p.n_seqs > 0x7fffffff || chunks > 0x7fffffff) return hipErrorInvalidConfiguration;
  // A chunk or two per thread of the selecting workgroup: no second launch (32 sequences that lose one
  // position: 12 us so, 17 with the copy of its own).
  const bool fused = chunks <= 2 * ST;
  const dim3 grid((uint32_t)p.n_seqs);
#define TPP_SELECT(KPT, FUSED)                                                                    \
  hipLaunchKernelGGL((evict_select_kernel<KPT, FUSED>), grid, dim3(ST), 0, stream, p, ml, cs)
#define TPP_SELECT_KPT(FUSED)                                 \
  if (p.max_len <= 4 * ST) TPP_SELECT(4, FUSED);              \
  else if (p.max_len <= 16 * ST) TPP_SELECT(16, FUSED);       \
  else if (p.max_len <= 32 * ST) TPP_SELECT(32, FUSED);       \
  else TPP_SELECT(0, FUSED)
  if (fused) {
    TPP_SELECT_KPT(true);
  } else {
    TPP_SELECT_KPT(false);
    const int64_t want = (chunks + 2 * CT - 1) / (2 * CT);   // two chunks per thread, at most 2048 groups
    const int64_t most = 2048 / p.n_seqs > 0 ? 2048 / p.n_seqs : 1;
    hipLaunchKernelGGL(evict_copy_kernel, dim3((uint32_t)p.n_seqs, (uint32_t)(want < most ? want : most)),
                       dim3(CT), 0, stream, p, ml, cs);
  }
#undef TPP_SELECT_KPT
#undef TPP_SELECT
  return hipGetLastError();
}

}  // namespace tpp

// cache_kernels.hip -- eviction of cached positions by their total attention weight, for gfx950.
//
// Per sequence: the e candidates of least total leave (ties by position), and what is kept behind the
// new length moves into the free places below it, in order.  The totals become unsigned keys of the
// same order, a radix selection (11 + 11 + 10 bits, one histogram each) finds the key T of the e-th
// smallest candidate, and how many candidates of exactly T leave.  Then the sequence is walked in
// order: each wavefront has a run of positions, counts its ties, its free places and its movers with
// ballots, and three counts per wavefront give every one its place in the lists.
//
// One workgroup of 16 wavefronts per sequence selects; a second kernel copies the moved rows of keys
// and values, a 16-byte chunk per lane.
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

__global__ __launch_bounds__(ST) void evict_select_kernel(EvictParams p, MoveLists ml) {
  __shared__ int32_t hist[BINS];
  __shared__ int32_t wsum[3][SW];
  __shared__ int32_t pick[3];     // digit, candidates below it; candidates in all
  const int tid = threadIdx.x, lane = tid & 63, wave = tid >> 6;
  const int64_t b = blockIdx.x;
  const int64_t len = gld<int64_t>(p.len + b);
  const int32_t n = (int32_t)(len < 0 ? 0 : len > p.max_len ? p.max_len : len);
  const int32_t want = n > p.budget ? (int32_t)(n - p.budget) : 0;
  const float* tot = p.totals + b * p.ldt;
  const int64_t* pos = p.pos ? p.pos + b * p.ldt : nullptr;
  const int64_t horizon = p.pos ? gld<int64_t>(p.horizon + b) : 0;
  const auto may_go = [&](int32_t t) { return !pos || gld<int64_t>(pos + t) < horizon; };

  // ---- the key of the last one to leave -------------------------------------------------------
  uint32_t prefix = 0;      // the digits found so far
  int32_t rank = 0, gone_n = 0;   // ordinal (from 0) among the candidates with that prefix
  if (want > 0) {
    for (int pass = 0; pass < 3; ++pass) {
      const int shift = pass == 0 ? 21 : pass == 1 ? 10 : 0;
      const int above = pass == 0 ? 32 : pass == 1 ? 21 : 10;   // bits above the digit start here
      const uint32_t mask = pass == 2 ? 1023u : 2047u;
      for (int i = tid; i < BINS; i += ST) hist[i] = 0;
      __syncthreads();
      for (int32_t t = tid; t < n; t += ST) {
        const uint32_t key = order_key(gld<float>(tot + t));
        const bool in = above == 32 || (key >> above) == (prefix >> above);
        if (in && may_go(t)) atomicAdd(&hist[(key >> shift) & mask], 1);
      }
      __syncthreads();
      // running sums of the histogram: two bins per thread
      const int32_t h0 = hist[2 * tid], h1 = hist[2 * tid + 1];
      int32_t run = h0 + h1;
#pragma unroll
      for (int d = 1; d < 64; d *= 2) {
        const int32_t up = __shfl_up(run, d, 64);
        if (lane >= d) run += up;
      }
      if (lane == 63) wsum[0][wave] = run;
      __syncthreads();
      int32_t before = 0, all = 0;
#pragma unroll
      for (int w = 0; w < SW; ++w) {
        const int32_t v = wsum[0][w];
        before += w < wave ? v : 0;
        all += v;
      }
      if (pass == 0) {
        gone_n = all < want ? all : want;
        rank = gone_n - 1;
      }
      const int32_t lo = before + run - h0 - h1;   // candidates below this thread's bins
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

  // ---- each wavefront's run of positions ------------------------------------------------------
  const int32_t runlen = (((n + SW - 1) / SW) + 63) / 64 * 64;
  const int32_t t0 = wave * runlen < n ? wave * runlen : n;
  const int32_t t1 = t0 + runlen < n ? t0 + runlen : n;
  int32_t ties = 0;
  if (gone_n > 0)
    for (int32_t t = t0 + lane; t - lane < t1; t += 64) {
      const bool tie = t < t1 && order_key(gld<float>(tot + t)) == prefix && may_go(t);
      ties += __popcll(__ballot(tie));
    }
  if (lane == 0) wsum[0][wave] = ties;
  __syncthreads();
  int32_t ties_before = 0;
  for (int w = 0; w < wave; ++w) ties_before += wsum[0][w];
  // walks the run; f(t, free place, mover) with all lanes
  const auto walk = [&](auto&& f) {
    int32_t seen = ties_before;
    for (int32_t t = t0 + lane; t - lane < t1; t += 64) {
      const bool in = t < t1;
      const uint32_t key = in ? order_key(gld<float>(tot + t)) : 0u;
      const bool cand = in && may_go(t);
      const uint64_t tie = __ballot(cand && key == prefix);
      const bool goes = cand && (key < prefix || (key == prefix && seen + lanes_below(tie) <= rank));
      seen += __popcll(tie);
      f(t, goes && t < left, in && !goes && t >= left);
    }
  };
  int32_t places = 0, movers = 0;
  if (gone_n > 0)
    walk([&](int32_t, bool place, bool mover) {
      places += __popcll(__ballot(place));
      movers += __popcll(__ballot(mover));
    });
  if (lane == 0) {
    wsum[1][wave] = places;
    wsum[2][wave] = movers;
  }
  __syncthreads();
  int32_t place_at = 0, mover_at = 0, moves = 0;
  for (int w = 0; w < SW; ++w) {
    if (w < wave) {
      place_at += wsum[1][w];
      mover_at += wsum[2][w];
    }
    moves += wsum[1][w];
  }
  int32_t* to = ml.to + b * ml.cap;
  int32_t* from = ml.from + b * ml.cap;
  if (gone_n > 0)
    walk([&](int32_t t, bool place, bool mover) {
      const uint64_t pm = __ballot(place), mm = __ballot(mover);
      if (place) gst<int32_t>(to + place_at + lanes_below(pm), t);
      if (mover) gst<int32_t>(from + mover_at + lanes_below(mm), t);
      place_at += __popcll(pm);
      mover_at += __popcll(mm);
    });
  __threadfence_block();
  __syncthreads();

  // ---- totals and positions ---------------------------------------------------------------------
  float* tot_out = p.totals_out + b * p.ldt;
  int64_t* pos_out = p.pos ? p.pos_out + b * p.ldt : nullptr;
  if (p.totals_out != p.totals)
    for (int32_t t = tid; t < left; t += ST) gst<float>(tot_out + t, gld<float>(tot + t));
  if (pos && p.pos_out != p.pos)
    for (int32_t t = tid; t < left; t += ST) gst<int64_t>(pos_out + t, gld<int64_t>(pos + t));
  __syncthreads();   // the free places' new values come after what was there
  for (int32_t j = tid; j < moves; j += ST) {
    const int32_t d = to[j], s = from[j];
    gst<float>(tot_out + d, gld<float>(tot + s));
    if (pos) gst<int64_t>(pos_out + d, gld<int64_t>(pos + s));
  }
  if (tid == 0) {
    ml.count[b] = moves;
    gst<int64_t>(p.len_out + b, left);
  }
}

// Element offset of position t of sequence b (head 0), or -1 where no page holds it.
__device__ __forceinline__ int64_t row_of(const EvictParams& p, int64_t b, int32_t t) {
  const int32_t j = fdiv((uint32_t)t, p.page);
  const int64_t page = gld<int64_t>(p.pages + b * p.ld_pages + j);
  if (page < 0 || page >= p.n_pages) return -1;
  return page * p.page_stride + (int64_t)(t - j * p.page_size) * p.pos_stride;
}

// The moved rows: a wavefront per (move, head), keys and values.
__global__ __launch_bounds__(CT) void evict_copy_kernel(EvictParams p, MoveLists ml, FastDiv heads) {
  const int lane = threadIdx.x & 63;
  const int64_t b = blockIdx.x;
  const int32_t moves = ml.count[b];
  const int32_t bytes = p.d * p.es;
  for (int64_t i = (int64_t)blockIdx.y * (CT / 64) + (threadIdx.x >> 6); i < (int64_t)moves * p.kv_heads;
       i += (int64_t)gridDim.y * (CT / 64)) {
    const int32_t j = (int32_t)(i / p.kv_heads), h = (int32_t)(i - (int64_t)j * p.kv_heads);
    const int64_t d = row_of(p, b, ml.to[b * ml.cap + j]), s = row_of(p, b, ml.from[b * ml.cap + j]);
    if (d < 0 || s < 0) continue;
    const int64_t db = (d + h * p.head_stride) * p.es, sb = (s + h * p.head_stride) * p.es;
    for (int32_t e = 2 * lane; e < bytes; e += 128) {
      gst<uint16_t>(static_cast<char*>(p.k) + db + e, gld<uint16_t>(static_cast<char*>(p.k) + sb + e));
      gst<uint16_t>(static_cast<char*>(p.v) + db + e, gld<uint16_t>(static_cast<char*>(p.v) + sb + e));
    }
  }
}

int64_t move_cap(const EvictParams& p) { return p.max_len > p.budget ? p.max_len - p.budget : 0; }

}  // namespace

int64_t evict_work_floats(const EvictParams& p) { return p.n_seqs * (2 * move_cap(p) + 1); }

hipError_t launch_evict(const EvictParams& p, float* work, hipStream_t stream) {
  if (p.n_seqs > 0x7fffffff) return hipErrorInvalidConfiguration;
  MoveLists ml;
  ml.cap = move_cap(p);
  ml.count = reinterpret_cast<int32_t*>(work);
  ml.to = ml.count + p.n_seqs;
  ml.from = ml.to + p.n_seqs * ml.cap;
  hipLaunchKernelGGL(evict_select_kernel, dim3((uint32_t)p.n_seqs), dim3(ST), 0, stream, p, ml);
  if (ml.cap > 0) {
    const int64_t want = (ml.cap * p.kv_heads + 15) / 16;   // four rows per wavefront
    hipLaunchKernelGGL(evict_copy_kernel, dim3((uint32_t)p.n_seqs, (uint32_t)(want < 1024 ? want : 1024)),
                       dim3(CT), 0, stream, p, ml, FastDiv(p.kv_heads));
  }
  return hipGetLastError();
}

}  // namespace tpp

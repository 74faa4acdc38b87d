// cache_kernels.hip -- eviction of cached positions by their total attention weight, for gfx950.
//
// Per sequence: the e candidates of least total leave (ties by position), and what is kept behind the
// new length moves into the free places below it, in order.  The totals become unsigned keys of the
// same order, a radix selection (11 + 11 + 10 bits, one histogram each) finds the key T of the e-th
// smallest candidate, and how many candidates of exactly T leave.  Each thread has a run of consecutive
// positions, and running sums over the threads of its ties, free places and movers give every one its
// place in the lists.  (Ballots over sets of 64 positions, a wavefront's run at a time, are scalar work,
// and the compute unit has one scalar unit for its 16 wavefronts: 27 us for 16384 positions, 20.4 so.)
//
// One workgroup of 16 wavefronts per sequence selects.  Up to 32 keys per thread stay in registers, so that
// memory is read once, with every load in flight; longer sequences are read again by each pass.
// The moved rows of keys and values, at most half a sequence, are copied by a second kernel, a 16-byte
// chunk per lane -- or, where a sequence can lose only a few, by the selecting workgroup itself, since a
// second launch would cost more than the copy.
//
// 8 key heads of 128 bf16: 8 sequences of 9001 to 16384 cut to 4096 55 us, of them 19 the selection, whose
// passes wait for each other on 8 of 256 compute units, and 36 the copy, 5.2 TB/s; 32 of 2049 that lose one
// 7.5 us.
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
constexpr int FEW = 4;            // positions that leave one by one rather than by selection
constexpr int FUSED_CHUNKS = 2 * ST;   // most chunks of a pool that the selecting workgroup copies

// The totals' order as unsigned integers: -0 as +0, NaN above everything.
__device__ __forceinline__ uint32_t order_key(float x) {
  if (x != x) return 0xffffffffu;
  const uint32_t u = __float_as_uint(x + 0.0f);
  return (u >> 31) ? ~u : u | 0x80000000u;
}

// What the selection leaves in the work space for the copy: per sequence a bit for each position, set
// in the free places (words of 16; null where nothing is handed on), the number of moves, and their free
// places and movers (cap of each).
struct MoveLists {
  uint16_t* gone;
  int32_t* count;
  int32_t* to;
  int32_t* from;
  int64_t cap, words;
};

// Element offset of position t of sequence b (head 0), or -1 where no page holds it.
__device__ __forceinline__ int64_t row_of(const EvictParams& p, int64_t b, int32_t t) {
  const int32_t j = fdiv((uint32_t)t, p.page);
  const int64_t page = gld<int64_t>(p.pages + b * p.ld_pages + j);
  if (page < 0 || page >= p.n_pages) return -1;
  return page * p.page_stride + (int64_t)(t - j * p.page_size) * p.pos_stride;
}

// How the moved rows are copied: `lanes` (a power of two up to 64) consecutive lanes take a row of one
// head, a 16-byte chunk each (of more than 64 chunks, every 64th), of the keys and of the values.  A row
// that is no multiple of 16 bytes ends with the chunk that ends with it.  Rows below 16 bytes (unit 2) go
// by 2 bytes to a lane.
struct CopyShape {
  FastDiv heads;              // kv_heads
  int32_t lanes, unit, units; // bytes of a chunk; chunks of a row
};

// STREAM: stored past the caches' replacement (a copy of its own is of many rows: 8 x 16384 cut to 4096 64.0
// us without, 55.6 so).
template <typename T, bool STREAM>
__device__ __forceinline__ void copy_rows(const EvictParams& p, const CopyShape& cs, int64_t b,
                                          const int32_t* to, const int32_t* from, int32_t rows,
                                          int32_t row, int32_t step, int32_t lane) {
  const int32_t bytes = p.d * p.es;
  char* kb = static_cast<char*>(p.k);
  char* vb = static_cast<char*>(p.v);
  for (; row < rows; row += step) {   // rows below 2^30 by the launcher
    const int32_t j = fdiv((uint32_t)row, cs.heads), h = row - j * p.kv_heads;
    const int64_t d = row_of(p, b, to[j]), s = row_of(p, b, from[j]);
    const int64_t dst = d < 0 || s < 0 ? -1 : (d + h * p.head_stride) * p.es;
    const int64_t src = (s + h * p.head_stride) * p.es;
    for (int32_t c = lane; c < cs.units; c += cs.lanes) {
      const int32_t e = (c + 1) * cs.unit <= bytes ? c * cs.unit : bytes - cs.unit;
      T k, v;
      if (dst >= 0) {
        k = gld<T>(kb + src + e);
        v = gld<T>(vb + src + e);
        if constexpr (STREAM) {
          __builtin_nontemporal_store(k, (GLOBAL_AS T*)(kb + dst + e));
          __builtin_nontemporal_store(v, (GLOBAL_AS T*)(vb + dst + e));
        } else {
          gst<T>(kb + dst + e, k);
          gst<T>(vb + dst + e, v);
        }
      }
    }
  }
}
// Wavefront `wave` of `waves` that copy the moves of sequence b.
template <bool STREAM>
__device__ __forceinline__ void copy_moves(const EvictParams& p, const CopyShape& cs, int64_t b,
                                           const int32_t* to, const int32_t* from, int32_t moves,
                                           int32_t wave, int32_t waves) {
  const int32_t lane = threadIdx.x & 63, slots = 64 / cs.lanes;
  const int32_t row = wave * slots + lane / cs.lanes, step = waves * slots;
  if (cs.unit == 16)
    copy_rows<u32x4_a2, STREAM>(p, cs, b, to, from, moves * p.kv_heads, row, step, lane % cs.lanes);
  else
    copy_rows<uint16_t, STREAM>(p, cs, b, to, from, moves * p.kv_heads, row, step, lane % cs.lanes);
}

template <int CTRL, int ROWS>
__device__ __forceinline__ uint32_t dpp_or_0(uint32_t v) {
  return (uint32_t)__builtin_amdgcn_update_dpp(0, (int)v, CTRL, ROWS, 0xf, true);
}
// The least of a wavefront's values, in every lane.
__device__ __forceinline__ uint32_t wave_min(uint32_t v) {
  const auto dpp = [](uint32_t x, auto ctrl) {
    return (uint32_t)__builtin_amdgcn_update_dpp((int)x, (int)x, decltype(ctrl)::value, 0xf, 0xf, false);
  };
  v = min(v, dpp(v, IntC<0xB1>()));    // lane ^ 1, lane ^ 2, the other quad of 8, the other 8 of 16
  v = min(v, dpp(v, IntC<0x4E>()));
  v = min(v, dpp(v, IntC<0x141>()));
  v = min(v, dpp(v, IntC<0x140>()));
  auto w = __builtin_amdgcn_permlane16_swap(v, v, false, false);
  v = min(w[0], w[1]);
  w = __builtin_amdgcn_permlane32_swap(v, v, false, false);
  return min(w[0], w[1]);
}
// Running sums over the workgroup: what the threads before this one have of v, and in `all` the total.
// Within a wavefront by register permutes (row shifts, then the rows' last lanes handed on).  The barriers
// also order what was in LDS before the call.
__device__ __forceinline__ uint32_t before_me(uint32_t v, uint32_t (&sums)[SW], uint32_t& all) {
  const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
  uint32_t up = v;
  up += dpp_or_0<0x111, 0xf>(up);   // from 1, 2, 4 and 8 lanes down
  up += dpp_or_0<0x112, 0xf>(up);
  up += dpp_or_0<0x114, 0xf>(up);
  up += dpp_or_0<0x118, 0xf>(up);
  up += dpp_or_0<0x142, 0xa>(up);   // the row before, then the half before
  up += dpp_or_0<0x143, 0xc>(up);
  __syncthreads();
  if (lane == 63) sums[wave] = up;
  __syncthreads();
  uint32_t before = up - v;
  all = 0;
#pragma unroll
  for (int w = 0; w < SW; ++w) {
    before += w < wave ? sums[w] : 0u;
    all += sums[w];
  }
  return before;
}

// KPT: consecutive positions of a thread; a sequence is taken in parts of KPT * ST positions.  One part's
// keys stay in registers; of several, each pass reads the totals again.  FUSED: this workgroup hands on
// the totals and copies the rows too, and the lists stay in LDS.
template <int KPT, bool FUSED>
__global__ __launch_bounds__(ST) void evict_select_kernel(EvictParams p, MoveLists ml, CopyShape cs) {
  constexpr int32_t PART = KPT * ST;
  __shared__ int32_t hist[BINS];
  __shared__ uint32_t sums[SW];
  __shared__ uint32_t turned[KPT == 4 ? 1 : PART + PART / 32];
  __shared__ int32_t pick[3];     // digit, candidates below it, candidates of it
  __shared__ uint32_t best[2][SW];
  __shared__ int32_t best_t[2][SW];
  __shared__ int32_t lists[FUSED ? 2 * FUSED_CHUNKS : 1];
  const int tid = threadIdx.x;
  const int64_t b = blockIdx.x;
  const int64_t len = gld<int64_t>(p.len + b);
  const int64_t horizon = p.pos ? gld<int64_t>(p.horizon + b) : 0;
  const int32_t n =
      __builtin_amdgcn_readfirstlane((int32_t)(len < 0 ? 0 : len > p.max_len ? p.max_len : len));
  const int32_t want = n > p.budget ? (int32_t)(n - p.budget) : 0;
  const float* tot = p.totals + b * p.ldt;
  const int64_t* pos = p.pos ? p.pos + b * p.ldt : nullptr;
  float* tot_out = p.totals_out + b * p.ldt;
  int64_t* pos_out = p.pos ? p.pos_out + b * p.ldt : nullptr;

  // Keys of this thread's positions of the part from `part` on; 0, which is no total's key, for a position
  // that is no candidate.  Read in order, 16 loads in flight before the first is waited for (past the end
  // the last position), and turned in LDS, a word in 33 left out against bank conflicts: a thread that read
  // its own run would touch a cache line for every 16 bytes.
  // (Four positions of a thread are 16 consecutive bytes: read where they belong, before the length is known.)
  uint32_t keys[KPT];
  f32x4 x4 = {0.0f, 0.0f, 0.0f, 0.0f};
  int64_t y4[4] = {0, 0, 0, 0};
  if constexpr (KPT == 4) {
    const int32_t t = tid * 4;
    if (t + 4 <= p.max_len) {
      x4 = gld<f32x4_a4>(tot + t);
      if (pos)
#pragma unroll
        for (int i = 0; i < 4; ++i) y4[i] = gld<int64_t>(pos + t + i);
    } else {
#pragma unroll
      for (int i = 0; i < 4; ++i)
        if (t + i < p.max_len) {
          x4[i] = gld<float>(tot + t + i);
          if (pos) y4[i] = gld<int64_t>(pos + t + i);
        }
    }
  }
  const auto load_keys = [&](int32_t part) {
    if constexpr (KPT == 4) {   // one part
#pragma unroll
      for (int i = 0; i < 4; ++i)
        keys[i] = tid * 4 + i < n && (!pos || y4[i] < horizon) ? order_key(x4[i]) : 0u;
      return;
    }
    constexpr int P = KPT < 16 ? KPT : 16;   // in flight
    __syncthreads();   // the part before is done with
#pragma unroll
    for (int i0 = 0; i0 < KPT; i0 += P) {
      float x[P];
      int64_t y[P];
#pragma unroll
      for (int i = 0; i < P; ++i) {
        const int32_t t = part + (i0 + i) * ST + tid, u = t < n ? t : n - 1;
        x[i] = gld<float>(tot + u);
        y[i] = pos ? gld<int64_t>(pos + u) : INT64_MIN;
      }
#pragma unroll
      for (int i = 0; i < P; ++i) {
        const int32_t at = (i0 + i) * ST + tid;
        turned[at + at / 32] = part + at < n && (!pos || y[i] < horizon) ? order_key(x[i]) : 0u;
      }
    }
    __syncthreads();
#pragma unroll
    for (int i = 0; i < KPT; ++i) keys[i] = turned[tid * KPT + i + (tid * KPT + i) / 32];
  };
  const bool several = n > PART;
  if (want > 0 && !several) load_keys(0);

  // ---- the key of the last one to leave ----------------------------------------------------------
  uint32_t prefix = 0;            // the digits found so far
  int32_t rank = 0, gone_n = 0;   // ordinal (from 0) among the candidates with that prefix
  bool all_ties = false;          // whether all candidates of that key leave
  int32_t cut = -1;               // or those of them up to this position
  if (want > 0 && want <= FEW && !several) {
    // A few leave: the least candidate behind the last one, by (key, position), as many times.  A wavefront's
    // is the first lane of its least key; the wavefronts meet in LDS.
    uint32_t last = 0;       // key and position of the last one
    int32_t last_t = -1;
    for (; gone_n < want; ++gone_n) {
      uint32_t key = ~0u;
      int32_t at = n;
#pragma unroll
      for (int i = KPT - 1; i >= 0; --i) {
        const int32_t t = tid * KPT + i;
        const bool after = keys[i] > last || (keys[i] == last && t > last_t);
        if (keys[i] != 0 && after && keys[i] <= key) {
          key = keys[i];
          at = t;
        }
      }
      const uint32_t least = wave_min(at < n ? key : ~0u);
      const uint64_t has = __ballot(at < n && key == least);
      const int first = has ? __builtin_ctzll(has) : 0;
      const int32_t t = __builtin_amdgcn_readlane(at, first);   // n where the wavefront has none
      if ((tid & 63) == 0) {
        best[gone_n & 1][tid >> 6] = least;
        best_t[gone_n & 1][tid >> 6] = has ? t : n;
      }
      __syncthreads();
      uint32_t k = ~0u;
      int32_t kt = n;
#pragma unroll
      for (int w = SW - 1; w >= 0; --w)
        if (best_t[gone_n & 1][w] < n && best[gone_n & 1][w] <= k) {
          k = best[gone_n & 1][w];
          kt = best_t[gone_n & 1][w];
        }
      if (kt == n) break;   // no candidate is left
      last = k;
      last_t = kt;
    }
    prefix = last;
    cut = last_t;
  } else if (want > 0) {
    hist[2 * tid] = hist[2 * tid + 1] = 0;
    __syncthreads();
    for (int pass = 0; pass < 3; ++pass) {
      const int shift = pass == 0 ? 21 : pass == 1 ? 10 : 0;
      const uint32_t mask = pass == 2 ? 1023u : 2047u;
      // the bits above the digit, which have to be those found
      const uint32_t found = pass == 0 ? 0u : pass == 1 ? 0xffe00000u : 0xfffffc00u;
      for (int32_t part = 0; part < n; part += PART) {
        if (several) load_keys(part);
#pragma unroll
        for (int i = 0; i < KPT; ++i)
          if (keys[i] != 0 && (keys[i] & found) == prefix) atomicAdd(&hist[(keys[i] >> shift) & mask], 1);
      }
      __syncthreads();
      const int32_t h0 = hist[2 * tid], h1 = hist[2 * tid + 1];   // two bins per thread
      hist[2 * tid] = hist[2 * tid + 1] = 0;                      // for the next pass
      uint32_t all;
      const int32_t lo = (int32_t)before_me(h0 + h1, sums, all);   // candidates below them
      if (pass == 0) {
        gone_n = (int32_t)all < want ? (int32_t)all : want;
        rank = gone_n - 1;
      }
      if (gone_n > 0) {
        if (rank >= lo && rank < lo + h0) {
          pick[0] = 2 * tid;
          pick[1] = lo;
          pick[2] = h0;
        } else if (rank >= lo + h0 && rank < lo + h0 + h1) {
          pick[0] = 2 * tid + 1;
          pick[1] = lo + h0;
          pick[2] = h1;
        }
      }
      __syncthreads();
      if (gone_n == 0) break;
      prefix |= (uint32_t)pick[0] << shift;
      rank -= pick[1];
      all_ties = rank + 1 == pick[2];
      if (all_ties) {   // all of this prefix leave, whatever their other bits
        prefix |= (1u << shift) - 1;
        break;
      }
    }
  }
  const int32_t left = n - gone_n;
  // candidates below `prefix` leave, and of those equal to it the first rank + 1

  // ---- the lists, part by part in order ------------------------------------------------------------
  int32_t* to = FUSED ? lists : ml.to + b * ml.cap;
  int32_t* from = FUSED ? lists + FUSED_CHUNKS : ml.from + b * ml.cap;
  int32_t places = 0, movers = 0;   // of the parts before
  int32_t seen = 0;     // ties of the parts before
  if (gone_n > 0)
    for (int32_t part = 0; part < n; part += PART) {
      if (several) load_keys(part);
      const int32_t t = part + tid * KPT;
      uint32_t goes = 0;
#pragma unroll
      for (int i = 0; i < KPT; ++i)   // 0 wraps: it is no candidate
        goes |= keys[i] - 1u < prefix - (all_ties ? 0u : 1u) ? 1u << i : 0u;
      if (cut >= 0) {   // the same for the whole workgroup
#pragma unroll
        for (int i = 0; i < KPT; ++i) goes |= keys[i] == prefix && t + i <= cut ? 1u << i : 0u;
      } else if (!all_ties) {
        uint32_t tie = 0;
#pragma unroll
        for (int i = 0; i < KPT; ++i) tie |= keys[i] == prefix ? 1u << i : 0u;
        uint32_t all;
        int32_t ordinal = seen + (int32_t)before_me(__popc(tie), sums, all);
        seen += (int32_t)all;
        for (; tie != 0 && ordinal <= rank; ++ordinal) {
          goes |= tie & -tie;
          tie &= tie - 1;
        }
      }
      // of this thread's KPT bits, those below the new length and those of the sequence
      const auto first = [&](int32_t count) {
        return count >= KPT ? (uint32_t)(((uint64_t)1 << KPT) - 1) : count <= 0 ? 0u : (1u << count) - 1u;
      };
      const uint32_t place = goes & first(left - t), mover = ~goes & ~first(left - t) & first(n - t);
      // both counts of a part (at most 2^15 each) in one sum
      static_assert(PART <= 1 << 15, "halves of 16 bits");
      uint32_t all;
      const uint32_t at = before_me((uint32_t)__popc(mover) << 16 | (uint32_t)__popc(place), sums, all);
      int32_t pa = places + (int32_t)(at & 0xffffu), ma = movers + (int32_t)(at >> 16);
      places += (int32_t)(all & 0xffffu);
      movers += (int32_t)(all >> 16);
#pragma unroll
      for (int i = 0; i < KPT; ++i) {
        if (place >> i & 1) to[pa++] = t + i;
        if (mover >> i & 1) from[ma++] = t + i;
      }
      if (!FUSED && ml.gone) {   // the free places' bits, 16 to a store
        if constexpr (KPT == 4) {
          uint32_t w = place << 4 * (tid & 3);
          w |= dpp_or_0<0xB1, 0xf>(w);   // lane ^ 1, lane ^ 2
          w |= dpp_or_0<0x4E, 0xf>(w);
          if (t < n && (tid & 3) == 0) gst<uint16_t>(ml.gone + b * ml.words + t / 16, (uint16_t)w);
        } else if (t < n) {
#pragma unroll
          for (int i = 0; i < KPT; i += 16)
            gst<uint16_t>(ml.gone + b * ml.words + t / 16 + i / 16, (uint16_t)(place >> i));
        }
      }
    }
  const int32_t moves = places;
  // totals and positions of all places: the free ones' are overwritten after the barrier
  if (FUSED && (p.totals_out != p.totals || (pos && p.pos_out != p.pos)))
    for (int32_t t = tid; t < left; t += 4 * ST) {
      float x[4];
      int64_t y[4];
#pragma unroll
      for (int i = 0; i < 4; ++i) {
        const int32_t u = t + i * ST < left ? t + i * ST : left - 1;
        x[i] = gld<float>(tot + u);
        y[i] = pos ? gld<int64_t>(pos + u) : 0;
      }
#pragma unroll
      for (int i = 0; i < 4; ++i) {
        const int32_t u = t + i * ST;
        if (u >= left) continue;
        gst<float>(tot_out + u, x[i]);
        if (pos) gst<int64_t>(pos_out + u, y[i]);
      }
    }
  __threadfence_block();
  __syncthreads();
  for (int32_t j = tid; j < moves; j += ST) {
    const int32_t d = to[j], s = from[j];
    gst<float>(tot_out + d, gld<float>(tot + s));
    if (pos) gst<int64_t>(pos_out + d, gld<int64_t>(pos + s));
  }
  if (tid == 0) {
    if (!FUSED) ml.count[b] = moves;
    gst<int64_t>(p.len_out + b, left);
  }
  if constexpr (FUSED) copy_moves<false>(p, cs, b, to, from, moves, tid >> 6, SW);
}

// `per` workgroups for each sequence: the first `hand` hand on the totals and positions of what stays
// where it is, 4 * CT each; the others copy the moved rows.
__global__ __launch_bounds__(CT) void evict_copy_kernel(EvictParams p, MoveLists ml, CopyShape cs,
                                                        int32_t per, FastDiv div, int32_t hand) {
  const int32_t seq = fdiv(blockIdx.x, div), y = (int32_t)blockIdx.x - seq * per;
  const int64_t b = seq;
  if (y >= hand) {
    copy_moves<true>(p, cs, b, ml.to + b * ml.cap, ml.from + b * ml.cap, ml.count[b],
                     (y - hand) * (CT / 64) + (threadIdx.x >> 6), (per - hand) * (CT / 64));
    return;
  }
  const int64_t len = gld<int64_t>(p.len_out + b);
  const int32_t left = (int32_t)len, moves = ml.count[b];
  const float* tot = p.totals + b * p.ldt;
  const int64_t* pos = p.pos ? p.pos + b * p.ldt : nullptr;
#pragma unroll
  for (int i = 0; i < 4; ++i) {
    const int32_t t = (y * 4 + i) * CT + threadIdx.x;
    if (t >= left) continue;
    // (a sequence without moves has no bits; the free places' values come from the selection)
    if (moves > 0 && gld<uint16_t>(ml.gone + b * ml.words + t / 16) >> (t & 15) & 1) continue;
    gst<float>(p.totals_out + b * p.ldt + t, gld<float>(tot + t));
    if (pos) gst<int64_t>(p.pos_out + b * p.ldt + t, gld<int64_t>(pos + t));
  }
}

// Most moves of a sequence: no more than leave, and no more than stay below the new length.
int64_t move_cap(const EvictParams& p) {
  const int64_t gone = p.max_len > p.budget ? p.max_len - p.budget : 0;
  return gone < p.max_len / 2 ? gone : p.max_len / 2;
}

// Words of 16 bits of a sequence: a thread writes all of its own, up to 32 positions.
int64_t gone_words(const EvictParams& p) { return (p.max_len + 31) / 32 * 2; }

CopyShape copy_shape(const EvictParams& p) {
  CopyShape cs;
  const int32_t bytes = p.d * p.es;
  cs.unit = bytes >= 16 ? 16 : 2;
  cs.units = (bytes + cs.unit - 1) / cs.unit;
  cs.lanes = 1;
  while (cs.lanes < cs.units && cs.lanes < 64) cs.lanes *= 2;
  cs.heads = FastDiv(p.kv_heads);
  return cs;
}

// Totals and positions stay where they are.
bool in_place(const EvictParams& p) { return p.totals_out == p.totals && p.pos_out == p.pos; }

// Whether the selecting workgroup hands on and copies what there is itself, with its lists in LDS and no work
// space: a chunk or two per thread, and totals that stay where they are or are few (32 sequences of 2049
// that lose one position: 10.9 us so, 16.4 with a copy of its own; handed on and losing one: 4 of 8000
// 14.0 us so, 15.2 with the copy's workgroups, 4 of 16000 16.7 and 15.5).
bool one_launch(const EvictParams& p) {
  return move_cap(p) * p.kv_heads * copy_shape(p).units <= FUSED_CHUNKS && (in_place(p) || p.max_len <= 8 * ST);
}

// Workgroups of a sequence that hand on its totals, and with those that copy rows: two rows per set of lanes,
// at most 8192 of the latter in all (2048: 66.6 us for 8 x 16384 cut to 4096, 64.1 so).
int64_t hand_groups(const EvictParams& p) { return in_place(p) ? 0 : (p.max_len + 4 * CT - 1) / (4 * CT); }
int64_t copy_groups(const EvictParams& p) {
  const int64_t want = (move_cap(p) * p.kv_heads * copy_shape(p).lanes + 2 * CT - 1) / (2 * CT);
  const int64_t most = 8192 / p.n_seqs > 0 ? 8192 / p.n_seqs : 1;
  return hand_groups(p) + (want < most ? want : most);
}

}  // namespace

int64_t evict_work_floats(const EvictParams& p) {
  if (p.n_seqs > most_groups(ST) || move_cap(p) > (1 << 30) / p.kv_heads) return -1;
  if (one_launch(p)) return 0;
  if (copy_groups(p) * p.n_seqs > most_groups(CT)) return -1;
  return p.n_seqs * (2 * move_cap(p) + 1 + gone_words(p) / 2);
}

hipError_t launch_evict(const EvictParams& p, float* work, hipStream_t stream) {
  if (evict_work_floats(p) < 0) return hipErrorInvalidConfiguration;
  const CopyShape cs = copy_shape(p);
  MoveLists ml = {};
  ml.cap = move_cap(p);
  const dim3 grid((uint32_t)p.n_seqs);
#define TPP_SELECT(KPT, FUSED)                                                                    \
  hipLaunchKernelGGL((evict_select_kernel<KPT, FUSED>), grid, dim3(ST), 0, stream, p, ml, cs)
  if (one_launch(p)) {
    if (p.max_len <= 4 * ST) TPP_SELECT(4, true);
    else if (p.max_len <= 16 * ST) TPP_SELECT(16, true);
    else TPP_SELECT(32, true);
  } else {
    ml.words = gone_words(p);
    ml.count = reinterpret_cast<int32_t*>(work);
    ml.to = ml.count + p.n_seqs;
    ml.from = ml.to + p.n_seqs * ml.cap;
    ml.gone = in_place(p) ? nullptr : reinterpret_cast<uint16_t*>(ml.from + p.n_seqs * ml.cap);
    // as few positions to a thread as do: with 16, the fewest that were turned in LDS, one sequence of 3082
    // cut to 1541 18.3 us, 11.3 so
    if (p.max_len <= 4 * ST) TPP_SELECT(4, false);
    else if (p.max_len <= 16 * ST) TPP_SELECT(16, false);
    else TPP_SELECT(32, false);
    const int64_t per = copy_groups(p);
    if (per > 0)
      hipLaunchKernelGGL(evict_copy_kernel, dim3((uint32_t)(per * p.n_seqs)), dim3(CT), 0, stream, p, ml,
                         cs, (int32_t)per, FastDiv(per), (int32_t)hand_groups(p));
  }
#undef TPP_SELECT
  return hipGetLastError();
}

}  // namespace tpp

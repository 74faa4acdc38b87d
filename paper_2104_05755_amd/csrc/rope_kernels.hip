// rope_kernels.hip -- norms of query and key heads with the position rotation, forward (also into a
// paged cache) and backward, for gfx950.
//
// A row is one head of one token: y = x r w with r = 1 / sqrt(mean(x^2) + eps), then the pairs of its
// first rot_dim entries turned by the token's angles.  Both are linear in y, so a row needs one sum
// over its entries and one pass; the backward pass turns the gradient back (the rotation's transpose),
// u = g w, and needs one more sum, of u xn.  8 (16) operations per entry of 2 or 4 bytes: bound by HBM.
//
// A lane has two 16-byte chunks of a row, placed so that what the rotation turns together is in one lane --
// chunks at i and i + rot_dim / 2 in the halves form (behind the rotated part any two), any two in the pairs
// form -- and the sums fold over the 4 to 64 lanes of the row by register permutes.  A wavefront has
// 64 / lanes rows.  A part that is no multiple of a chunk ends with the chunk that ends with it, whose first
// entries another lane counts and stores.  Rows that are too short for that: one per wavefront, a rotated
// pair or an entry behind the rotated part to a lane, four rows in flight.
//
// 32 + 8 heads of 128 bf16, 8192 tokens: forward 33.2 us, 5.2 TB/s; backward 50.8 us, 5.0 TB/s, 4 of them the
// fold of the norm weights' gradients.  2048 tokens into a cache 10.8 us, 4.8 TB/s; one token 5.8 us from
// call to call, 3.0 of them the kernel.  1533 tokens of 21 + 7 fp32 heads of 77, backward: 15.5 us, 2.6
// TB/s, where a copy of as many bytes takes 7.0: a workgroup goes two or three times through a loop whose
// position, angles (4 bytes a load in the pairs form) and rows wait for each other, and the fold is 4 us.
#include <hip/hip_runtime.h>

#include <type_traits>

#include "brgemm_device.h"
#include "internal.h"

namespace tpp {
namespace {

using namespace dev;

constexpr int QT = 256;   // threads per workgroup: 4 wavefronts
constexpr int QW = QT / 64;

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

template <int CTRL>
__device__ __forceinline__ float dpp(float v) {
  return __int_as_float(__builtin_amdgcn_update_dpp(0, __float_as_int(v), CTRL, 0xf, 0xf, true));
}
// The sum over groups of LANES (4 .. 64) consecutive lanes, in every one of them.
template <int LANES>
__device__ __forceinline__ float lanes_sum(float v) {
  v += dpp<0xB1>(v);                           // lane ^ 1
  v += dpp<0x4E>(v);                           // lane ^ 2
  if constexpr (LANES >= 8) v += dpp<0x141>(v);    // the other quad of 8
  if constexpr (LANES >= 16) v += dpp<0x140>(v);   // the other 8 of 16
  if constexpr (LANES >= 32) {
    const auto w = __builtin_amdgcn_permlane16_swap(__float_as_uint(v), __float_as_uint(v), false, false);
    v = __uint_as_float(w[0]) + __uint_as_float(w[1]);
  }
  if constexpr (LANES >= 64) {
    const auto w = __builtin_amdgcn_permlane32_swap(__float_as_uint(v), __float_as_uint(v), false, false);
    v = __uint_as_float(w[0]) + __uint_as_float(w[1]);
  }
  return v;
}

// First element of head `head` of cache slot `slot` (inside the pools).
__device__ __forceinline__ int64_t slot_base(const QkParams& p, int64_t slot, int32_t head) {
  const int64_t page = p.n_slots <= 0x7fffffff ? (int64_t)fdiv((uint32_t)slot, p.page)
                                               : slot / p.page_size;
  return page * p.page_stride + (slot - page * p.page_size) * p.pos_stride + head * p.head_stride;
}

// Both sides are read before the choice (a lane's own choice of a kernel argument's address would put
// the arguments into scratch memory).
template <typename T>
__device__ __forceinline__ T pick(bool c, T a, T b) {
  return c ? a : b;
}

// A row of the forward pass: where it comes from and goes to.
struct Row {
  const void* x;
  void* out;            // null: not written
  const float* w;       // null: a value, copied
  int64_t from, to;     // elements
  int64_t pos;          // -1: padding
};
__device__ __forceinline__ Row row_at(const QkParams& p, int32_t row, int32_t per_token,
                                      const FastDiv& div) {
  Row r;
  const int64_t t = fdiv((uint32_t)row, div);
  int32_t head = row - (int32_t)t * per_token;
  const int64_t pos = gld<int64_t>(p.pos + t);
  r.pos = pos >= 0 && pos < p.n_positions ? pos : -1;
  const bool q = head < p.side[0].heads;
  if (!q) head -= p.side[0].heads;
  const bool v = !q && head >= p.side[1].heads;
  if (v) head -= p.side[1].heads;
  r.x = pick(q, p.side[0].x, pick(v, p.v, p.side[1].x));
  r.w = pick<const float*>(q, p.side[0].w, pick<const float*>(v, nullptr, p.side[1].w));
  r.from = t * pick(q, p.side[0].ldx, pick(v, p.ldv, p.side[1].ldx)) + (int64_t)head * p.d;
  r.out = pick(q, p.side[0].out, p.side[1].out);
  r.to = t * pick(q, p.side[0].ldo, p.side[1].ldo) + (int64_t)head * p.d;
  if (!q && p.slot) {
    const int64_t slot = gld<int64_t>(p.slot + t);
    const bool held = r.pos >= 0 && slot >= 0 && slot < p.n_slots;
    r.out = pick<void*>(held, pick(v, p.vc, p.kc), nullptr);
    if (held) r.to = slot_base(p, slot, head);
  }
  return r;
}

// ---- rows of whole chunks -----------------------------------------------------------------------
// V entries of a 16-byte chunk.
template <bool BF16>
struct Chunk {
  static constexpr int V = BF16 ? 8 : 4;
  static constexpr int ES = BF16 ? 2 : 4;
};
// How rows go through the caches.  What is read or written once only displaces what may be read again, from
// the 32 MB of the L2s and the 256 MB behind them: outputs beyond the former are stored past their replacement
// (4096 tokens of 32 + 8 heads of 128 bf16 23.4 us, 17.5 so), and where inputs and outputs pass half of the
// latter, inputs are loaded so too, if every load takes whole lines (8192 tokens 37.3 us and 32.9, the
// backward pass 56.0 and 51.2; 4096 tokens 25.4; rows of 160 bytes 15.4 and 18.1).
enum { CACHED, STREAM_OUT, STREAM };
template <bool BF16, int HOW>
__device__ __forceinline__ u32x4 load_chunk(const void* p, int64_t at) {
  const GLOBAL_AS u32x4_a2* from =
      (const GLOBAL_AS u32x4_a2*)(static_cast<const char*>(p) + at * Chunk<BF16>::ES);
  return HOW == STREAM ? (u32x4)__builtin_nontemporal_load(from) : (u32x4)*from;
}
template <bool BF16>
__device__ __forceinline__ void widen(u32x4 w, float (&x)[Chunk<BF16>::V]) {
#pragma unroll
  for (int e = 0; e < 4; ++e) {
    if constexpr (BF16) {
      x[2 * e] = __uint_as_float(w[e] << 16);
      x[2 * e + 1] = __uint_as_float(w[e] & 0xffff0000u);
    } else {
      x[e] = __uint_as_float(w[e]);
    }
  }
}
template <bool BF16, int HOW>
__device__ __forceinline__ void store_chunk(void* p, int64_t at, const float (&v)[Chunk<BF16>::V]) {
  u32x4 w;
#pragma unroll
  for (int e = 0; e < 4; ++e) {
    if constexpr (BF16) w[e] = pack_bf16x2(v[2 * e], v[2 * e + 1]);
    else w[e] = __float_as_uint(v[e]);
  }
  GLOBAL_AS u32x4_a2* to = (GLOBAL_AS u32x4_a2*)(static_cast<char*>(p) + at * Chunk<BF16>::ES);
  if constexpr (HOW != CACHED) __builtin_nontemporal_store((u32x4_a2)w, to);
  else *to = w;
}
template <int V>
__device__ __forceinline__ void load_floats(const float* p, float (&v)[V]) {
#pragma unroll
  for (int g = 0; g < V / 4; ++g) {
    const f32x4 w = gld<f32x4_a4>(p + 4 * g);
#pragma unroll
    for (int e = 0; e < 4; ++e) v[4 * g + e] = w[e];
  }
}

// The two chunks of lane c of a row: their first entries, and how many entries of each belong to another
// lane's chunk as well (a part that is no multiple of V ends with the chunk that ends with it).  `turned`:
// entry e of one goes with entry e of the other (halves).
struct Chunks {
  int32_t a, b, dup_a, dup_b;
  bool turned;
};
// Chunk c of the n >= V entries from `first` on; a chunk past the last is the last again, all of it another's.
template <int V>
__device__ __forceinline__ int32_t chunk_at(int32_t first, int32_t n, int32_t c, int32_t& dup) {
  const int32_t at = c * V < n - V ? c * V : n - V;
  dup = c * V - at < V ? c * V - at : V;
  return first + at;
}
template <int V, bool WHOLE>
__device__ __forceinline__ Chunks chunks_of(const QkParams& p, int32_t c) {
  Chunks k;
  const int32_t half = p.rot_dim / 2, rest = p.d - p.rot_dim;
  if constexpr (WHOLE) {
    const int32_t i = c * V;
    k.dup_a = k.dup_b = 0;
    k.turned = !p.pairs && i < half;
    k.a = p.pairs ? i : k.turned ? i : half + i;
    k.b = p.pairs ? p.d / 2 + i : k.turned ? half + i : p.rot_dim + rest / 2 + (i - half);
    return k;
  }
  const int32_t lanes = p.pairs ? 0 : (half + V - 1) / V;   // of the rotated part
  k.turned = c < lanes;
  if (k.turned) {
    k.a = chunk_at<V>(0, half, c, k.dup_a);
    k.b = half + k.a;
    k.dup_b = k.dup_a;
  } else {
    // two chunks of the rest (pairs: of the row); a rest below V is the end of the row's last chunk
    const int32_t first = p.pairs ? 0 : p.rot_dim, n = p.d - first, j = 2 * (c - lanes);
    if (n < V) {
      k.a = k.b = p.d - V;
      k.dup_a = V - n;
      k.dup_b = V;
    } else {
      k.a = chunk_at<V>(first, n, j, k.dup_a);
      k.b = chunk_at<V>(first, n, j + 1, k.dup_b);
    }
  }
  return k;
}

// Cosines and sines of the pairs of a lane's chunks: halves: entry e of both chunks; pairs: pair e / 2
// of chunk A at e / 2, of chunk B at V / 2 + e / 2.  What is not turned (behind the rotated part, or of a
// padding token: pos < 0) reads nothing and has cosine 1, sine 0.
template <int V>
__device__ __forceinline__ void load_angles(const QkParams& p, int64_t pos, int32_t a, int32_t b,
                                            bool turned, float (&c)[V], float (&s)[V]) {
  const int32_t half = p.rot_dim / 2;
  const float* row = p.rot + pos * p.rot_dim;
  if (!p.pairs) {
    if (turned && pos >= 0) {
      load_floats<V>(row + a, c);
      load_floats<V>(row + half + a, s);
    } else {
#pragma unroll
      for (int e = 0; e < V; ++e) {
        c[e] = 1.0f;
        s[e] = 0.0f;
      }
    }
    return;
  }
#pragma unroll
  for (int e = 0; e < V; ++e) {
    const int32_t i = e < V / 2 ? a / 2 + e : b / 2 + e - V / 2;
    const bool in = i < half && pos >= 0;
    c[e] = in ? gld<float>(row + i) : 1.0f;
    s[e] = in ? gld<float>(row + half + i) : 0.0f;
  }
}
// The rotation of a lane's two chunks (the other way where back).  What is not turned is left as it is: a
// sine of 0 times an infinity would be NaN in an entry that has nothing to do with it.
template <int V>
__device__ __forceinline__ void turn(const QkParams& p, bool back, const Chunks& k, const float (&c)[V],
                                     const float (&s)[V], float (&x)[V], float (&y)[V]) {
  const auto one = [&](bool on, float& a, float& b, float co, float si) {
    if (back) si = -si;
    const float t = a * co - b * si, u = b * co + a * si;
    a = on ? t : a;
    b = on ? u : b;
  };
  if (!p.pairs) {
#pragma unroll
    for (int e = 0; e < V; ++e) one(k.turned, x[e], y[e], c[e], s[e]);
  } else {
    const int32_t half = p.rot_dim / 2;
#pragma unroll
    for (int e = 0; e < V / 2; ++e) {
      one(k.a / 2 + e < half, x[2 * e], x[2 * e + 1], c[e], s[e]);
      one(k.b / 2 + e < half, y[2 * e], y[2 * e + 1], c[V / 2 + e], s[V / 2 + e]);
    }
  }
}

// Whether the rows are whole chunks whose pairs meet in a lane, and whether they go by chunks at all: both
// halves of the rotated part hold one, no pair lies across the border of the last (odd) one, and the chunks
// fit a wavefront.
bool whole_chunks(const QkParams& p) {
  const int32_t two = p.bf16 ? 16 : 8;
  return p.d % two == 0 && (p.pairs || p.rot_dim % two == 0);
}
// Lanes with chunks of a row.
int32_t chunk_lanes(const QkParams& p) {
  const int32_t v = p.bf16 ? 8 : 4;
  if (whole_chunks(p)) return p.d / (2 * v);
  const int32_t half = p.pairs ? 0 : p.rot_dim / 2, rest = p.d - 2 * half;
  return (half + v - 1) / v + ((rest + v - 1) / v + 1) / 2;
}
bool chunked(const QkParams& p) {
  const int32_t v = p.bf16 ? 8 : 4;
  if (p.d < v || chunk_lanes(p) > 64) return false;
  return p.pairs ? p.d % 2 == 0 || p.rot_dim <= p.d - v : p.rot_dim == 0 || p.rot_dim >= 2 * v;
}

template <int V>
__device__ __forceinline__ float squares(const float (&x)[V], int32_t dup) {
  float sum = 0.0f;
#pragma unroll
  for (int e = 0; e < V; ++e) sum += e >= dup ? x[e] * x[e] : 0.0f;
  return sum;
}
// A chunk's entries but those that another lane stores.
template <bool BF16, bool WHOLE, int HOW>
__device__ __forceinline__ void store_own(void* p, int64_t at, const float (&v)[Chunk<BF16>::V], int32_t dup) {
  if (WHOLE || dup == 0) {
    store_chunk<BF16, HOW>(p, at, v);
  } else {
#pragma unroll
    for (int e = 1; e < Chunk<BF16>::V; ++e)
      if (e >= dup) store_elem(p, at + e, v[e], BF16);
  }
}

template <bool BF16, bool WHOLE, int LANES, int HOW>
__global__ __launch_bounds__(QT) void qk_chunk_kernel(QkParams p, int32_t rows, int32_t per_token,
                                                      FastDiv div, int32_t used) {
  constexpr int V = Chunk<BF16>::V;
  const int lane = threadIdx.x & 63;
  const int32_t row = ((int32_t)blockIdx.x * QW + (threadIdx.x >> 6)) * (64 / LANES) + lane / LANES;
  const int32_t i = lane % LANES;
  if (row >= rows) return;   // whole rows: the folds below stay within one
  const Row r = row_at(p, row, per_token, div);
  if (!r.out) return;
  const bool in = i < used;   // lanes past the row's chunks repeat its first
  const Chunks k = chunks_of<V, WHOLE>(p, in ? i : 0);
  const int32_t a = k.a, b = k.b;
  const u32x4 wx = load_chunk<BF16, HOW>(r.x, r.from + a), wy = load_chunk<BF16, HOW>(r.x, r.from + b);
  if (!r.w) {
    if (in) {   // what two lanes store is the same
      gst<u32x4_a2>(static_cast<char*>(r.out) + (r.to + a) * Chunk<BF16>::ES, wx);
      gst<u32x4_a2>(static_cast<char*>(r.out) + (r.to + b) * Chunk<BF16>::ES, wy);
    }
    return;
  }
  float x[V], y[V], c[V], s[V], wa[V], wb[V];
  load_angles<V>(p, r.pos, a, b, k.turned, c, s);
  load_floats<V>(r.w + a, wa);
  load_floats<V>(r.w + b, wb);
  widen<BF16>(wx, x);
  widen<BF16>(wy, y);
  const float sum = squares<V>(x, k.dup_a) + squares<V>(y, k.dup_b);
  const float rstd = 1.0f / sqrtf(lanes_sum<LANES>(in ? sum : 0.0f) / (float)p.d + p.eps);
#pragma unroll
  for (int e = 0; e < V; ++e) {
    x[e] = r.pos < 0 ? 0.0f : x[e] * rstd * wa[e];
    y[e] = r.pos < 0 ? 0.0f : y[e] * rstd * wb[e];
  }
  turn<V>(p, false, k, c, s, x, y);
  if (in) {
    store_own<BF16, WHOLE, HOW>(r.out, r.to + a, x, k.dup_a);
    store_own<BF16, WHOLE, HOW>(r.out, r.to + b, y, k.dup_b);
  }
}

// Backward.  Workgroup w of a side (the first nq of the queries, the rest of the keys) takes every n-th
// set of QW * 64 / LANES rows and keeps its part of the weights' gradient in registers; parts go to
// `part` (a row of D per workgroup), or straight to dw where a side has one workgroup.
template <bool BF16, bool WHOLE, int LANES, int HOW>
__global__ __launch_bounds__(QT) void qk_backward_chunk_kernel(QkParams p, int32_t nq, float* part,
                                                               int32_t used) {
  constexpr int V = Chunk<BF16>::V, SLOTS = 64 / LANES;
  __shared__ float acc[QW][LANES * 2 * V];
  const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
  const bool keys = (int32_t)blockIdx.x >= nq;
  const int32_t wg = blockIdx.x - (keys ? nq : 0), n_wg = keys ? (int32_t)gridDim.x - nq : nq;
  const QkSide sd = keys ? p.side[1] : p.side[0];
  const bool in = lane % LANES < used;
  const Chunks k = chunks_of<V, WHOLE>(p, in ? lane % LANES : 0);
  const int32_t a = k.a, b = k.b;
  float wa[V], wb[V], da[V], db[V];
#pragma unroll
  for (int e = 0; e < V; ++e) wa[e] = wb[e] = da[e] = db[e] = 0.0f;
  // this lane's row, stepped without divisions
  const int64_t first = ((int64_t)wg * QW + wave) * SLOTS + lane / LANES;
  const int64_t step = (int64_t)n_wg * QW * SLOTS;
  const int64_t step_t = step / (sd.heads ? sd.heads : 1);
  const int32_t step_h = (int32_t)(step - step_t * sd.heads);
  int64_t t = sd.heads ? first / sd.heads : p.tokens;
  int32_t h = (int32_t)(first - t * sd.heads);
  if (t < p.tokens) {
    load_floats<V>(sd.w + a, wa);
    load_floats<V>(sd.w + b, wb);
  }
  while (t < p.tokens) {   // the lanes of a row leave together
    const int64_t pos = gld<int64_t>(p.pos + t);
    const bool held = pos >= 0 && pos < p.n_positions;
    const int64_t hd = (int64_t)h * p.d;
    const int64_t fx = t * sd.ldx + hd, fg = t * sd.ldg + hd;
    const u32x4 xw = load_chunk<BF16, HOW>(sd.x, fx + a), yw = load_chunk<BF16, HOW>(sd.x, fx + b);
    const u32x4 gw = load_chunk<BF16, HOW>(sd.g, fg + a), fw = load_chunk<BF16, HOW>(sd.g, fg + b);
    float x[V], y[V], g[V], f[V], c[V], s[V];
    load_angles<V>(p, held ? pos : -1, a, b, k.turned, c, s);
    widen<BF16>(xw, x);
    widen<BF16>(yw, y);
    widen<BF16>(gw, g);
    widen<BF16>(fw, f);
    turn<V>(p, true, k, c, s, g, f);
    const float xx = squares<V>(x, k.dup_a) + squares<V>(y, k.dup_b);
    float ux = 0.0f;
#pragma unroll
    for (int e = 0; e < V; ++e) {
      ux += e >= k.dup_a ? g[e] * wa[e] * x[e] : 0.0f;
      ux += e >= k.dup_b ? f[e] * wb[e] * y[e] : 0.0f;
    }
    const float r = 1.0f / sqrtf(lanes_sum<LANES>(in ? xx : 0.0f) / (float)p.d + p.eps);
    const float m = lanes_sum<LANES>(in ? ux : 0.0f) * r / (float)p.d;   // mean(u xn)
#pragma unroll
    for (int e = 0; e < V; ++e) {
      const float xn = x[e] * r, yn = y[e] * r;
      if (held) {
        da[e] += g[e] * xn;
        db[e] += f[e] * yn;
      }
      x[e] = held ? r * (g[e] * wa[e] - xn * m) : 0.0f;
      y[e] = held ? r * (f[e] * wb[e] - yn * m) : 0.0f;
    }
    if (in) {
      store_own<BF16, WHOLE, HOW>(sd.out, t * sd.ldo + hd + a, x, k.dup_a);
      store_own<BF16, WHOLE, HOW>(sd.out, t * sd.ldo + hd + b, y, k.dup_b);
    }
    t += step_t;
    h += step_h;
    if (h >= sd.heads) {
      h -= sd.heads;
      ++t;
    }
  }
  // the rows of a wavefront, then the wavefronts, added in a fixed order
#pragma unroll
  for (int e = 0; e < V; ++e) {
#pragma unroll
    for (int d = LANES; d < 64; d *= 2) {
      da[e] += __shfl_xor(da[e], d, 64);
      db[e] += __shfl_xor(db[e], d, 64);
    }
    if (lane < LANES) {
      acc[wave][e * LANES + lane] = da[e];
      acc[wave][(V + e) * LANES + lane] = db[e];
    }
  }
  __syncthreads();
  for (int32_t j = threadIdx.x; j < LANES * 2 * V; j += QT) {
    const int32_t ln = j % LANES, e = j / LANES;
    if (ln >= used) continue;
    const Chunks o = chunks_of<V, WHOLE>(p, ln);
    if (e < V ? e < o.dup_a : e - V < o.dup_b) continue;
    const float v = ((acc[0][j] + acc[1][j]) + acc[2][j]) + acc[3][j];
    gst<float>((part ? part + (int64_t)blockIdx.x * p.d : sd.dw) + (e < V ? o.a + e : o.b + e - V), v);
  }
}

// ---- other rows -----------------------------------------------------------------------------------
constexpr int IN_FLIGHT = 4;   // rows of a wavefront

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

template <int NU>
__global__ __launch_bounds__(QT) void qk_unit_kernel(QkParams p, int32_t rows, int32_t per_token,
                                                     FastDiv div) {
  const int lane = threadIdx.x & 63;
  const int32_t row0 = ((int32_t)blockIdx.x * QW + (threadIdx.x >> 6)) * IN_FLIGHT;
  const int32_t units = p.d - p.rot_dim / 2;
  Row r[IN_FLIGHT];
  float xa[IN_FLIGHT][NU], xb[IN_FLIGHT][NU];
#pragma unroll
  for (int k = 0; k < IN_FLIGHT; ++k) {
    r[k] = row_at(p, row0 + k < rows ? row0 + k : rows - 1, per_token, div);
    if (row0 + k >= rows) r[k].out = nullptr;
#pragma unroll
    for (int i = 0; i < NU; ++i) {
      const int32_t u = lane + 64 * i;
      xa[k][i] = xb[k][i] = 0.0f;
      if (u >= units) continue;
      int32_t a, b;
      unit_entries(p, u, a, b);
      xa[k][i] = load_elem(r[k].x, r[k].from + a, p.bf16);
      if (b >= 0) xb[k][i] = load_elem(r[k].x, r[k].from + b, p.bf16);
    }
  }
#pragma unroll
  for (int k = 0; k < IN_FLIGHT; ++k) {
    float sum = 0.0f;
#pragma unroll
    for (int i = 0; i < NU; ++i) sum += xa[k][i] * xa[k][i] + xb[k][i] * xb[k][i];
    const float rstd = 1.0f / sqrtf(lanes_sum<64>(sum) / (float)p.d + p.eps);
    if (!r[k].out) continue;
#pragma unroll
    for (int i = 0; i < NU; ++i) {
      const int32_t u = lane + 64 * i;
      if (u >= units) continue;
      int32_t a, b;
      unit_entries(p, u, a, b);
      float ya = xa[k][i], yb = xb[k][i];   // a value: copied
      if (r[k].w) {
        const bool held = r[k].pos >= 0;
        ya = held ? ya * rstd * gld<float>(r[k].w + a) : 0.0f;
        if (b >= 0 && held) {
          yb = yb * rstd * gld<float>(r[k].w + b);
          const float c = gld<float>(p.rot + r[k].pos * p.rot_dim + u);
          const float s = gld<float>(p.rot + r[k].pos * p.rot_dim + p.rot_dim / 2 + u);
          const float t = ya * c - yb * s;
          yb = yb * c + ya * s;
          ya = t;
        } else {
          yb = 0.0f;
        }
      }
      store_elem(r[k].out, r[k].to + a, ya, p.bf16);
      if (b >= 0) store_elem(r[k].out, r[k].to + b, yb, p.bf16);
    }
  }
}

template <int NU>
__global__ __launch_bounds__(QT) void qk_backward_unit_kernel(QkParams p, int32_t nq, float* part) {
  __shared__ float acc[QW][2 * 64 * NU];
  const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
  const bool keys = (int32_t)blockIdx.x >= nq;
  const int32_t wg = blockIdx.x - (keys ? nq : 0), n_wg = keys ? (int32_t)gridDim.x - nq : nq;
  const QkSide sd = keys ? p.side[1] : p.side[0];
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
  const int64_t step = (int64_t)n_wg * QW * IN_FLIGHT;
  for (int64_t row0 = ((int64_t)wg * QW + wave) * IN_FLIGHT; row0 < rows; row0 += step) {
    float xa[IN_FLIGHT][NU], xb[IN_FLIGHT][NU], ga[IN_FLIGHT][NU], gb[IN_FLIGHT][NU];
    float c[IN_FLIGHT][NU], s[IN_FLIGHT][NU];
    int64_t to[IN_FLIGHT];
    bool held[IN_FLIGHT];
    // the first row's token by division, the others' by counting on
    int64_t t = row0 / sd.heads;
    int32_t head = (int32_t)(row0 - t * sd.heads);
#pragma unroll
    for (int k = 0; k < IN_FLIGHT; ++k) {
      const bool there = row0 + k < rows;
      const int64_t pos = there ? gld<int64_t>(p.pos + t) : -1;
      held[k] = pos >= 0 && pos < p.n_positions;
      const int64_t hd = (int64_t)head * p.d;
      to[k] = there ? t * sd.ldo + hd : -1;
#pragma unroll
      for (int i = 0; i < NU; ++i) {
        const int32_t u = lane + 64 * i;
        xa[k][i] = xb[k][i] = ga[k][i] = gb[k][i] = s[k][i] = 0.0f;
        c[k][i] = 1.0f;
        if (u >= units || !held[k]) continue;
        int32_t a, b;
        unit_entries(p, u, a, b);
        xa[k][i] = load_elem(sd.x, t * sd.ldx + hd + a, p.bf16);
        ga[k][i] = load_elem(sd.g, t * sd.ldg + hd + a, p.bf16);
        if (b >= 0) {
          xb[k][i] = load_elem(sd.x, t * sd.ldx + hd + b, p.bf16);
          gb[k][i] = load_elem(sd.g, t * sd.ldg + hd + b, p.bf16);
          c[k][i] = gld<float>(p.rot + pos * p.rot_dim + u);
          s[k][i] = gld<float>(p.rot + pos * p.rot_dim + p.rot_dim / 2 + u);
        }
      }
      if (++head == sd.heads) {
        head = 0;
        ++t;
      }
    }
#pragma unroll
    for (int k = 0; k < IN_FLIGHT; ++k) {
      float xx = 0.0f, ux = 0.0f;
#pragma unroll
      for (int i = 0; i < NU; ++i) {
        if (lane + 64 * i < p.rot_dim / 2) {   // (an entry alone: 0 times an infinity would be NaN)
          const float g = ga[k][i] * c[k][i] + gb[k][i] * s[k][i];
          gb[k][i] = gb[k][i] * c[k][i] - ga[k][i] * s[k][i];
          ga[k][i] = g;
        }
        xx += xa[k][i] * xa[k][i] + xb[k][i] * xb[k][i];
        ux += ga[k][i] * wa[i] * xa[k][i] + gb[k][i] * wb[i] * xb[k][i];
      }
      const float r = 1.0f / sqrtf(lanes_sum<64>(xx) / (float)p.d + p.eps);
      const float m = lanes_sum<64>(ux) * r / (float)p.d;   // mean(u xn)
      if (to[k] < 0) continue;
#pragma unroll
      for (int i = 0; i < NU; ++i) {
        const int32_t u = lane + 64 * i;
        if (u >= units) continue;
        int32_t a, b;
        unit_entries(p, u, a, b);
        const float na = xa[k][i] * r, nb = xb[k][i] * r;
        if (held[k]) {
          da[i] += ga[k][i] * na;
          db[i] += gb[k][i] * nb;
        }
        store_elem(sd.out, to[k] + a, held[k] ? r * (ga[k][i] * wa[i] - na * m) : 0.0f, p.bf16);
        if (b >= 0) store_elem(sd.out, to[k] + b, held[k] ? r * (gb[k][i] * wb[i] - nb * m) : 0.0f, p.bf16);
      }
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

// dw of a side: its workgroups' parts.  A workgroup has 16 entries; 64 sets of 16 lanes take every 64th part,
// 8 in flight, and meet in order.
constexpr int FT = 1024, FE = 16, FS = FT / FE;
__global__ __launch_bounds__(FT) void qk_fold_kernel(QkParams p, int32_t nq, int32_t nk,
                                                     const float* part) {
  __shared__ float acc[FS][FE];
  const bool keys = blockIdx.y != 0;
  const int32_t heads = keys ? p.side[1].heads : p.side[0].heads;
  if (heads == 0) return;
  const int32_t set = threadIdx.x / FE, lane = threadIdx.x % FE;
  const int32_t e = blockIdx.x * FE + lane, n = keys ? nk : nq;
  const float* from = part + (int64_t)(keys ? nq : 0) * p.d + e;
  float sum = 0.0f;
  for (int32_t i = set; i < n; i += 8 * FS) {
    float x[8];
#pragma unroll
    for (int u = 0; u < 8; ++u)
      x[u] = e < p.d && i + u * FS < n ? gld<float>(from + (int64_t)(i + u * FS) * p.d) : 0.0f;
#pragma unroll
    for (int u = 0; u < 8; ++u) sum += x[u];
  }
  acc[set][lane] = sum;
  __syncthreads();
#pragma unroll
  for (int h = FS / 2; h > 0; h /= 2) {
    if (set < h) acc[set][lane] += acc[set + h][lane];
    __syncthreads();
  }
  if (set == 0 && e < p.d) gst<float>((keys ? p.side[1].dw : p.side[0].dw) + e, acc[0][lane]);
}

int lanes_of(const QkParams& p) {
  int lanes = 4;
  while (lanes < chunk_lanes(p)) lanes *= 2;
  return lanes;
}

// Rows that a wavefront takes at once.
int rows_at_once(const QkParams& p) { return chunked(p) ? 64 / lanes_of(p) : IN_FLIGHT; }

// How a pass goes through the caches, by what it moves (see above).
int cache_use(const QkParams& p, bool backward) {
  if (p.slot || !whole_chunks(p)) return CACHED;   // keys and queries on their way to attention
  const int64_t es = p.bf16 ? 2 : 4;
  const int64_t out = p.tokens * (p.side[0].heads + p.side[1].heads) * p.d * es;
  if (out <= int64_t(32) << 20) return CACHED;
  bool lines = p.d * es % 128 == 0;
  for (const QkSide& s : p.side)
    if (s.heads > 0)
      lines = lines && s.ldx * es % 128 == 0 && (reinterpret_cast<uintptr_t>(s.x) & 127) == 0 &&
              (!backward || (s.ldg * es % 128 == 0 && (reinterpret_cast<uintptr_t>(s.g) & 127) == 0));
  return lines && out * (backward ? 3 : 2) > int64_t(128) << 20 ? STREAM : STREAM_OUT;
}

// f(type, whole chunks, lanes of a row, cache use) for the instance that rows of chunks take.
template <bool BF16, bool WHOLE, int HOW, typename F>
void by_lanes(const QkParams& p, const F& f) {
  const std::integral_constant<bool, BF16> t;
  const std::integral_constant<bool, WHOLE> w;
  const IntC<HOW> how;
  switch (lanes_of(p)) {
    case 4: return f(t, w, IntC<4>(), how);
    case 8: return f(t, w, IntC<8>(), how);
    case 16: return f(t, w, IntC<16>(), how);
    case 32: return f(t, w, IntC<32>(), how);
  }
  // (512 entries of bf16 in whole chunks are 32 lanes)
  if constexpr (!BF16 || !WHOLE) f(t, w, IntC<64>(), how);
}
template <typename F>
void by_chunks(const QkParams& p, bool backward, const F& f) {
  const int how = cache_use(p, backward);
  const auto type = [&](auto t) {
    constexpr bool BF16 = decltype(t)::value;
    if (!whole_chunks(p)) by_lanes<BF16, false, CACHED>(p, f);
    else if (how == STREAM) by_lanes<BF16, true, STREAM>(p, f);
    else if (how == STREAM_OUT) by_lanes<BF16, true, STREAM_OUT>(p, f);
    else by_lanes<BF16, true, CACHED>(p, f);
  };
  if (p.bf16) type(std::true_type());
  else type(std::false_type());
}

// Workgroups of the two sides in the backward pass: 1024 in all where there are rows for them.
void backward_groups(const QkParams& p, int32_t& nq, int32_t& nk) {
  const int32_t heads = p.side[0].heads + p.side[1].heads, rows = QW * rows_at_once(p);
  int32_t n[2];
  for (int s = 0; s < 2; ++s) {
    const int64_t full = (p.tokens * p.side[s].heads + rows - 1) / rows;
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
  // rows count in 31 bits within a launch, and threads in 32
  const int32_t wg = QW * rows_at_once(p);
  const int64_t most = most_groups(QT) * wg, step = (most < 0x7fff0000 ? most : 0x7fff0000) / per;
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
    const int32_t rows = (int32_t)(q.tokens * per);
    const dim3 grid((uint32_t)(((int64_t)rows + wg - 1) / wg));
#define TPP_QK_UNITS(NU) \
  hipLaunchKernelGGL((qk_unit_kernel<NU>), grid, dim3(QT), 0, stream, q, rows, per, div)
    if (chunked(p)) {
      by_chunks(p, false, [&](auto bf16, auto whole, auto lanes, auto how) {
        hipLaunchKernelGGL((qk_chunk_kernel<decltype(bf16)::value, decltype(whole)::value,
                                            decltype(lanes)::value, decltype(how)::value>),
                           grid, dim3(QT), 0, stream, q, rows, per, div, chunk_lanes(p));
      });
    } else if (units <= 64) {
      TPP_QK_UNITS(1);
    } else if (units <= 128) {
      TPP_QK_UNITS(2);
    } else if (units <= 256) {
      TPP_QK_UNITS(4);
    } else {
      TPP_QK_UNITS(8);
    }
#undef TPP_QK_UNITS
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
#define TPP_QKB_UNITS(NU) \
  hipLaunchKernelGGL((qk_backward_unit_kernel<NU>), dim3(nq + nk), dim3(QT), 0, stream, p, nq, work)
  if (chunked(p)) {
    by_chunks(p, true, [&](auto bf16, auto whole, auto lanes, auto how) {
      hipLaunchKernelGGL((qk_backward_chunk_kernel<decltype(bf16)::value, decltype(whole)::value,
                                                   decltype(lanes)::value, decltype(how)::value>),
                         dim3(nq + nk), dim3(QT), 0, stream, p, nq, work, chunk_lanes(p));
    });
  } else if (units <= 64) {
    TPP_QKB_UNITS(1);
  } else if (units <= 128) {
    TPP_QKB_UNITS(2);
  } else if (units <= 256) {
    TPP_QKB_UNITS(4);
  } else {
    TPP_QKB_UNITS(8);
  }
#undef TPP_QKB_UNITS
  if (work)
    hipLaunchKernelGGL(qk_fold_kernel, dim3((p.d + FE - 1) / FE, 2), dim3(FT), 0, stream, p, nq, nk, work);
  return hipGetLastError();
}

}  // namespace tpp

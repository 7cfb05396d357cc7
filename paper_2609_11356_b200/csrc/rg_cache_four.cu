// Rows into a paged cache of four-bit codes (rg_kv_append_four), with the rotation on the way, and back out of it (rg_kv_read_four).  The format is
// rg_four_bit.cuh's.
//
// Keys are rotated and quantised in 64 bits (the pair's sine and cosine as well): a code is a step function, and an fp32 rotation, whose result is off by
// 2^-22 or so, would put one key in some hundred thousand on the other side of a border between codes, so that two caches of one text would differ.  (Doing only
// the close ones in 64 bits costs more: their code is never in the instruction cache, 3 us in a call of 64 tokens.)  Queries are rotated as rg_rope does it,
// with its bits.
//
// What bounds it: for single tokens the latency of place, page, sine in 64 bits and store; for prompts waits for memory that the warps of an SM do not cover and, next to
// them, instructions (by the counters issue slots 59 % busy appending, 58 % reading; of 11 and 16 cycles that a warp takes for an instruction 4.6 and 7.5 are waits for loads).
// A thread takes one group of 16 elements of one row (a query, or a key and a value) and the group
// that the rotation pairs with it: 16-byte loads, several of them in flight, no exchange between threads, and a key's 8 code bytes and its scale byte are
// a thread's own.  Threads run over two groups, then the CTA's tokens, then the chunks of the head: neighbours write the neighbouring slots of a tile.
// 8 key heads and 32 query heads of 128 in bf16: 10.5 k tokens of 5 prompts 56 us (4 TB/s; 99.8 with remainders instead of magic sums, 67.5 with a second look at
// close codes, 63 with queries dealt out as keys are; rg_kv_append, which moves more bytes and has no codes to make, 47.5), 64 single tokens 5.3 us (3.7).  Reading those tokens
// back: 17.2 us (55 MB: 3.2 TB/s, half the copy's rate) and 3.2; two heads of a thread in flight 18.1.
#include <algorithm>
#include <type_traits>

#include "rg_common.cuh"
#include "rg_four_bit.cuh"
#include "rg_internal.h"
#include "rg_place.cuh"

namespace rg {

__device__ unsigned int g_cache4_status_word = 0;

namespace {

constexpr int THREADS = 256;
constexpr int TOKENS = THREADS / 32;                   // most tokens of a CTA: one warp looks up each one's place; a tile's slots

template <int DT>
using Elem = typename std::conditional<DT == RG_F32, float, uint16_t>::type;

// Eight elements as they lie in memory, and as fp32.
template <int DT>
struct Eight { uint4 w[DT == RG_F32 ? 2 : 1]; };
template <int DT>
__device__ __forceinline__ Eight<DT> load8(const Elem<DT>* src, bool vec) {
  Eight<DT> r;
  if (vec) {
#pragma unroll
    for (int i = 0; i < (DT == RG_F32 ? 2 : 1); ++i) r.w[i] = *(reinterpret_cast<const uint4*>(src) + i);
  } else {
    Elem<DT>* const to = reinterpret_cast<Elem<DT>*>(&r);
#pragma unroll
    for (int i = 0; i < 8; ++i) to[i] = src[i];
  }
  return r;
}
template <int DT>
__device__ __forceinline__ void widen8(const Eight<DT>& r, float* v) {
  if constexpr (DT == RG_F32) {
#pragma unroll
    for (int i = 0; i < 2; ++i) { v[4 * i] = __uint_as_float(r.w[i].x); v[4 * i + 1] = __uint_as_float(r.w[i].y); v[4 * i + 2] = __uint_as_float(r.w[i].z); v[4 * i + 3] = __uint_as_float(r.w[i].w); }
  } else {
    const uint32_t w[4] = {r.w[0].x, r.w[0].y, r.w[0].z, r.w[0].w};
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      v[2 * i] = DT == RG_F16 ? f16_bits_to_f32(w[i] & 0xffffu) : bf16_bits_to_f32(w[i]);          // bf16: the upper half leaves by the shift
      v[2 * i + 1] = DT == RG_F16 ? f16_bits_to_f32(w[i] >> 16) : __uint_as_float(w[i] & 0xffff0000u);
    }
  }
}
template <int DT>
__device__ __forceinline__ void store8(Elem<DT>* dst, const float* v) {
  if constexpr (DT == RG_F32) {
    *reinterpret_cast<float4*>(dst) = make_float4(v[0], v[1], v[2], v[3]);
    *reinterpret_cast<float4*>(dst + 4) = make_float4(v[4], v[5], v[6], v[7]);
  } else {
    *reinterpret_cast<uint4*>(dst) = make_uint4(pack_16x2(v[0], v[1], DT), pack_16x2(v[2], v[3], DT), pack_16x2(v[4], v[5], DT), pack_16x2(v[6], v[7], DT));
  }
}

// Where the pages of the CTA's tokens are: page (-1: no place in the cache, -2: a row of no sequence), slot and place.
struct Places {
  int64_t page[TOKENS], place[TOKENS];
  int32_t slot[TOKENS];
  __device__ __forceinline__ void look_up(const Cache4Params& p, int64_t t0, int n_tok, bool read) {
    const int w = threadIdx.x >> 5;
    if (w >= n_tok) return;
    int seq;
    int64_t at = 0, id = -2;
    if (place_of(p, t0 + w, seq, at)) {
      id = page_of(p, seq, at);
      if (id < 0 && (threadIdx.x & 31) == 0) atomicCAS(&g_cache4_status_word, 0u, (unsigned)(read ? RG_PAGE_CODE_READ : RG_PAGE_CODE_APPEND));
    }
    if ((threadIdx.x & 31) == 0) { page[w] = id; slot[w] = (int32_t)(at >= 0 ? at % p.page_size : 0); place[w] = at; }
  }
};

// A thread's token, chunk of 32 elements, half of it (its group) and first head, and how many heads further its next one is.  Threads run over the halves, the
// tokens, the chunks and the heads; what is left of the CTA has nothing to do.
struct Spot {
  int t, chunk, g, head, heads;
  bool active;
  __device__ __forceinline__ Spot(const Cache4Params& p, int n_tok) {
    const int per_head = p.d / 32 * 2 * p.tile, r = threadIdx.x % per_head;
    head = threadIdx.x / per_head;
    heads = THREADS / per_head;
    g = r & 1;
    t = (r >> 1) & (p.tile - 1);
    chunk = (r >> 1) / p.tile;
    active = head < heads && t < n_tok;
  }
};

// A pair's place in the CTA's tables of sines: eight pairs are a thread's, and threads that hold neighbouring eights, or one of neighbouring tokens, read different
// banks (eights are 9 apart; rows of keys 2, of queries 8 modulo 16).
__device__ __forceinline__ int pair_at(int row, int t, int j) { return t * row + j + (j >> 3); }
__host__ __device__ constexpr int pair_row(int half) { const int n = half + (half >> 3) + 1; return n + (18 - n % 16) % 16; }
__host__ __device__ constexpr int query_row(int half) { const int n = half + (half >> 3) + 1; return n + (24 - n % 16) % 16; }

// A query's 16 elements: pairs 8 u .. 8 u + 7 whole (another thread's stores must not reach them: the result may lie where the queries do), what is not
// rotated as it lies.  Element c of this order, as an element of the head.
__device__ __forceinline__ int paired(const Cache4Params& p, int c) { return c >= p.rot || p.style == RG_ROPE_PAIRS ? c : (c >> 1) + (c & 1) * (p.rot >> 1); }
// HALVES: pair e is elements e of the two eights, else neighbours.
__device__ __forceinline__ float turn_one(float a, float b, float s, float c) { return f_fma(b, s, f_mul(a, c)); }
__device__ __forceinline__ double turn_one(double a, double b, double s, double c) { return __fma_rn(b, s, __dmul_rn(a, c)); }
template <bool HALVES, typename T, typename T2>
__device__ __forceinline__ void rotate16(T (&v)[16], const T2* cs) {
#pragma unroll
  for (int e = 0; e < 8; ++e) {
    const T2 w = cs[e];
    T &x = v[HALVES ? e : 2 * e], &y = v[HALVES ? 8 + e : 2 * e + 1];
    const T x0 = x;
    x = turn_one(x0, -y, w.y, w.x);
    y = turn_one(y, x0, w.y, w.x);
  }
}
// Heads that no whole eights are rotated in, or rows that no 16-byte access reaches: element by element.
template <int DT>
__device__ __noinline__ void rotate_query_slowly(const Cache4Params& p, const Elem<DT>* src, Elem<DT>* dst, int u, const float2* cs) {
  for (int e = 0; e < 8; ++e) {
    const int i = paired(p, 16 * u + 2 * e), j = paired(p, 16 * u + 2 * e + 1);
    float x = load_scalar(src, DT, i), y = load_scalar(src, DT, j);
    if (16 * u + 2 * e < p.rot) {
      const float2 w = cs[e];
      const float x0 = x;
      x = f_fma(-y, w.y, f_mul(x0, w.x));
      y = f_fma(x0, w.y, f_mul(y, w.x));
    }
    store_scalar(dst, DT, i, x);
    store_scalar(dst, DT, j, y);
  }
}

// Pair j's angle for a token, as a fraction of a turn.
__device__ __forceinline__ double turn_of(const Cache4Params& p, int64_t token, int64_t place, int j) {
  int64_t pos = place;
  if (p.pos) {
    const int axis = (j >= p.axis_end[0]) + (j >= p.axis_end[1]) + (j >= p.axis_end[2]);
    const int64_t k = (int64_t)axis * p.pos_ld + token;
    pos = p.pos64 ? static_cast<const int64_t*>(p.pos)[k] : (int64_t)static_cast<const int32_t*>(p.pos)[k];
  }
  const double turns = __dmul_rn(__dmul_rn((double)pos, p.inv_freq[j]), 0x1.45f306dc9c883p-3);      // 1 / (2 pi)
  return turns - rint(turns);
}
// An element's pair, the other element of it, and whether it is the second of the two.
__device__ __forceinline__ int pair_of(const Cache4Params& p, int i, int& other, bool& second) {
  const int half = p.rot >> 1;
  const bool pairs = p.style == RG_ROPE_PAIRS;
  second = pairs ? i & 1 : i >= half;
  other = pairs ? i ^ 1 : second ? i - half : i + half;
  return pairs ? i >> 1 : second ? other : i;
}
// An element of a key, rotated in 64 bits; or, not rotated, of a value.
template <int DT>
__device__ __forceinline__ double element(const Cache4Params& p, const Elem<DT>* src, bool rotate, int i, const double2* cs, int row, int t) {
  const double x = (double)load_scalar(src, DT, i);
  if (!rotate || i >= p.rot) return x;
  int other;
  bool second;
  const int j = pair_of(p, i, other, second);
  const double y = (double)load_scalar(src, DT, other);
  const double2 w = cs[pair_at(row, t, j)];
  return __fma_rn(second ? y : -y, w.y, __dmul_rn(x, w.x));
}
// Codes and scale byte of a group with numbers that are too large, infinite or NaN (which becomes 0): elements e0 .. e0 + n - 1, n = 16, or n = 8 where the neighbouring
// lane has the other eight and calls too.
struct Codes { uint32_t w[2], b; };
template <int DT>
__device__ __noinline__ Codes quantise_slowly(const Cache4Params& p, const Elem<DT>* src, bool rotate, int e0, int n, const double2* cs, int row, int t) {
  double amax = 0.0;
#pragma unroll 1
  for (int e = 0; e < n; ++e) amax = fmax(amax, fabs(element<DT>(p, src, rotate, e0 + e, cs, row, t)));       // passes over NaN
  if (n == 8) amax = fmax(amax, __shfl_xor_sync(3u << (threadIdx.x & 30), amax, 1));
  Codes r = {{0u, 0u}, scale4_byte(magnitude4_value(((uint32_t)__double2hiint(amax) & 0x7fffffffu) | min((uint32_t)__double2loint(amax), 1u)))};
  const double inv = inverse4(scale4(r.b));
#pragma unroll 1
  for (int e = 0; e < n; ++e) {
    double x = element<DT>(p, src, rotate, e0 + e, cs, row, t);
    x = x == x ? fmin(fmax(x, -61440.0), 57600.0) : 0.0;
    const double t = __dadd_rn(__dadd_rn(__dmul_rn(x, inv), 6144.0), -6144.0);
    r.w[e >> 3] |= (uint32_t)((int)rint(fmin(fmax(t, -8.0), 7.25)) + 8) << (4 * ((e & 7) >> 1) + 16 * (e & 1));
  }
  return r;
}

template <int DT>
__global__ void __launch_bounds__(THREADS, 4) append4_kernel(const __grid_constant__ Cache4Params p) {
  extern __shared__ __align__(16) uint8_t smem[];
  __shared__ Places at;
  const int64_t t0 = (int64_t)blockIdx.x * p.tile;
  const int n_tok = (int)min((int64_t)p.tile, p.tokens - t0);
  const int half = p.rot >> 1, row = pair_row(half), row_q = query_row(half);
  double2* const cs64 = reinterpret_cast<double2*>(smem);              // [tokens][row] (cos, sin) for keys, and for queries
  float2* const csq = reinterpret_cast<float2*>(cs64 + p.tile * row);
  const int h0 = blockIdx.y * p.head_group, n_heads = min(p.head_group, p.heads_all - h0);
  // a thread's token and group are the same for all its heads
  const Spot spot(p, n_tok);
  const int t = spot.t, chunk = spot.chunk, g = spot.g;
  // what the kernel in front wrote is read from here on; the one behind may be set up meanwhile (it waits in the same way)
  asm volatile("griddepcontrol.wait;" ::: "memory");
  asm volatile("griddepcontrol.launch_dependents;" ::: "memory");
  at.look_up(p, t0, n_tok, false);
  __syncthreads();
  // heads: pairs of a key and a value, then queries
  const int hk = p.st[0].heads, end = h0 + n_heads;
  const bool keys = p.rot && h0 < hk, queries = end > hk;
  for (int i = threadIdx.x; i < n_tok * half; i += THREADS) {
    const int tok = i / half, j = i - tok * half;
    const double turn = turn_of(p, t0 + tok, at.place[tok], j);
    if (keys) {
      double s, c;
      sincospi(2.0 * turn, &s, &c);
      cs64[pair_at(row, tok, j)] = make_double2(c, s);
    }
    if (queries) {
      float s, c;
      sincospif(2.0f * (float)turn, &s, &c);
      csq[pair_at(row_q, tok, j)] = make_float2(c, s);
    }
  }
  __syncthreads();

  int i = h0 + spot.head;
  if (spot.head >= spot.heads) return;
  // Sixteen elements that a thread rotates: pairs 8 u .. 8 u + 7, or, behind the rotated ones, elements 16 u .. 16 u + 15.
  struct Sixteen {
    int u, first, second;
    bool turned, halves;
    __device__ __forceinline__ Sixteen(const Cache4Params& p, int u) : u(u), turned(16 * u < p.rot), halves(turned && p.style == RG_ROPE_HALF) {
      first = halves ? 8 * u : 16 * u;
      second = halves ? (p.rot >> 1) + 8 * u : first + 8;
    }
  };
  // ---- keys and values
  const int64_t page = spot.active ? at.page[t] : -2;
  const Sixteen mine(p, 2 * chunk + g);
  const int u = mine.u, first = mine.first, second = mine.second;
  const bool turned = mine.turned, halves = mine.halves;
  const int slot = at.slot[t];
  const int64_t in_page = page * p.st[0].dst_page + (int64_t)(slot >> 3) * tile4_bytes(p.d), in_page_v = page * p.st[1].dst_page + (int64_t)(slot >> 3) * tile4_bytes(p.d);
  // the eight elements (a word) from e on in a tile, and the scale of its group
  auto word_at = [&](int e) -> int { return codes4_at(e >> 5, slot & 7) + (e >> 3 & 3) * 4; };
  auto scale_at = [&](int e) -> int { return scales4_at(p.d, e >> 5, slot & 7) + (e >> 4 & 1); };
  auto max8 = [](const float* v) -> float {                            // NaN if one is
    float m = 0.0f;
#pragma unroll
    for (int e = 0; e < 8; e += 2) m = absmax3_nan(m, v[e], v[e + 1]);
    return m;
  };
  // a whole group: elements 16 u ..
  auto put_group = [&](uint8_t* tile, const Elem<DT>* src, const auto* v, bool rotated) {
    uint32_t b;
    uint2 w;
    float amax;
    if constexpr (sizeof(*v) == 8) {
      amax = magnitude4_value(max(magnitude4(v), magnitude4(v + 8)));
      b = scale4_byte(amax);
      const double inv = inverse4(scale4(b));
      w = make_uint2(codes4(v, inv), codes4(v + 8, inv));
    } else {
      amax = absmax3_nan(0.0f, max8(v), max8(v + 8));
      b = scale4_byte(amax);
      const float inv = __frcp_rn(scale4(b));
      w = make_uint2(codes4(v, inv), codes4(v + 8, inv));
    }
    if (!(amax <= 57600.0f)) {
      const Codes c = quantise_slowly<DT>(p, src, rotated, 16 * u, 16, cs64, row, t);
      w = make_uint2(c.w[0], c.w[1]);
      b = c.b;
    }
    *reinterpret_cast<uint2*>(tile + word_at(16 * u)) = w;
    tile[scale_at(16 * u)] = (uint8_t)b;
  };
  // half a group, elements e .. e + 7; the neighbouring lane has the other half
  auto put_half = [&](uint8_t* tile, const Elem<DT>* src, const double* v, int e) {
    const uint32_t mine = magnitude4(v);
    const float amax = magnitude4_value(max(mine, __shfl_xor_sync(3u << (threadIdx.x & 30), mine, 1)));
    uint32_t b = scale4_byte(amax), w = codes4(v, inverse4(scale4(b)));
    if (!(amax <= 57600.0f)) {
      const Codes c = quantise_slowly<DT>(p, src, true, e, 8, cs64, row, t);
      w = c.w[0];
      b = c.b;
    }
    *reinterpret_cast<uint32_t*>(tile + word_at(e)) = w;
    if (!(e & 8)) tile[scale_at(e)] = (uint8_t)b;
  };
  const bool whole_eights = p.style == RG_ROPE_HALF ? p.rot % 32 == 0 : p.rot % 16 == 0;      // of the rotated elements' groups
  const int k_first = whole_eights ? first : 16 * u, k_second = whole_eights ? second : 16 * u + 8;      // 16-byte accesses reach them
  const double2* const csk = cs64 + pair_at(row, t, 8 * u);
  for (; i < min(end, hk); i += spot.heads) {
    if (page < 0) continue;                                            // no place for key and value
    const Elem<DT>* k_src = static_cast<const Elem<DT>*>(p.st[0].src) + (t0 + t) * p.st[0].src_tok + (int64_t)i * p.st[0].src_head;
    const Elem<DT>* v_src = static_cast<const Elem<DT>*>(p.st[1].src) + (t0 + t) * p.st[1].src_tok + (int64_t)i * p.st[1].src_head;
    uint8_t* const k_tile = static_cast<uint8_t*>(p.st[0].dst) + in_page + (int64_t)i * p.st[0].dst_head;
    uint8_t* const v_tile = static_cast<uint8_t*>(p.st[1].dst) + in_page_v + (int64_t)i * p.st[1].dst_head;
    const Eight<DT> ka = load8<DT>(k_src + k_first, p.st[0].vec), kb = load8<DT>(k_src + k_second, p.st[0].vec);
    const Eight<DT> va = load8<DT>(v_src + 16 * u, p.st[1].vec), vb = load8<DT>(v_src + 16 * u + 8, p.st[1].vec);
    float v[16];
    widen8<DT>(ka, v); widen8<DT>(kb, v + 8);
    if (turned || DT == RG_F32) {
      double x[16];
      if (!whole_eights && turned) {
#pragma unroll
        for (int e = 0; e < 16; ++e) x[e] = element<DT>(p, k_src, true, 16 * u + e, cs64, row, t);
      } else {
#pragma unroll
        for (int e = 0; e < 16; ++e) x[e] = (double)v[e];
        if (halves) rotate16<true>(x, csk);
        else if (turned) rotate16<false>(x, csk);
      }
      if (halves && whole_eights) {
        put_half(k_tile, k_src, x, first);
        put_half(k_tile, k_src, x + 8, second);
      } else {
        put_group(k_tile, k_src, x, turned);
      }
    } else {
      put_group(k_tile, k_src, v, false);
    }
    widen8<DT>(va, v); widen8<DT>(vb, v + 8);
    if constexpr (DT == RG_F32) {
      double x[16];
#pragma unroll
      for (int e = 0; e < 16; ++e) x[e] = (double)v[e];
      put_group(v_tile, v_src, x, false);
    } else {
      put_group(v_tile, v_src, v, false);
    }
  }

  // ---- queries, two heads at a time.  Here a head's threads run over its groups first, then over the tokens: neighbours read and write neighbouring pieces of a row
  // (10.5 k tokens with 32 heads of queries: 56 us, 63 in the keys' order).
  if (i >= end) return;
  const int r = threadIdx.x % (p.d / 16 * p.tile), tq = r / (p.d / 16);
  if (tq >= n_tok || at.page[tq] == -2) return;
  const Sixteen own(p, r % (p.d / 16));
  const Cache4Stream& st = p.st[2];
  const Elem<DT>* src = static_cast<const Elem<DT>*>(st.src) + (t0 + tq) * st.src_tok + (int64_t)(i - hk) * st.src_head;
  Elem<DT>* dst = static_cast<Elem<DT>*>(st.dst) + (t0 + tq) * st.dst_tok + (int64_t)(i - hk) * st.dst_head;
  const int64_t src_step = (int64_t)spot.heads * st.src_head, dst_step = (int64_t)spot.heads * st.dst_head;
  const float2* const cs = csq + pair_at(row_q, tq, 8 * own.u);
  if (!st.vec || p.rot % 16) {
    for (; i < end; i += spot.heads, src += src_step, dst += dst_step) rotate_query_slowly<DT>(p, src, dst, own.u, cs);
    return;
  }
  auto turn_and_put = [&](Elem<DT>* to, const Eight<DT>& a, const Eight<DT>& b) {
    float v[16];
    widen8<DT>(a, v); widen8<DT>(b, v + 8);
    if (own.halves) rotate16<true>(v, cs);
    else if (own.turned) rotate16<false>(v, cs);
    store8<DT>(to + own.first, v);
    store8<DT>(to + own.second, v + 8);
  };
  for (; i + spot.heads < end; i += 2 * spot.heads, src += 2 * src_step, dst += 2 * dst_step) {
    const Eight<DT> a0 = load8<DT>(src + own.first, true), b0 = load8<DT>(src + own.second, true), a1 = load8<DT>(src + src_step + own.first, true), b1 = load8<DT>(src + src_step + own.second, true);
    turn_and_put(dst, a0, b0);
    turn_and_put(dst + dst_step, a1, b1);
  }
  if (i < end) turn_and_put(dst, load8<DT>(src + own.first, true), load8<DT>(src + own.second, true));
}

// The other way: a thread takes a group's codes and stores 16 elements.
template <int DT>
__global__ void __launch_bounds__(THREADS) read4_kernel(const __grid_constant__ Cache4Params p) {
  __shared__ Places at;
  const int64_t t0 = (int64_t)blockIdx.x * p.tile;
  const int n_tok = (int)min((int64_t)p.tile, p.tokens - t0);
  const int h0 = blockIdx.y * p.head_group, n_heads = min(p.head_group, p.heads_all - h0);
  asm volatile("griddepcontrol.wait;" ::: "memory");
  asm volatile("griddepcontrol.launch_dependents;" ::: "memory");
  at.look_up(p, t0, n_tok, true);
  __syncthreads();
  const Spot spot(p, n_tok);
  const int t = spot.t, chunk = spot.chunk, g = spot.g;
  if (!spot.active) return;
  const int64_t page = at.page[t];
  if (page == -2) return;
  const int slot = at.slot[t], code_at = codes4_at(chunk, slot & 7) + 8 * g, scale_at = scales4_at(p.d, chunk, slot & 7) + g;
  for (int i = h0 + spot.head; i < h0 + n_heads; i += spot.heads) {
    const int k = i >= p.st[0].heads ? 1 : 0, h = i - (k ? p.st[0].heads : 0);
    const Cache4Stream& st = p.st[k];
    uint2 w = make_uint2(0x88888888u, 0x88888888u);                    // a row without a place: zeros
    uint32_t b = 0;
    if (page >= 0) {
      const uint8_t* tile = static_cast<const uint8_t*>(st.src) + page * st.dst_page + (int64_t)h * st.src_head + (int64_t)(slot >> 3) * tile4_bytes(p.d);
      w = *reinterpret_cast<const uint2*>(tile + code_at);
      b = tile[scale_at];
    }
    const float s = scale4(b);
    float v[16];
#pragma unroll
    for (int e = 0; e < 16; ++e) v[e] = f_mul((float)((int)((e < 8 ? w.x : w.y) >> (4 * ((e & 7) >> 1) + 16 * (e & 1)) & 15u) - 8), s);
    Elem<DT>* dst = static_cast<Elem<DT>*>(st.dst) + (t0 + t) * st.dst_tok + (int64_t)h * st.dst_head + 32 * chunk + 16 * g;
    if (st.vec) {
      store8<DT>(dst, v);
      store8<DT>(dst + 8, v + 8);
    } else {
#pragma unroll
      for (int e = 0; e < 16; ++e) store_scalar(dst, DT, e, v[e]);
    }
  }
}

template <typename Kernel>
cudaError_t launch(Kernel kernel, const Cache4Params& p, dim3 grid, size_t smem, cudaStream_t st) {
  cudaLaunchConfig_t cfg = {};
  cfg.gridDim = grid;
  cfg.blockDim = dim3(THREADS, 1, 1);
  cfg.dynamicSmemBytes = smem;
  cfg.stream = st;
  cudaLaunchAttribute attr[1];
  attr[0].id = cudaLaunchAttributeProgrammaticStreamSerialization;
  attr[0].val.programmaticStreamSerializationAllowed = 1;
  cfg.attrs = attr;
  cfg.numAttrs = 1;
  return cudaLaunchKernelEx(&cfg, kernel, p);
}

}  // namespace

// All arguments were validated by the caller; d a multiple of 32 up to 128, blocks and their strides multiples of 16 bytes.
rg_status_t launch_cache4(Cache4Params p, int dtype, bool read, cudaStream_t st) {
  const int es = dtype == RG_F32 ? 4 : 2;
  p.heads_all = 0;
  for (int k = 0; k < p.n_streams; ++k) {
    Cache4Stream& s = p.st[k];
    if (read || k != 1) p.heads_all += s.heads;                          // written, a key and its value go together
    // the sides that are rows
    const bool src = !read, dst = read || k == 2;
    s.vec = (!src || (reinterpret_cast<uintptr_t>(s.src) % 16 == 0 && s.src_tok * es % 16 == 0 && s.src_head * es % 16 == 0)) &&
            (!dst || (reinterpret_cast<uintptr_t>(s.dst) % 16 == 0 && s.dst_tok * es % 16 == 0 && s.dst_head * es % 16 == 0));
  }
  const int sms = current_device().sms, units = p.d / 16;
  // tokens of a CTA: a tile's slots, unless the grid does not cover the GPU then
  int64_t tile = 1;
  while (tile < TOKENS && (p.tokens + 2 * tile - 1) / (2 * tile) >= 2 * sms) tile *= 2;
  // heads of a CTA: all, unless few tokens leave SMs without work
  const int64_t tiles = (p.tokens + tile - 1) / tile;
  int groups = 1;
  while (tiles * groups < 2 * sms && groups < p.heads_all && tile * ((p.heads_all + groups - 1) / groups) * units > THREADS) ++groups;
  p.tile = (int)tile;
  p.head_group = (p.heads_all + groups - 1) / groups;
  groups = (p.heads_all + p.head_group - 1) / p.head_group;
  const dim3 grid((unsigned)tiles, (unsigned)groups, 1);
  const size_t smem = read || !p.rot ? 0 : (size_t)tile * (pair_row(p.rot / 2) * sizeof(double2) + query_row(p.rot / 2) * sizeof(float2));
  cudaError_t e;
  if (read) e = dtype == RG_F32 ? launch(read4_kernel<RG_F32>, p, grid, 0, st) : dtype == RG_F16 ? launch(read4_kernel<RG_F16>, p, grid, 0, st) : launch(read4_kernel<RG_BF16>, p, grid, 0, st);
  else e = dtype == RG_F32 ? launch(append4_kernel<RG_F32>, p, grid, smem, st) : dtype == RG_F16 ? launch(append4_kernel<RG_F16>, p, grid, smem, st) : launch(append4_kernel<RG_BF16>, p, grid, smem, st);
  return e == cudaSuccess ? RG_OK : RG_ERR_CUDA;
}

rg_status_t read_and_clear_cache4_status(uint32_t* code) {
  unsigned int v = 0, zero = 0;
  if (cudaMemcpyFromSymbol(&v, g_cache4_status_word, sizeof(v)) != cudaSuccess) return RG_ERR_CUDA;
  if (v != 0 && cudaMemcpyToSymbol(g_cache4_status_word, &zero, sizeof(zero)) != cudaSuccess) return RG_ERR_CUDA;
  *code = v;
  return v ? RG_ERR_PAGE : RG_OK;
}

}  // namespace rg

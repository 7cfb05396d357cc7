// Rows into a paged cache of four-bit codes (rg_kv_append_four), with the rotation on the way, and back out of it (rg_kv_read_four).  The format is
// rg_four_bit.cuh's.
//
// Keys are rotated in 64 bits (the pair's sine and cosine as well): a code is a step function, and an fp32 rotation, whose result is off by 2^-22 or
// so, would put one key in some hundred thousand on the other side of a border between codes; even a 64-bit one rounded to fp32 does so for one in ten
// million.  Codes are chosen in fp32; a group in which that is close (one in 30000) is done again in 64 bits.  Queries are rotated as rg_rope does it, with its bits.
//
// What bounds it: bytes for prompts, latency for single tokens.  A thread takes one group of 16 elements of one row (query, key or value) and the group
// that the rotation pairs with it: 32-byte loads, no exchange between threads, and a key's 8 code bytes and its scale byte are a thread's own.
// Threads run over two groups, then the CTA's tokens, then the chunks of the head: neighbours write the neighbouring slots of a tile.
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

// 16 elements from `src` on as fp32
template <int DT>
__device__ __forceinline__ void load16(const Elem<DT>* src, bool vec, float (&v)[16]) {
  if (vec) {
    constexpr int WORDS = DT == RG_F32 ? 16 : 8;
    uint32_t w[WORDS];
#pragma unroll
    for (int i = 0; i < WORDS / 4; ++i) {
      const uint4 x = *(reinterpret_cast<const uint4*>(src) + i);
      w[4 * i] = x.x; w[4 * i + 1] = x.y; w[4 * i + 2] = x.z; w[4 * i + 3] = x.w;
    }
#pragma unroll
    for (int i = 0; i < 16; ++i) {
      if constexpr (DT == RG_F32) v[i] = __uint_as_float(w[i]);
      else { const uint32_t h = i & 1 ? w[i / 2] >> 16 : w[i / 2] & 0xffffu; v[i] = DT == RG_F16 ? f16_bits_to_f32(h) : bf16_bits_to_f32(h); }
    }
  } else {
#pragma unroll
    for (int i = 0; i < 16; ++i) {
      if constexpr (DT == RG_F32) v[i] = src[i];
      else v[i] = DT == RG_F16 ? f16_bits_to_f32(src[i]) : bf16_bits_to_f32(src[i]);
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

// A pair's place in the CTA's tables of sines: threads that hold neighbouring groups, or one group of neighbouring tokens, read different banks (rows are
// 2 modulo 16 apart, a group's pairs one more than their count).
__device__ __forceinline__ int pair_at(int row, int t, int j, int per_group) { return t * row + j + (per_group == 16 ? j >> 4 : j >> 3); }
__host__ __device__ constexpr int pair_row(int half) { const int n = half + (half >> 3) + 1; return n + (18 - n % 16) % 16; }

// A query's 16 elements: pairs 8 u .. 8 u + 7 whole (another thread's stores must not reach them: the result may lie where the queries do), what is not
// rotated as it lies.  Element c of this order, as an element of the head.
__device__ __forceinline__ int paired(const Cache4Params& p, int c) { return c >= p.rot || p.style == RG_ROPE_PAIRS ? c : (c >> 1) + (c & 1) * (p.rot >> 1); }
template <int DT>
__device__ __forceinline__ void rotate_query(const Cache4Params& p, const Elem<DT>* src, Elem<DT>* dst, bool vec, int u, const float2* cs, int row, int t) {
  const int half = p.rot >> 1;
  const bool halves = p.style == RG_ROPE_HALF && 16 * u < p.rot, wide = vec && p.rot % 16 == 0;
  constexpr int EIGHT = DT == RG_F32 ? 2 : 1;                          // 16-byte words of 8 elements
  const int first = halves ? 8 * u : 16 * u, second = halves ? half + 8 * u : first + 8;
  float v[16];                                                         // pairs side by side
  if (wide) {
    uint32_t w[8 * EIGHT];
#pragma unroll
    for (int i = 0; i < 2 * EIGHT; ++i) {
      const uint4 x = *(reinterpret_cast<const uint4*>(src + (i < EIGHT ? first : second)) + i % EIGHT);
      w[4 * i] = x.x; w[4 * i + 1] = x.y; w[4 * i + 2] = x.z; w[4 * i + 3] = x.w;
    }
    float x[16];
#pragma unroll
    for (int i = 0; i < 16; ++i) {
      if constexpr (DT == RG_F32) x[i] = __uint_as_float(w[i]);
      else { const uint32_t h = i & 1 ? w[i / 2] >> 16 : w[i / 2] & 0xffffu; x[i] = DT == RG_F16 ? f16_bits_to_f32(h) : bf16_bits_to_f32(h); }
    }
#pragma unroll
    for (int i = 0; i < 16; ++i) v[i] = halves ? x[(i >> 1) + 8 * (i & 1)] : x[i];
  } else {
#pragma unroll
    for (int i = 0; i < 16; ++i) v[i] = load_scalar(src, DT, paired(p, 16 * u + i));
  }
#pragma unroll
  for (int e = 0; e < 8; ++e) {
    if (16 * u + 2 * e >= p.rot) break;
    const float2 w = cs[pair_at(row, t, 8 * u + e, 8)];
    const float x = v[2 * e], y = v[2 * e + 1];
    v[2 * e] = f_fma(-y, w.y, f_mul(x, w.x));
    v[2 * e + 1] = f_fma(x, w.y, f_mul(y, w.x));
  }
  if (wide) {
    float x[16];
#pragma unroll
    for (int i = 0; i < 16; ++i) x[i] = halves ? v[2 * (i & 7) + (i >> 3)] : v[i];
    store8<DT>(dst + first, x);
    store8<DT>(dst + second, x + 8);
  } else {
#pragma unroll
    for (int i = 0; i < 16; ++i) store_scalar(dst, DT, paired(p, 16 * u + i), v[i]);
  }
}

// An element of a key, rotated in 64 bits.
template <int DT>
__device__ __forceinline__ double rotated_key(const Cache4Params& p, const Elem<DT>* src, int i, const double2* cs, int row, int t) {
  const double x = (double)load_scalar(src, DT, i);
  if (i >= p.rot) return x;
  const int half = p.rot >> 1;
  const bool pairs = p.style == RG_ROPE_PAIRS, second = pairs ? i & 1 : i >= half;
  const double y = (double)load_scalar(src, DT, pairs ? i ^ 1 : second ? i - half : i + half);
  const double2 w = cs[pair_at(row, t, pairs ? i >> 1 : second ? i - half : i, pairs ? 8 : 16)];
  return __fma_rn(second ? y : -y, w.y, __dmul_rn(x, w.x));
}
// A group's codes and scale byte from there.
template <int DT>
__device__ __noinline__ uint3 quantise_in_64_bits(const Cache4Params& p, const Elem<DT>* src, int e0, const double2* cs, int row, int t) {
  double amax = 0.0;
  for (int e = 0; e < 16; ++e) amax = fmax(amax, fabs(rotated_key<DT>(p, src, e0 + e, cs, row, t)));
  uint32_t b = scale4_byte(__double2float_rn(amax));
  while (b > 0 && 7.5 * (double)scale4(b - 1) >= amax) --b;
  while (b < 255 && 7.5 * (double)scale4(b) < amax) ++b;
  const double s = (double)scale4(b);
  uint32_t w[2] = {0u, 0u};
#pragma unroll
  for (int q = 0; q < 2; ++q)
    for (int e = 0; e < 8; ++e) {
      const double x = rotated_key<DT>(p, src, e0 + 8 * q + e, cs, row, t);
      const int c = x == x ? (int)fmin(fmax(rint(x / s), -8.0), 7.0) : 0;
      w[q] |= (uint32_t)(c + 8) << (4 * (e >> 1) + 16 * (e & 1));
    }
  return make_uint3(w[0], w[1], b);
}

template <int DT>
__global__ void __launch_bounds__(THREADS) append4_kernel(const __grid_constant__ Cache4Params p) {
  extern __shared__ __align__(16) uint8_t smem[];
  __shared__ Places at;
  const int64_t t0 = (int64_t)blockIdx.x * p.tile;
  const int n_tok = (int)min((int64_t)p.tile, p.tokens - t0);
  const int half = p.rot >> 1, row = pair_row(half), per_group = p.style == RG_ROPE_HALF ? 16 : 8;      // pairs that 16 neighbouring elements belong to
  double2* cs64 = reinterpret_cast<double2*>(smem);                    // [tokens][row] (cos, sin)
  float2* cs32 = reinterpret_cast<float2*>(cs64 + p.tile * row);
  const int h0 = blockIdx.y * p.head_group, n_heads = min(p.head_group, p.heads_all - h0);
  // what the kernel in front wrote is read from here on; the one behind may be set up meanwhile (it waits in the same way)
  asm volatile("griddepcontrol.wait;" ::: "memory");
  asm volatile("griddepcontrol.launch_dependents;" ::: "memory");
  at.look_up(p, t0, n_tok, false);
  __syncthreads();
  // streams: keys, values, queries
  const bool keys = p.rot && h0 < p.st[0].heads, queries = h0 + n_heads > p.st[0].heads + p.st[1].heads;
  for (int i = threadIdx.x; i < n_tok * half; i += THREADS) {
    const int t = i / half, j = i - t * half;
    int64_t pos;
    if (p.pos) {
      const int axis = (j >= p.axis_end[0]) + (j >= p.axis_end[1]) + (j >= p.axis_end[2]);
      const int64_t k = (int64_t)axis * p.pos_ld + t0 + t;
      pos = p.pos64 ? static_cast<const int64_t*>(p.pos)[k] : (int64_t)static_cast<const int32_t*>(p.pos)[k];
    } else {
      pos = at.place[t];
    }
    const double turns = __dmul_rn(__dmul_rn((double)pos, p.inv_freq[j]), 0x1.45f306dc9c883p-3);      // 1 / (2 pi)
    const double part = turns - rint(turns);
    if (keys) {
      double s, c;
      sincospi(2.0 * part, &s, &c);
      cs64[pair_at(row, t, j, per_group)] = make_double2(c, s);
    }
    if (queries) {
      float s, c;
      sincospif(2.0f * (float)part, &s, &c);
      cs32[pair_at(row, t, j, 8)] = make_float2(c, s);
    }
  }
  __syncthreads();

  const int chunks = p.d / 32, per_chunk = 2 * n_tok, per_head = chunks * per_chunk, all = n_heads * per_head;
  for (int i = threadIdx.x; i < all; i += THREADS) {
    int h = h0 + i / per_head, r = i % per_head;
    const int chunk = r / per_chunk;
    r -= chunk * per_chunk;
    const int t = r >> 1, e0 = 32 * chunk + 16 * (r & 1);              // first element of the thread's group
    int k = 0;
    if (h >= p.st[0].heads) { h -= p.st[0].heads; k = 1; }
    if (k == 1 && h >= p.st[1].heads) { h -= p.st[1].heads; k = 2; }
    const Cache4Stream& st = p.st[k];
    const int64_t page = at.page[t];
    if (page == -2 || (k < 2 && page < 0)) continue;
    const Elem<DT>* src = static_cast<const Elem<DT>*>(st.src) + (t0 + t) * st.src_tok + (int64_t)h * st.src_head;
    if (k == 2) {
      rotate_query<DT>(p, src, static_cast<Elem<DT>*>(st.dst) + (t0 + t) * st.dst_tok + (int64_t)h * st.dst_head, st.vec, e0 >> 4, cs32, row, t);
      continue;
    }
    float v[16];
    load16<DT>(src + e0, st.vec, v);
    if (k == 0 && e0 < p.rot) {
      float y[16];                                                     // each element's partner
      if (p.style == RG_ROPE_PAIRS) {
#pragma unroll
        for (int e = 0; e < 16; ++e) y[e] = v[e ^ 1];
      } else if (half % 16 == 0) {
        load16<DT>(src + (e0 < half ? e0 + half : e0 - half), st.vec, y);
      } else {
#pragma unroll
        for (int e = 0; e < 16; ++e) {
          const int i = e0 + e;
          y[e] = i < p.rot ? load_scalar(src, DT, i < half ? i + half : i - half) : 0.0f;
        }
      }
#pragma unroll
      for (int e = 0; e < 16; ++e) {
        const int i = e0 + e;
        if (i >= p.rot) break;
        const bool second = p.style == RG_ROPE_PAIRS ? e & 1 : i >= half;
        const int j = p.style == RG_ROPE_PAIRS ? i >> 1 : second ? i - half : i;
        const double2 w = cs64[pair_at(row, t, j, per_group)];
        v[e] = __double2float_rn(__fma_rn((double)(second ? y[e] : -y[e]), w.y, __dmul_rn((double)v[e], w.x)));
      }
    }
    float amax = 0.0f;
#pragma unroll
    for (int e = 0; e < 16; ++e) amax = fmaxf(amax, fabsf(v[e]));
    uint32_t b = scale4_byte(amax);
    const float s = scale4(b), inv = __frcp_rn(s);
    uint32_t w[2];
    bool near = scale4_near(amax);
#pragma unroll
    for (int q = 0; q < 2; ++q) {
      w[q] = 0;
#pragma unroll
      for (int e = 0; e < 8; ++e) w[q] |= code4(v[8 * q + e], s, inv, near) << (4 * (e >> 1) + 16 * (e & 1));
    }
    if (near && k == 0 && e0 < p.rot) {
      const uint3 exact = quantise_in_64_bits<DT>(p, src, e0, cs64, row, t);
      w[0] = exact.x; w[1] = exact.y; b = exact.z;
    }
    const int slot = at.slot[t];
    uint8_t* tile = static_cast<uint8_t*>(st.dst) + page * st.dst_page + (int64_t)h * st.dst_head + (int64_t)(slot >> 3) * tile4_bytes(p.d);
    *reinterpret_cast<uint2*>(tile + codes4_at(chunk, slot & 7) + 8 * (r & 1)) = make_uint2(w[0], w[1]);
    tile[scales4_at(p.d, chunk, slot & 7) + (r & 1)] = (uint8_t)b;
  }
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
  const int chunks = p.d / 32, per_chunk = 2 * n_tok, per_head = chunks * per_chunk, all = n_heads * per_head;
  for (int i = threadIdx.x; i < all; i += THREADS) {
    int h = h0 + i / per_head, r = i % per_head;
    const int chunk = r / per_chunk;
    r -= chunk * per_chunk;
    const int t = r >> 1, k = h >= p.st[0].heads ? 1 : 0;
    h -= k ? p.st[0].heads : 0;
    const Cache4Stream& st = p.st[k];
    const int64_t page = at.page[t];
    if (page == -2) continue;
    uint2 w = make_uint2(0x88888888u, 0x88888888u);                    // a row without a place: zeros
    uint32_t b = 0;
    if (page >= 0) {
      const int slot = at.slot[t];
      const uint8_t* tile = static_cast<const uint8_t*>(st.src) + page * st.dst_page + (int64_t)h * st.src_head + (int64_t)(slot >> 3) * tile4_bytes(p.d);
      w = *reinterpret_cast<const uint2*>(tile + codes4_at(chunk, slot & 7) + 8 * (r & 1));
      b = tile[scales4_at(p.d, chunk, slot & 7) + (r & 1)];
    }
    const float s = scale4(b);
    float v[16];
#pragma unroll
    for (int e = 0; e < 16; ++e) v[e] = f_mul((float)((int)((e < 8 ? w.x : w.y) >> (4 * ((e & 7) >> 1) + 16 * (e & 1)) & 15u) - 8), s);
    Elem<DT>* dst = static_cast<Elem<DT>*>(st.dst) + (t0 + t) * st.dst_tok + (int64_t)h * st.dst_head + 32 * chunk + 16 * (r & 1);
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
    p.heads_all += s.heads;
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
  const size_t smem = read || !p.rot ? 0 : (size_t)tile * pair_row(p.rot / 2) * (sizeof(double2) + sizeof(float2));
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

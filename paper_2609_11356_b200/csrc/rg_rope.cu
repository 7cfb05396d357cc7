// Rotary positions with several axes, alone (rg_rope) and on the way into a paged cache (rg_kv_append).
//
//   angle(t, j) = pos[axis(j)][t] * inv_freq[j]
//   a' = a cos - b sin,  b' = b cos + a sin           for the two elements (a, b) of pair j
//
// The angle is formed in 64 bits and reduced to a fraction of a turn there (a position of a million leaves an fp32
// product no bits of the angle); sine and cosine of that fraction and the rotation are fp32, with one rounding to the
// output type.  The transpose of a rotation is the rotation by the negative angle: the gradient is the same kernel.
//
// What bounds it: bytes.  A CTA takes a few tokens and a group of heads; sine and cosine of a token's pairs are
// computed once per CTA into shared memory (about 100 instructions for each pair, against all heads that use it) and
// every thread then moves 2 * VEC elements of one head at a time with 16-byte accesses.  One launch rotates the
// queries, rotates the keys into their pages and copies the values into theirs.
#include "rg_common.cuh"
#include "rg_internal.h"

namespace rg {

__device__ unsigned int g_paged_status_word = 0;

namespace {

constexpr int ROPE_THREADS = 256;
constexpr int ROPE_TOKENS = ROPE_THREADS / 32;         // most tokens of a CTA: one warp looks up each one's place

// VEC elements as fp32, and back with one rounding each
template <int DT, int VEC>
struct Pack;
template <int DT>
struct Pack<DT, 1> {
  using Raw = typename std::conditional<DT == RG_F32, uint32_t, uint16_t>::type;
  static __device__ __forceinline__ void get(const Raw& r, float (&v)[1]) {
    v[0] = DT == RG_F32 ? __uint_as_float((uint32_t)r) : DT == RG_F16 ? f16_bits_to_f32(r) : bf16_bits_to_f32(r);
  }
  static __device__ __forceinline__ Raw put(const float (&v)[1]) {
    if (DT == RG_F32) return (Raw)__float_as_uint(v[0]);
    if (DT == RG_F16) return (Raw)__half_as_ushort(__float2half_rn(v[0]));
    return (Raw)__bfloat16_as_ushort(__float2bfloat16_rn(v[0]));
  }
};
template <int DT, int WORDS>
__device__ __forceinline__ void words_get(const uint32_t (&w)[WORDS], float* v) {
#pragma unroll
  for (int i = 0; i < WORDS; ++i) {
    if (DT == RG_F32) v[i] = __uint_as_float(w[i]);
    else {
      v[2 * i] = DT == RG_F16 ? f16_bits_to_f32(w[i] & 0xffffu) : bf16_bits_to_f32(w[i] & 0xffffu);
      v[2 * i + 1] = DT == RG_F16 ? f16_bits_to_f32(w[i] >> 16) : bf16_bits_to_f32(w[i] >> 16);
    }
  }
}
template <int DT, int WORDS>
__device__ __forceinline__ void words_put(uint32_t (&w)[WORDS], const float* v) {
#pragma unroll
  for (int i = 0; i < WORDS; ++i) w[i] = DT == RG_F32 ? __float_as_uint(v[i]) : pack_16x2(v[2 * i], v[2 * i + 1], DT);
}
template <int DT>
struct Pack<DT, 8> {                                    // 16-bit types
  using Raw = uint4;
  static __device__ __forceinline__ void get(const Raw& r, float (&v)[8]) { const uint32_t w[4] = {r.x, r.y, r.z, r.w}; words_get<DT, 4>(w, v); }
  static __device__ __forceinline__ Raw put(const float (&v)[8]) { uint32_t w[4]; words_put<DT, 4>(w, v); return make_uint4(w[0], w[1], w[2], w[3]); }
};
template <int DT>
struct Pack<DT, 4> {
  using Raw = typename std::conditional<DT == RG_F32, uint4, uint2>::type;
  static __device__ __forceinline__ void get(const uint4& r, float (&v)[4]) { const uint32_t w[4] = {r.x, r.y, r.z, r.w}; words_get<RG_F32, 4>(w, v); }
  static __device__ __forceinline__ void get(const uint2& r, float (&v)[4]) { const uint32_t w[2] = {r.x, r.y}; words_get<DT, 2>(w, v); }
  static __device__ __forceinline__ Raw put(const float (&v)[4]) { Raw r; put_to(r, v); return r; }
  static __device__ __forceinline__ void put_to(uint4& r, const float (&v)[4]) { uint32_t w[4]; words_put<RG_F32, 4>(w, v); r = make_uint4(w[0], w[1], w[2], w[3]); }
  static __device__ __forceinline__ void put_to(uint2& r, const float (&v)[4]) { uint32_t w[2]; words_put<DT, 2>(w, v); r = make_uint2(w[0], w[1]); }
};

// Which sequence a row belongs to and its place there; the whole warp calls.  The count of sequences that end at or
// before the row is its sequence (lengths of zero included), whatever the order of the additions.
__device__ __forceinline__ bool place_of(const RopeParams& p, int64_t t, int& seq, int64_t& place) {
  const int lane = threadIdx.x & 31;
  int before = 0;
  for (int i = lane; i < p.n_seqs; i += 32) before += p.cu_q[i + 1] <= t ? 1 : 0;
  seq = __reduce_add_sync(0xffffffffu, before);
  if (seq >= p.n_seqs) return false;                    // a row behind the last sequence
  if (t < p.cu_q[seq]) return false;
  place = (int64_t)p.seq_lens[seq] - ((int64_t)p.cu_q[seq + 1] - t);
  return true;
}

template <int DT, int VEC, bool PAGED>
__global__ void __launch_bounds__(ROPE_THREADS) rope_kernel(const __grid_constant__ RopeParams p) {
  using P = Pack<DT, VEC>;
  using Raw = typename P::Raw;
  constexpr int ES = DT == RG_F32 ? 4 : 2;
  extern __shared__ float2 cs[];                        // [tokens of the CTA][rot / 2] (cos, sin)
  __shared__ int64_t s_page[ROPE_TOKENS];               // page of the token's slot; -1: no place for its key and value; -2: not a row at all
  __shared__ int32_t s_slot[ROPE_TOKENS];
  __shared__ int64_t s_pos[ROPE_TOKENS];
  const int64_t t0 = (int64_t)blockIdx.x * p.tile;
  const int n_tok = (int)min((int64_t)p.tile, p.tokens - t0);
  const int half = p.rot >> 1;
  if (PAGED) {
    const int w = threadIdx.x >> 5;
    if (w < n_tok) {
      int seq;
      int64_t place = 0, page = -2;
      if (place_of(p, t0 + w, seq, place)) {
        page = -1;
        if (place >= 0 && place < (int64_t)p.table_cols * p.page_size) {
          const int64_t id = p.table[(int64_t)seq * p.table_ld + place / p.page_size];
          if (id >= 0 && id < p.pages) page = id;
        }
        if (page < 0 && (threadIdx.x & 31) == 0) atomicCAS(&g_paged_status_word, 0u, (unsigned)RG_PAGE_CODE_APPEND);
      }
      if ((threadIdx.x & 31) == 0) { s_page[w] = page; s_slot[w] = (int32_t)(place >= 0 ? place % p.page_size : 0); s_pos[w] = place; }
    }
    __syncthreads();
  }
  for (int i = threadIdx.x; i < n_tok * half; i += ROPE_THREADS) {
    const int t = i / half, j = i - t * half;
    int64_t at;
    if (p.pos) {
      const int axis = (j >= p.axis_end[0]) + (j >= p.axis_end[1]) + (j >= p.axis_end[2]);
      const int64_t k = (int64_t)axis * p.pos_ld + t0 + t;
      at = p.pos64 ? static_cast<const int64_t*>(p.pos)[k] : (int64_t)static_cast<const int32_t*>(p.pos)[k];
    } else {
      at = s_pos[t];
    }
    const double turns = __dmul_rn(__dmul_rn((double)at, p.inv_freq[j]), 0x1.45f306dc9c883p-3);      // 1 / (2 pi)
    const float frac = (float)(turns - rint(turns));
    float s, c;
    sincospif(2.0f * frac, &s, &c);
    cs[i] = make_float2(c, p.inverse ? -s : s);
  }
  __syncthreads();

  const int h0 = blockIdx.y * p.head_group, n_heads = min(p.head_group, p.heads_all - h0);
  const int units = p.d / (2 * VEC), turned = half / VEC;   // a unit is 2 * VEC elements of one head
  const int per_tok = n_heads * units;
  for (int i = threadIdx.x; i < n_tok * per_tok; i += ROPE_THREADS) {
    const int t = i / per_tok, r = i - t * per_tok;
    int h = r / units;
    const int u = r - h * units;
    h += h0;
    int k = 0;
    if (PAGED) {
      if (h >= p.st[0].heads) { h -= p.st[0].heads; k = 1; }
      if (k == 1 && h >= p.st[1].heads) { h -= p.st[1].heads; k = 2; }
    }
    const RopeStream& st = p.st[k];
    const char* src = static_cast<const char*>(st.src) + ((t0 + t) * st.src_tok + h * st.src_head) * ES;
    char* dst = static_cast<char*>(st.dst) + h * st.dst_head * ES;
    if (PAGED) {
      const int64_t page = s_page[t];
      if (page == -2 || (st.paged && page < 0)) continue;
      dst += st.paged ? (page * st.dst_page + s_slot[t] * st.dst_tok) * ES : (t0 + t) * st.dst_tok * ES;
    } else {
      dst += (t0 + t) * st.dst_tok * ES;
    }
    // element offsets of the unit's two vectors
    int ea, eb;
    const bool turn = u < turned && st.rotate;
    if (turn && p.style == RG_ROPE_HALF) { ea = u * VEC; eb = half + u * VEC; }
    else { ea = 2 * u * VEC; eb = ea + VEC; }
    Raw ra = *reinterpret_cast<const Raw*>(src + ea * ES), rb = *reinterpret_cast<const Raw*>(src + eb * ES);
    if (turn) {
      const float2* f = cs + t * half + u * VEC;
      float a[VEC], b[VEC];
      P::get(ra, a); P::get(rb, b);
      if (p.style == RG_ROPE_HALF || VEC == 1) {
#pragma unroll
        for (int e = 0; e < VEC; ++e) {
          const float2 w = f[e];
          const float x = a[e], y = b[e];
          a[e] = f_fma(-y, w.y, f_mul(x, w.x));
          b[e] = f_fma(x, w.y, f_mul(y, w.x));
        }
      } else {
        constexpr int H = VEC > 1 ? VEC / 2 : 1;
        float v[2 * VEC];
#pragma unroll
        for (int e = 0; e < VEC; ++e) { v[e] = a[e]; v[VEC + e] = b[e]; }
#pragma unroll
        for (int e = 0; e < 2 * H; ++e) {
          const float2 w = f[e];
          const float x = v[2 * e], y = v[2 * e + 1];
          v[2 * e] = f_fma(-y, w.y, f_mul(x, w.x));
          v[2 * e + 1] = f_fma(x, w.y, f_mul(y, w.x));
        }
#pragma unroll
        for (int e = 0; e < VEC; ++e) { a[e] = v[e]; b[e] = v[VEC + e]; }
      }
      ra = P::put(a); rb = P::put(b);
    }
    *reinterpret_cast<Raw*>(dst + ea * ES) = ra;
    *reinterpret_cast<Raw*>(dst + eb * ES) = rb;
  }
}

template <int DT, int VEC>
cudaError_t launch(const RopeParams& p, dim3 grid, size_t smem, bool paged, cudaStream_t st) {
  if (paged) rope_kernel<DT, VEC, true><<<grid, ROPE_THREADS, smem, st>>>(p);
  else rope_kernel<DT, VEC, false><<<grid, ROPE_THREADS, smem, st>>>(p);
  return cudaGetLastError();
}

}  // namespace

// All arguments were validated by the caller; rot <= 512, d even, every stream's last dimension contiguous.
rg_status_t launch_rope(RopeParams p, int dtype, bool paged, cudaStream_t st) {
  const int es = dtype == RG_F32 ? 4 : 2;
  // the widest vector that divides both parts of a head in twos and that every address allows
  int vec = 16 / es;
  auto fits = [&](int v) {
    const int64_t bytes = (int64_t)v * es;
    const int half = p.rot / 2;
    if (half % v || (p.d - p.rot) % (2 * v)) return false;
    if (p.d % (2 * v)) return false;
    for (int k = 0; k < p.n_streams; ++k) {
      const RopeStream& s = p.st[k];
      const int64_t all[] = {s.src_tok, s.src_head, s.dst_tok, s.dst_head, s.dst_page};
      for (int64_t x : all) if ((x * es) % bytes) return false;
      if (reinterpret_cast<uintptr_t>(s.src) % bytes || reinterpret_cast<uintptr_t>(s.dst) % bytes) return false;
    }
    return true;
  };
  while (vec > 1 && !fits(vec)) vec = vec > 4 ? 4 : 1;
  p.heads_all = 0;
  for (int k = 0; k < p.n_streams; ++k) p.heads_all += p.st[k].heads;
  const int units = p.d / (2 * vec);
  const int sms = current_device().sms;
  // tokens of a CTA: as many as give each thread a few units, while the grid still covers the GPU
  int64_t tile = 1;
  while (tile < ROPE_TOKENS && tile * p.heads_all * units < 4 * ROPE_THREADS && (p.tokens + 2 * tile - 1) / (2 * tile) >= 4 * sms) tile *= 2;
  // few tokens: their heads are dealt to several CTAs, one unit a thread
  int groups = 1;
  const int64_t tiles = (p.tokens + tile - 1) / tile;
  while (tiles * groups < 2 * sms && groups < p.heads_all && tile * ((p.heads_all + groups - 1) / groups) * units > ROPE_THREADS) ++groups;
  p.tile = (int)tile;
  p.head_group = (p.heads_all + groups - 1) / groups;
  groups = (p.heads_all + p.head_group - 1) / p.head_group;
  const dim3 grid((unsigned)tiles, (unsigned)groups, 1);
  const size_t smem = (size_t)tile * (p.rot / 2) * sizeof(float2);
  cudaError_t e;
  if (dtype == RG_F32) e = vec == 4 ? launch<RG_F32, 4>(p, grid, smem, paged, st) : launch<RG_F32, 1>(p, grid, smem, paged, st);
  else if (dtype == RG_F16) e = vec == 8 ? launch<RG_F16, 8>(p, grid, smem, paged, st) : vec == 4 ? launch<RG_F16, 4>(p, grid, smem, paged, st) : launch<RG_F16, 1>(p, grid, smem, paged, st);
  else e = vec == 8 ? launch<RG_BF16, 8>(p, grid, smem, paged, st) : vec == 4 ? launch<RG_BF16, 4>(p, grid, smem, paged, st) : launch<RG_BF16, 1>(p, grid, smem, paged, st);
  return e == cudaSuccess ? RG_OK : RG_ERR_CUDA;
}

rg_status_t read_and_clear_paged_status(uint32_t* code) {
  unsigned int v = 0, zero = 0;
  if (cudaMemcpyFromSymbol(&v, g_paged_status_word, sizeof(v)) != cudaSuccess) return RG_ERR_CUDA;
  if (v != 0 && cudaMemcpyToSymbol(g_paged_status_word, &zero, sizeof(zero)) != cudaSuccess) return RG_ERR_CUDA;
  if (code) *code = v;
  return v ? RG_ERR_PAGE : RG_OK;
}

}  // namespace rg

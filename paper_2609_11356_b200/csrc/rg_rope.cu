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
#include <algorithm>
#include <type_traits>

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

// Units a thread has in flight before the CTA works out its angles.  Alone the rotation gains by four (8192 tokens of 32 heads of 128, 134 MB:
// 28 -> 24 us on the device, 5.6 TB/s; 25.7 called on rotating inputs).  With the cache (three sets of strides, places to look up) the registers they take cost more than they bring (257 MB: 49 us
// without, 54 with, on the device); there more CTAs at once do it.
template <bool PAGED> constexpr int BATCH = PAGED ? 1 : 4;
constexpr int PAGED_UNITS = 8;                         // units of a thread with the cache, one after the other (257 MB: 48 us with four, 46.7 with eight)

template <int DT, int VEC, bool PAGED>
__global__ void __launch_bounds__(ROPE_THREADS, PAGED ? 6 : 4) rope_kernel(const __grid_constant__ RopeParams p) {
  using P = Pack<DT, VEC>;
  using Raw = typename P::Raw;
  constexpr int ES = DT == RG_F32 ? 4 : 2, FLY = BATCH<PAGED>;
  extern __shared__ __align__(16) float2 cs[];                        // [tokens of the CTA][rot / 2] (cos, sin)
  __shared__ int64_t s_page[ROPE_TOKENS];               // page of the token's slot; -1: no place for its key and value; -2: not a row at all
  __shared__ int32_t s_slot[ROPE_TOKENS];
  __shared__ int64_t s_pos[ROPE_TOKENS];
  const int64_t t0 = (int64_t)blockIdx.x * p.tile;
  const int n_tok = (int)min((int64_t)p.tile, p.tokens - t0);
  const int half = p.rot >> 1;
  const int h0 = blockIdx.y * p.head_group, n_heads = min(p.head_group, p.heads_all - h0);
  const int units = p.d / (2 * VEC), turned = half / VEC;   // a unit is 2 * VEC elements of one head
  const int per_tok = p.head_group * units, all = n_tok * per_tok;      // the last group of heads may be short: its missing heads are passed over

  // the i-th unit of the CTA: token, stream, head, unit of the head
  auto find = [&](int i, int& t, int& k, int& h, int& u) -> bool {
    t = p.inv_per_tok ? (int)__umulhi((uint32_t)i, p.inv_per_tok) : i;      // exact divisions: dividend times divisor stays below 2^32; 0: by one
    const int r = i - t * per_tok;
    h = p.inv_units ? (int)__umulhi((uint32_t)r, p.inv_units) : r;
    u = r - h * units;
    if (h >= n_heads) return false;
    h += h0;
    k = 0;
    if (PAGED) {
      if (h >= p.st[0].heads) { h -= p.st[0].heads; k = 1; }
      if (k == 1 && h >= p.st[1].heads) { h -= p.st[1].heads; k = 2; }
    }
    return true;
  };
  // Where pair j's cosine and sine lie in the token's row: units side by side, so that the lanes of a warp, which hold neighbouring units, read
  // neighbouring words (pair by pair they would read every 64th byte: four-way bank conflicts took a third of the time).
  auto spot = [&](int j) -> int { return VEC == 1 ? j : ((j % VEC >> 1) * turned + j / VEC) * 2 + (j & 1); };
  // element offsets of a unit's two vectors
  auto offsets = [&](bool turn, int u, int& ea, int& eb) {
    if (turn && p.style == RG_ROPE_HALF) { ea = u * VEC; eb = half + u * VEC; }
    else { ea = 2 * u * VEC; eb = ea + VEC; }
  };
  Raw ra[FLY], rb[FLY];
  auto load = [&](int first) {
#pragma unroll
    for (int q = 0; q < FLY; ++q) {
      const int i = first + q * ROPE_THREADS;
      if (i >= all) break;
      int t, k, h, u, ea, eb;
      if (!find(i, t, k, h, u)) continue;
      const RopeStream& st = p.st[k];
      offsets(u < turned && st.rotate, u, ea, eb);
      const char* src = static_cast<const char*>(st.src) + ((t0 + t) * st.src_tok + h * st.src_head) * ES;
      ra[q] = *reinterpret_cast<const Raw*>(src + ea * ES);
      rb[q] = *reinterpret_cast<const Raw*>(src + eb * ES);
    }
  };
  // what the kernel in front wrote is read from here on; the one behind may be set up meanwhile (it waits in the same way)
  asm volatile("griddepcontrol.wait;" ::: "memory");
  asm volatile("griddepcontrol.launch_dependents;" ::: "memory");
  if (!PAGED) load(threadIdx.x);                        // on their way while the angles are worked out

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
    cs[t * half + spot(j)] = make_float2(c, p.inverse ? -s : s);
  }
  __syncthreads();

  for (int first = threadIdx.x; first < all; first += FLY * ROPE_THREADS) {
    if (PAGED || first != threadIdx.x) load(first);
#pragma unroll
    for (int q = 0; q < FLY; ++q) {
      const int i = first + q * ROPE_THREADS;
      if (i >= all) break;
      int t, k, h, u, ea, eb;
      if (!find(i, t, k, h, u)) continue;
      const RopeStream& st = p.st[k];
      const bool turn = u < turned && st.rotate;
      offsets(turn, u, ea, eb);
      char* dst = static_cast<char*>(st.dst) + h * st.dst_head * ES;
      if (PAGED) {
        const int64_t page = s_page[t];
        if (page == -2 || (st.paged && page < 0)) continue;
        dst += st.paged ? (page * st.dst_page + s_slot[t] * st.dst_tok) * ES : (t0 + t) * st.dst_tok * ES;
      } else {
        dst += (t0 + t) * st.dst_tok * ES;
      }
      Raw wa = ra[q], wb = rb[q];
      if (turn) {
        float2 f[VEC];
        if constexpr (VEC == 1) {
          f[0] = cs[t * half + u];
        } else {
#pragma unroll
          for (int e = 0; e < VEC; e += 2) {
            const float4 w = *reinterpret_cast<const float4*>(cs + t * half + ((e >> 1) * turned + u) * 2);
            f[e] = make_float2(w.x, w.y);
            f[e + 1 < VEC ? e + 1 : e] = make_float2(w.z, w.w);
          }
        }
        float v[2 * VEC];
        {
          float a[VEC], b[VEC];
          P::get(wa, a); P::get(wb, b);
#pragma unroll
          for (int e = 0; e < VEC; ++e) { v[e] = a[e]; v[VEC + e] = b[e]; }
        }
        // pair e of the unit: elements e and VEC + e, or the neighbours 2e and 2e + 1
        if (p.style == RG_ROPE_HALF || VEC == 1) {
#pragma unroll
          for (int e = 0; e < VEC; ++e) {
            const float2 w = f[e];
            const float x = v[e], y = v[VEC + e];
            v[e] = f_fma(-y, w.y, f_mul(x, w.x));
            v[VEC + e] = f_fma(x, w.y, f_mul(y, w.x));
          }
        } else {
#pragma unroll
          for (int e = 0; e < VEC; ++e) {
            const float2 w = f[e];
            const float x = v[2 * e], y = v[2 * e + 1];
            v[2 * e] = f_fma(-y, w.y, f_mul(x, w.x));
            v[2 * e + 1] = f_fma(x, w.y, f_mul(y, w.x));
          }
        }
        float a[VEC], b[VEC];
#pragma unroll
        for (int e = 0; e < VEC; ++e) { a[e] = v[e]; b[e] = v[VEC + e]; }
        wa = P::put(a); wb = P::put(b);
      }
      *reinterpret_cast<Raw*>(dst + ea * ES) = wa;
      *reinterpret_cast<Raw*>(dst + eb * ES) = wb;
    }
  }
}

template <int DT, int VEC>
cudaError_t launch(const RopeParams& p, dim3 grid, size_t smem, bool paged, cudaStream_t st) {
  cudaLaunchConfig_t cfg = {};
  cfg.gridDim = grid;
  cfg.blockDim = dim3(ROPE_THREADS, 1, 1);
  cfg.dynamicSmemBytes = smem;
  cfg.stream = st;
  cudaLaunchAttribute attr[1];
  attr[0].id = cudaLaunchAttributeProgrammaticStreamSerialization;
  attr[0].val.programmaticStreamSerializationAllowed = 1;
  cfg.attrs = attr;
  cfg.numAttrs = 1;
  return cudaLaunchKernelEx(&cfg, paged ? rope_kernel<DT, VEC, true> : rope_kernel<DT, VEC, false>, p);
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
  // tokens of a CTA: as many as give a thread its units, while the grid still covers the GPU
  int64_t tile = 1;
  while (tile < ROPE_TOKENS && 2 * tile * p.heads_all * units <= (paged ? PAGED_UNITS : BATCH<false>) * ROPE_THREADS && (p.tokens + 2 * tile - 1) / (2 * tile) >= 4 * sms) tile *= 2;
  // heads of a CTA: all, unless few tokens leave SMs without work; at most 8192 units a token keep the kernel's divisions exact
  const int64_t tiles = (p.tokens + tile - 1) / tile;
  int groups = (int)(((int64_t)p.heads_all * units + 8191) / 8192);
  while (tiles * groups < 2 * sms && groups < p.heads_all && tile * ((p.heads_all + groups - 1) / groups) * units > ROPE_THREADS) ++groups;
  p.tile = (int)tile;
  p.head_group = (p.heads_all + groups - 1) / groups;
  groups = (p.heads_all + p.head_group - 1) / p.head_group;
  auto inverse = [](uint32_t n) { return n > 1 ? (uint32_t)((uint64_t(1) << 32) / n + 1) : 0u; };
  p.inv_units = inverse(units);
  p.inv_per_tok = inverse((uint32_t)p.head_group * units);
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

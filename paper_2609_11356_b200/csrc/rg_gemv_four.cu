// Products of a few rows with weights held in four bits (rg_gemv_four):
//   C[m][n] = epilogue( sum over groups G of scale[n][G] * ( sum over k in G of A[m][k] (u[n][k] - z[n][G]) ) )
//
// The inner sum is a chain of 16-wide tensor-core steps from a zero accumulator: u - z is an integer of at most four bits and a sign, exact in bf16 and
// fp16, so nothing is rounded before the products' fp32 sum.  The scale multiplies a finished group once, in fp32 (fused, onto the running sum of a part of
// K): no weight is ever narrowed, whatever the scales' type.  A part is a run of whole 256-wide stages, at most eight of them over K; parts are added in
// ascending order.  The cut follows from K alone and an accumulator's column is one row of A, so a row's bits do not depend on M.
//
// What bounds it: the bytes of the codes, and next the instructions that unpack them (1.4 a code and lane: a mask that makes a float's mantissa of the nibble,
// and one subtraction, for two codes).  Weights are the 16 rows of mma.sync's first operand, read straight from the natural order of the codes: a warp's
// lanes hold whole words of eight codes, and the order of k within a group is the tensor core's own affair as long as A's elements follow it.
// tcgen05 would want the unpacked weights in shared or tensor memory, a trip that costs more than these few rows' products.
// A tile is 16 MT rows of weights; one to eight warps share it, each with one or more parts of K, and every warp streams its own stages into shared memory, a
// TMA box at a time.
#include <cuda.h>

#include <algorithm>
#include <type_traits>

#include "rg_common.cuh"
#include "rg_internal.h"
#include "rg_ptx.cuh"

namespace rg {

__device__ unsigned int g_gemv_four_status_word = 0;      // waits that gave up

namespace {

constexpr int PARTS = 8;                               // most parts of K
constexpr int SPAN = 256;                              // k of a stage: 128 bytes a row of weights

struct W4Params {
  const void* scales;
  const uint8_t* zeros;
  const uint16_t* A;
  void* C;
  int64_t scale_ld, zero_ld, lda, ldc;
  int32_t M, N, K, groups;
  int32_t scale_dtype, c_dtype, w_static;
  int32_t part;                                        // stages of a part
  int32_t rows;                                        // of A, for one CTA
  int32_t wpt, per_cta;                                // warps of a tile (a power of two up to PARTS), tiles of a CTA
  EpilogueArgs epi;
};

template <bool F16>
__device__ __forceinline__ uint32_t add2(uint32_t a, uint32_t b) {
  uint32_t d;
  if (F16) asm("add.rn.f16x2 %0, %1, %2;" : "=r"(d) : "r"(a), "r"(b));
  else asm("add.rn.bf16x2 %0, %1, %2;" : "=r"(d) : "r"(a), "r"(b));
  return d;
}
// d = a b + c, or a b
template <bool F16, bool FIRST>
__device__ __forceinline__ void mma16(float (&c)[4], uint32_t a0, uint32_t a1, uint32_t a2, uint32_t a3, uint32_t b0, uint32_t b1) {
  const float z0 = FIRST ? 0.0f : c[0], z1 = FIRST ? 0.0f : c[1], z2 = FIRST ? 0.0f : c[2], z3 = FIRST ? 0.0f : c[3];
  if (F16)
    asm volatile("mma.sync.aligned.m16n8k16.row.col.f32.f16.f16.f32 {%0, %1, %2, %3}, {%4, %5, %6, %7}, {%8, %9}, {%10, %11, %12, %13};"
                 : "=f"(c[0]), "=f"(c[1]), "=f"(c[2]), "=f"(c[3]) : "r"(a0), "r"(a1), "r"(a2), "r"(a3), "r"(b0), "r"(b1), "f"(z0), "f"(z1), "f"(z2), "f"(z3));
  else
    asm volatile("mma.sync.aligned.m16n8k16.row.col.f32.bf16.bf16.f32 {%0, %1, %2, %3}, {%4, %5, %6, %7}, {%8, %9}, {%10, %11, %12, %13};"
                 : "=f"(c[0]), "=f"(c[1]), "=f"(c[2]), "=f"(c[3]) : "r"(a0), "r"(a1), "r"(a2), "r"(a3), "r"(b0), "r"(b1), "f"(z0), "f"(z1), "f"(z2), "f"(z3));
}
// Codes i and i + 4 of a word in the halves of a word, less the zero point: the mask puts them into the mantissa of 128 (bf16) or 1024 (fp16), and
// `less` is -(128 + z) or -(1024 + z) twice.
// One operation masks and sets: with both constants in registers, which the compiler would not choose by itself.
template <bool F16, int I>
__device__ __forceinline__ uint32_t unpack(uint32_t w, uint32_t mask, uint32_t magic, uint32_t less) {
  uint32_t x;
  asm("lop3.b32 %0, %1, %2, %3, 0xea;" : "=r"(x) : "r"(w >> (4 * I)), "r"(mask), "r"(magic));      // (w & mask) | magic
  return add2<F16>(x, less);
}

constexpr int STAGE = 16 * 128;                        // bytes of a stage's codes for 16 rows
template <int GROUP> constexpr int PER = SPAN / GROUP;                 // groups of a stage

template <int GROUP, int MT, int NT, int WARPS>
struct Shape4 {
  static constexpr int ROWS = 8 * NT, COLS = 16 * MT, DEPTH = MT == 1 ? 4 : 2;       // stages of a warp's ring, one being worked on
  static constexpr int SLOT = MT * STAGE, SCALES = PER<GROUP> * COLS * 8;           // (scale, less) pairs of a stage
  static constexpr int PART = ROWS * (COLS + 1) * 4;   // a part's sums, of all the rows there can be
  static constexpr int SCALE_AT = WARPS * DEPTH * SLOT, BAR_AT = SCALE_AT + WARPS * SCALES, FLAG_AT = BAR_AT + WARPS * DEPTH * 8, PART_AT = FLAG_AT + 16, SMEM = 1024 + PART_AT;
  static constexpr int MOST = SMEM + (WARPS == 8 ? 1 : 2) * PARTS * PART;      // eight warps share one tile, of four two at least
  static_assert(MOST <= 232448 && BAR_AT % 8 == 0, "fits the SM");
};

__device__ __forceinline__ void load_box(uint32_t dst, const CUtensorMap* map, int32_t x, int32_t y, uint32_t bar) {
  asm volatile("cp.async.bulk.tensor.4d.shared::cluster.global.mbarrier::complete_tx::bytes [%0], [%1, {%2, %3, %4, %4}], [%5];"
               ::"r"(dst), "l"(reinterpret_cast<uint64_t>(map)), "r"(x), "r"(y), "r"(0), "r"(bar) : "memory");
}

template <bool F16, int GROUP, int MT, int NT, int WARPS>
__global__ void __launch_bounds__(WARPS * 32, NT <= 2 ? 16 / WARPS : 8 / WARPS) gemv_w4_kernel(const __grid_constant__ CUtensorMap codes, const __grid_constant__ W4Params p) {
  using S = Shape4<GROUP, MT, NT, WARPS>;
  constexpr int G = PER<GROUP>, WORDS = GROUP / 32;    // words of eight codes that a lane takes of each row and group
  constexpr int COLS = S::COLS, DEPTH = S::DEPTH;
  extern __shared__ uint8_t smem_raw[];
  uint8_t* const smem = smem_raw + ((1024u - (smem_u32(smem_raw) & 1023u)) & 1023u);
  const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
  uint8_t* const mine = smem + warp * (DEPTH * S::SLOT);
  float2* const sz = reinterpret_cast<float2*>(smem + S::SCALE_AT + warp * S::SCALES);      // [MT][G][16] (scale, less)
  const uint32_t bars = smem_u32(smem + S::BAR_AT) + warp * (DEPTH * 8);
  volatile int* const abort_flag = reinterpret_cast<volatile int*>(smem + S::FLAG_AT);
  const int m0 = (int)blockIdx.y * p.rows, rows = min(p.rows, p.M - m0);
  // the warp's tile, and its parts of K: the first one, how many, and their stages
  const int own = warp / p.wpt, tile = blockIdx.x * p.per_cta + own, stages = (p.K + SPAN - 1) / SPAN, n_parts = (stages + p.part - 1) / p.part;
  const int share = PARTS / p.wpt, part0 = (warp - own * p.wpt) * share;
  const int s0 = part0 * p.part, n_st = tile * COLS < p.N ? max(0, min(stages - s0, share * p.part)) : 0;
  if (threadIdx.x == 0) {
    for (int i = 0; i < WARPS * DEPTH; ++i) mbar_init(smem_u32(smem + S::BAR_AT) + 8 * i, 1);
    *abort_flag = 0;
    asm volatile("fence.mbarrier_init.release.cluster;" ::: "memory");
  }
  __syncthreads();

  // Requests run ahead of the arithmetic.  A box is COLS rows of 128 bytes, 16-byte piece c at c ^ (row & 7), zeros behind the last row and behind K (A
  // has zeros there too, and the rows' sums are dropped).
  int r_i = 0;
  auto request = [&] {
    if (r_i >= n_st) return;
    if (lane == 0) {
      mbar_expect_tx(bars + 8 * (r_i % DEPTH), S::SLOT);
      load_box(smem_u32(mine) + r_i % DEPTH * S::SLOT, &codes, (s0 + r_i) * (SPAN / 4), tile * COLS, bars + 8 * (r_i % DEPTH));
    }
    ++r_i;
  };
  // The scales and zero points of a stage, G * COLS of each, one stage ahead: a lane's share is one group of rows lane / G, STEP further, ...
  constexpr int SHARE = G * COLS / 32, STEP = 32 / G;
  float scale[SHARE];
  uint32_t zero[SHARE];
  const int64_t n_first = (int64_t)tile * COLS + lane / G;
  int s_group = s0 * G + lane % G;
  const int s_left = (int)(p.N - n_first);
  int64_t s_from = n_first * p.scale_ld + s_group, z_from = n_first * p.zero_ld + s_group;
  const int64_t s_step = STEP * p.scale_ld, z_step = STEP * p.zero_ld;
  auto fetch = [&] {
    const int left = s_group < p.groups ? s_left : 0;
    auto load = [&](auto get) {
#pragma unroll
      for (int q = 0; q < SHARE; ++q) scale[q] = STEP * q < left ? get(s_from + q * s_step) : 0.0f;
    };
    if (p.scale_dtype == RG_BF16) load([&](int64_t i) { return bf16_bits_to_f32(__ldg(static_cast<const uint16_t*>(p.scales) + i)); });
    else if (p.scale_dtype == RG_F16) load([&](int64_t i) { return f16_bits_to_f32(__ldg(static_cast<const uint16_t*>(p.scales) + i)); });
    else load([&](int64_t i) { return __ldg(static_cast<const float*>(p.scales) + i); });
#pragma unroll
    for (int q = 0; q < SHARE; ++q) zero[q] = p.zeros && STEP * q < left ? __ldg(p.zeros + z_from + q * z_step) : 8u;
    s_from += G; z_from += G; s_group += G;
  };
  auto put = [&] {
#pragma unroll
    for (int q = 0; q < SHARE; ++q) {
      const int row = lane / G + STEP * q;
      const uint32_t less = (zero[q] & 15u) * 0x10001u + (F16 ? 0xe400e400u : 0xc300c300u);       // -(1024 + z), -(128 + z)
      sz[((row >> 4) * G + lane % G) * 16 + (row & 15)] = make_float2(scale[q], __uint_as_float(less));
    }
  };

  asm volatile("griddepcontrol.launch_dependents;" ::: "memory");
  // with the promise that nothing in flight writes the weights their first stages are on their way before the kernels ahead have finished
  if (!p.w_static) asm volatile("griddepcontrol.wait;" ::: "memory");
#pragma unroll
  for (int i = 0; i < DEPTH - 1; ++i) request();
  if (n_st > 0) fetch();
  if (p.w_static) asm volatile("griddepcontrol.wait;" ::: "memory");

  const int t = lane & 3, rr = lane >> 2;
  const int r = (rr >> 2) | (rr & 2) | (rr & 1) << 2;  // the lane's row of the upper eight: neighbours differ in the bits that the pieces' order uses
  const uint16_t* x_at[NT];                            // columns behind the last row of A repeat it: nobody reads their sums
#pragma unroll
  for (int j = 0; j < NT; ++j) x_at[j] = p.A + (int64_t)(m0 + min(8 * j + rr, rows - 1)) * p.lda + s0 * SPAN + t * (GROUP / 4);
  // a lane's first word within a row's 128 bytes; a group's place further on only turns bits of it
  const uint32_t w_lane = r * 128 + ((((t * (GROUP / 8)) >> 4) ^ r) << 4) + (t * (GROUP / 8) & 15);
  uint32_t mask = 0x000f000fu, magic = F16 ? 0x64006400u : 0x43004300u;
  asm("" : "+r"(mask), "+r"(magic));
  float sum[MT][NT][4];
  // A's elements of a stage, on their way before the codes are waited for.  TAIL: the last stage of K, of which `left` elements are there.
  constexpr int HELD = NT == 1 ? G : 1;                // groups of A's elements that there are registers for
  uint4 x_of[HELD][NT][WORDS];
  auto load_x = [&](int g, int left, auto tail) {
#pragma unroll
    for (int j = 0; j < NT; ++j)
#pragma unroll
      for (int i = 0; i < WORDS; ++i)
        x_of[g % HELD][j][i] = !decltype(tail)::value || g * GROUP + t * (GROUP / 4) + 8 * i < left ? __ldg(reinterpret_cast<const uint4*>(x_at[j] + g * GROUP + 8 * i)) : make_uint4(0u, 0u, 0u, 0u);
  };
  auto window = [&](int g, uint32_t at, const float2* s) {
    float acc[MT][NT][4];
    // this lane's words of its rows: GROUP / 4 codes from the group's k + t GROUP / 4 on
    uint32_t w[MT][2][WORDS];
    float2 f[MT][2];
#pragma unroll
    for (int a = 0; a < MT; ++a)
#pragma unroll
      for (int u = 0; u < 2; ++u) {
        const uint8_t* from = mine + at + a * STAGE + u * 1024;
        if constexpr (WORDS == 4) { const uint4 x = *reinterpret_cast<const uint4*>(from); w[a][u][0] = x.x; w[a][u][1] = x.y; w[a][u][2] = x.z; w[a][u][3] = x.w; }
        else if constexpr (WORDS == 2) { const uint2 x = *reinterpret_cast<const uint2*>(from); w[a][u][0] = x.x; w[a][u][1] = x.y; }
        else w[a][u][0] = *reinterpret_cast<const uint32_t*>(from);
        f[a][u] = s[a * (G * 16) + 8 * u];
      }
#pragma unroll
    for (int x = 0; x < WORDS; ++x) {
      // A's elements in the codes' order: 0 4, 1 5, 2 6, 3 7
      uint32_t b0[NT], b1[NT], b2[NT], b3[NT];
#pragma unroll
      for (int j = 0; j < NT; ++j) {
        b0[j] = __byte_perm(x_of[g % HELD][j][x].x, x_of[g % HELD][j][x].z, 0x5410); b1[j] = __byte_perm(x_of[g % HELD][j][x].x, x_of[g % HELD][j][x].z, 0x7632);
        b2[j] = __byte_perm(x_of[g % HELD][j][x].y, x_of[g % HELD][j][x].w, 0x5410); b3[j] = __byte_perm(x_of[g % HELD][j][x].y, x_of[g % HELD][j][x].w, 0x7632);
      }
#pragma unroll
      for (int a = 0; a < MT; ++a) {
        const uint32_t up = w[a][0][x], down = w[a][1][x], lu = __float_as_uint(f[a][0].y), ld = __float_as_uint(f[a][1].y);
        const uint32_t u0 = unpack<F16, 0>(up, mask, magic, lu), u1 = unpack<F16, 1>(up, mask, magic, lu), u2 = unpack<F16, 2>(up, mask, magic, lu), u3 = unpack<F16, 3>(up, mask, magic, lu);
        const uint32_t d0 = unpack<F16, 0>(down, mask, magic, ld), d1 = unpack<F16, 1>(down, mask, magic, ld), d2 = unpack<F16, 2>(down, mask, magic, ld), d3 = unpack<F16, 3>(down, mask, magic, ld);
#pragma unroll
        for (int j = 0; j < NT; ++j) {
          if (x == 0) mma16<F16, true>(acc[a][j], u0, d0, u1, d1, b0[j], b1[j]);
          else mma16<F16, false>(acc[a][j], u0, d0, u1, d1, b0[j], b1[j]);
          mma16<F16, false>(acc[a][j], u2, d2, u3, d3, b2[j], b3[j]);
        }
      }
    }
#pragma unroll
    for (int a = 0; a < MT; ++a)
#pragma unroll
      for (int j = 0; j < NT; ++j)
#pragma unroll
        for (int e = 0; e < 4; ++e) sum[a][j][e] = f_fma(f[a][e >> 1].x, acc[a][j][e], sum[a][j][e]);
  };

#pragma unroll
  for (int a = 0; a < MT; ++a)
#pragma unroll
    for (int j = 0; j < NT; ++j)
#pragma unroll
      for (int e = 0; e < 4; ++e) sum[a][j][e] = 0.0f;
  int in_part = 0, part = part0;
  auto stage = [&](int i, int left, auto tail) {
    if (HELD == G) {
#pragma unroll
      for (int g = 0; g < G; ++g) load_x(g, left, tail);
    }
    put();
    if (i + 1 < n_st) fetch();
    request();
    const uint32_t slot = i % DEPTH;
    warp_mbar_wait(bars + 8 * slot, (i / DEPTH) & 1, abort_flag, &g_gemv_four_status_word, 0x4000u | slot);      // one that gives up lets the kernel run out
    __syncwarp();                                      // and every lane's scales are there
#pragma unroll
    for (int g = 0; g < G; ++g) {
      if (decltype(tail)::value && g * GROUP >= left) break;
      if (HELD != G) load_x(g, left, tail);
      window(g, slot * S::SLOT + (w_lane ^ (g * (GROUP / 2))), sz + r + g * 16);
    }
#pragma unroll
    for (int j = 0; j < NT; ++j) x_at[j] += SPAN;
    __syncwarp();                                      // the slot and the scales are free
  };
  for (int i = 0; i < n_st; ++i) {
    const int left = p.K - (s0 + i) * SPAN;
    if (left >= SPAN) stage(i, left, std::false_type{});
    else stage(i, left, std::true_type{});
    if (++in_part == p.part || i + 1 == n_st) {
      // A part is done.  The parts are joined in ascending order: by the tile's only warp as it goes, into the place of the first, or by all warps at the end.
      float* const to = reinterpret_cast<float*>(smem + S::PART_AT) + ((p.wpt == 1 ? own : own * PARTS + part) * rows + 2 * t) * (COLS + 1) + r;       // [rows][COLS + 1]
      const bool onto = p.wpt == 1 && part > 0;
#pragma unroll
      for (int a = 0; a < MT; ++a)
#pragma unroll
        for (int j = 0; j < NT; ++j)
#pragma unroll
          for (int e = 0; e < 4; ++e) {
            float* const at = to + (8 * j + (e & 1)) * (COLS + 1) + 16 * a + 8 * (e >> 1);
            if (8 * j + 2 * t + (e & 1) < rows) *at = onto ? f_add(*at, sum[a][j][e]) : sum[a][j][e];
            sum[a][j][e] = 0.0f;
          }
      in_part = 0;
      ++part;
    }
  }
  __syncthreads();
  const int places = p.wpt == 1 ? 1 : n_parts;
  for (int x = threadIdx.x; x < p.per_cta * rows * COLS; x += WARPS * 32) {
    const int col = x % COLS, tile_row = x / COLS, which = tile_row / rows, row = tile_row - which * rows, n = (blockIdx.x * p.per_cta + which) * COLS + col;
    if (n >= p.N) continue;
    const float* from = reinterpret_cast<const float*>(smem + S::PART_AT) + (which * (p.wpt == 1 ? 1 : PARTS) * rows + row) * (COLS + 1) + col;
    float v = *from;
    for (int q = 1; q < places; ++q) v = f_add(v, from[q * rows * (COLS + 1)]);
    store_scalar(p.C, p.c_dtype, (int64_t)(m0 + row) * p.ldc + n, apply_epilogue(v, p.epi, m0 + row, n));
  }
  if (*abort_flag) {                                   // a wait gave up: let copies in flight end
    const uint64_t t0 = globaltimer_ns();
    while (globaltimer_ns() - t0 < 200000ull) __nanosleep(1000);
  }
}

template <bool F16, int GROUP, int MT, int NT, int WARPS>
cudaError_t launch(const rg_weights_four_t* W, W4Params p, int wpt, cudaStream_t st) {
  using S = Shape4<GROUP, MT, NT, WARPS>;
  static DeviceOnce configured;
  const DeviceInfo dev = current_device();
  if (!configured.has(dev.dev)) {
    const cudaError_t e = cudaFuncSetAttribute(gemv_w4_kernel<F16, GROUP, MT, NT, WARPS>, cudaFuncAttributeMaxDynamicSharedMemorySize, S::MOST);
    if (e != cudaSuccess) return e;
    configured.set(dev.dev);
  }
  CUtensorMap codes;                                   // four codes an element of 16 bits
  if (!make_tmap_4d(&codes, W->codes, RG_BF16, {p.K / 4, p.N, 1, 1}, {W->code_ld / 2, 0, 0}, {SPAN / 4, S::COLS, 1, 1})) return cudaErrorInvalidValue;
  const int passes = (p.M + S::ROWS - 1) / S::ROWS;
  p.rows = passes == 1 ? p.M : ((p.M + passes - 1) / passes + 7) / 8 * 8;
  p.wpt = wpt;
  p.per_cta = WARPS / wpt;
  const int tiles = (p.N + S::COLS - 1) / S::COLS;
  cudaLaunchConfig_t cfg = {};
  cfg.gridDim = dim3((unsigned)((tiles + p.per_cta - 1) / p.per_cta), (unsigned)((p.M + p.rows - 1) / p.rows), 1);
  cfg.blockDim = dim3(WARPS * 32, 1, 1);
  cfg.dynamicSmemBytes = S::SMEM + p.per_cta * (wpt > 1 ? PARTS : 1) * p.rows * (S::COLS + 1) * 4;
  cfg.stream = st;
  cudaLaunchAttribute attr[1];
  attr[0].id = cudaLaunchAttributeProgrammaticStreamSerialization;
  attr[0].val.programmaticStreamSerializationAllowed = 1;
  cfg.attrs = attr;
  cfg.numAttrs = 1;
  return cudaLaunchKernelEx(&cfg, gemv_w4_kernel<F16, GROUP, MT, NT, WARPS>, codes, p);
}
// Warps: enough for every SM to have WARPS_PER_SM, in tiles of 32 rows of weights (A's elements are read and put in order once for them) if that is enough
// with eight warps a tile, else of 16; and no more a tile than that takes.
constexpr int WARPS_PER_SM = 12;
template <bool F16, int GROUP, int NT>
cudaError_t launch_rows(const rg_weights_four_t* W, const W4Params& p, cudaStream_t st) {
  const int64_t want = (int64_t)WARPS_PER_SM * current_device().sms;
  const int64_t wide = (p.N + 31) / 32;
  if (wide * PARTS >= want || NT > 2) {
    int wpt = PARTS;
    while (wpt > 1 && wide * (wpt / 2) >= want) wpt /= 2;
    if (wpt == 8) return launch<F16, GROUP, 2, NT, 8>(W, p, wpt, st);
    return launch<F16, GROUP, 2, NT, 4>(W, p, wpt, st);
  }
  if constexpr (NT <= 2) return launch<F16, GROUP, 1, NT, 8>(W, p, PARTS, st);
  return cudaErrorInvalidValue;
}
template <bool F16, int GROUP>
cudaError_t launch_group(const rg_weights_four_t* W, const W4Params& p, cudaStream_t st) {
  return p.M <= 8 ? launch_rows<F16, GROUP, 1>(W, p, st) : p.M <= 16 ? launch_rows<F16, GROUP, 2>(W, p, st) : launch_rows<F16, GROUP, 4>(W, p, st);
}
template <bool F16>
cudaError_t launch_type(const rg_weights_four_t* W, const W4Params& p, cudaStream_t st) {
  return W->group == 32 ? launch_group<F16, 32>(W, p, st) : W->group == 64 ? launch_group<F16, 64>(W, p, st) : launch_group<F16, 128>(W, p, st);
}

}  // namespace

// All arguments were validated by the caller.
rg_status_t launch_gemv_w4(const rg_weights_four_t* W, const rg_tensor_t* A, const rg_tensor_t* C, const rg_epilogue_t* epi, cudaStream_t st) {
  W4Params p{};
  p.scales = W->scales; p.zeros = static_cast<const uint8_t*>(W->zeros);
  p.scale_ld = W->scale_ld; p.zero_ld = W->zero_ld; p.scale_dtype = W->scale_dtype; p.w_static = W->w_static;
  p.A = static_cast<const uint16_t*>(A->ptr); p.C = C->ptr; p.lda = A->ld; p.ldc = C->ld; p.c_dtype = C->dtype;
  p.M = (int32_t)A->rows; p.N = (int32_t)W->rows; p.K = (int32_t)W->cols;
  p.groups = (p.K + W->group - 1) / W->group;
  const int stages = (p.K + SPAN - 1) / SPAN;
  p.part = (stages + PARTS - 1) / PARTS;
  if (epi) {
    p.epi.bias = epi->bias; p.epi.bias_dtype = epi->bias_dtype; p.epi.act = epi->act;
    p.epi.residual = epi->residual; p.epi.residual_dtype = epi->residual_dtype; p.epi.ldr = epi->ldr;
  }
  const cudaError_t e = A->dtype == RG_F16 ? launch_type<true>(W, p, st) : launch_type<false>(W, p, st);
  return e == cudaSuccess ? RG_OK : RG_ERR_CUDA;
}

rg_status_t read_and_clear_gemv_four_status(uint32_t* code) {
  unsigned int v = 0, zero = 0;
  if (cudaMemcpyFromSymbol(&v, g_gemv_four_status_word, sizeof(v)) != cudaSuccess) return RG_ERR_CUDA;
  if (v != 0 && cudaMemcpyToSymbol(g_gemv_four_status_word, &zero, sizeof(zero)) != cudaSuccess) return RG_ERR_CUDA;
  *code = v;
  return v ? RG_ERR_TIMEOUT : RG_OK;
}

}  // namespace rg

// Products of a few rows with weights held in four bits (rg_gemv_four):
//   C[m][n] = epilogue( sum over groups G of scale[n][G] * ( sum over k in G of A[m][k] (u[n][k] - z[n][G]) ) )
//
// The inner sum is a chain of 16-wide tensor-core steps from a zero accumulator: u - z is an integer of at most four bits and a sign, exact in bf16 and
// fp16, so nothing is rounded before the products' fp32 sum.  The scale multiplies a finished group once, in fp32 (fused, onto the running sum of a part of
// K): no weight is ever narrowed, whatever the scales' type.  A part is a run of whole 256-wide stages, at most eight of them over K; the lower and the
// upper four are each added in ascending order, and then to one another, and zero last of all: parts that a form adds as zeros, and another does not, would else tell a
// sum of -0 (of products below the smallest number) apart.  The cut follows from K alone and an accumulator's column is one row of A, so a row's bits do not depend on M.
//
// Weights are the 16 rows of mma.sync's first operand, read straight from the natural order of the codes: a warp's lanes hold whole words of eight codes, and
// the order of k within a group is the tensor core's own affair as long as A's elements follow it.  tcgen05 would want the unpacked weights in shared or
// tensor memory, a trip that costs more than these few rows' products.  Every warp streams its own stages into shared memory, a TMA box at a time.
//
// Two kernels.  One to four rows (a rule below has the exceptions): a warp copies A's elements along with its codes and never waits for another warp until all its parts are done.
// More: eight warps share A's elements in shared memory, stage by stage.  28672 x 4096 in groups of 128, bf16, zero points, a graph of calls on rotating weights, us:
//   rows          1      2      3      4      5      8     16     40
//   the first    21.3   21.6   22.2   22.6
//   the second                 26.2   26.1   26.2   26.5   31.5   58.6
// What bounds them: the bytes of the codes would take 9.4 us.  The instructions that unpack them (a mask that makes a float's mantissa of the nibble, and one
// subtraction, for two codes, with a shift for three of four) keep the half-rate integer pipe busy for 8 us, and 12 to 16 warps of an SM do not cover all
// waits between them; a grid of 128-row blocks also fills its last wave only in part.
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
  int32_t share, ctas;                                 // parts of a CTA, CTAs with the same weights' rows: a cluster
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

// ---------------------------------------------------------------- one to four rows
// A CTA's tile is 16 MT rows of weights; its four or eight warps share it, each with one or two parts of K.
constexpr int FEW = 4;                                 // rows
template <int GROUP, int MT, int WARPS>
struct Shape4 {
  static constexpr int COLS = 16 * MT, DEPTH = MT == 1 ? 3 : 2;       // stages of a warp's ring, one being worked on
  static constexpr int SLOT = MT * STAGE, SCALES = PER<GROUP> * COLS * 8;           // (scale, less) pairs of a stage
  static constexpr int X_ROW = SPAN * 2 + 16;          // a row of a stage of A; rows begin in different banks
  static constexpr int SCALE_AT = WARPS * DEPTH * SLOT, BAR_AT = SCALE_AT + WARPS * SCALES, FLAG_AT = BAR_AT + WARPS * DEPTH * 8, PART_AT = FLAG_AT + 16, SMEM = 1024 + PART_AT;
  static constexpr int ROW = PARTS * (COLS + 1) * 4 + WARPS * DEPTH * X_ROW;         // for every row of A: its parts' sums and, behind them all, its stages
  static constexpr int MOST = SMEM + FEW * ROW;
  static_assert(MOST <= 120 * 1024 && BAR_AT % 8 == 0, "fits the SM, but for four rows of eight warps in groups of 32 twice");
};

__device__ __forceinline__ void load_box(uint32_t dst, const CUtensorMap* map, int32_t x, int32_t y, uint32_t bar) {
  asm volatile("cp.async.bulk.tensor.4d.shared::cluster.global.mbarrier::complete_tx::bytes [%0], [%1, {%2, %3, %4, %4}], [%5];"
               ::"r"(dst), "l"(reinterpret_cast<uint64_t>(map)), "r"(x), "r"(y), "r"(0), "r"(bar) : "memory");
}

// The sum of the parts of K: of the lower and of the upper four, each in ascending order.  The epilogue takes it with zero added.
__device__ __forceinline__ float join(const float (&q)[PARTS]) {
  return f_add(f_add(f_add(f_add(q[0], q[1]), q[2]), q[3]), f_add(f_add(f_add(q[4], q[5]), q[6]), q[7]));
}

// The scales and zero points of a warp's stages, PER * 16 MT of each a stage, fetched one stage ahead: a lane's share is one group of rows lane / PER, STEP further, ...
template <int GROUP, int MT>
struct Scales {
  static constexpr int G = PER<GROUP>, SHARE = G * 16 * MT / 32, STEP = 32 / G;
  float scale[SHARE];
  uint32_t zero[SHARE];
  int64_t s_from, z_from, s_step, z_step;
  int group, left;
  __device__ __forceinline__ Scales(const W4Params& p, int64_t row, int first_group)
      : s_from(row * p.scale_ld + first_group), z_from(row * p.zero_ld + first_group), s_step(STEP * p.scale_ld), z_step(STEP * p.zero_ld), group(first_group), left((int)max(p.N - row, (int64_t)0)) {}
  __device__ __forceinline__ void fetch(const W4Params& p) {
    const int n = group < p.groups ? left : 0;
    auto load = [&](auto get) {
#pragma unroll
      for (int q = 0; q < SHARE; ++q) scale[q] = STEP * q < n ? get(s_from + q * s_step) : 0.0f;
    };
    if (p.scale_dtype == RG_BF16) load([&](int64_t i) { return bf16_bits_to_f32(__ldg(static_cast<const uint16_t*>(p.scales) + i)); });
    else if (p.scale_dtype == RG_F16) load([&](int64_t i) { return f16_bits_to_f32(__ldg(static_cast<const uint16_t*>(p.scales) + i)); });
    else load([&](int64_t i) { return __ldg(static_cast<const float*>(p.scales) + i); });
#pragma unroll
    for (int q = 0; q < SHARE; ++q) zero[q] = p.zeros && STEP * q < n ? __ldg(p.zeros + z_from + q * z_step) : 8u;
    s_from += G; z_from += G; group += G;
  }
  // as (scale, -(128 + z) or -(1024 + z) twice) pairs [MT][G][16]
  __device__ __forceinline__ void put(float2* sz, bool f16) const {
    const int lane = threadIdx.x & 31;
#pragma unroll
    for (int q = 0; q < SHARE; ++q) {
      const int row = lane / G + STEP * q;
      const uint32_t less = (zero[q] & 15u) * 0x10001u + (f16 ? 0xe400e400u : 0xc300c300u);
      sz[((row >> 4) * G + lane % G) * 16 + (row & 15)] = make_float2(scale[q], __uint_as_float(less));
    }
  }
};

template <bool F16, int GROUP, int MT, int WARPS>
__global__ void __launch_bounds__(WARPS * 32, 16 / WARPS) gemv_w4_kernel(const __grid_constant__ CUtensorMap codes, const __grid_constant__ W4Params p) {
  using S = Shape4<GROUP, MT, WARPS>;
  constexpr int G = PER<GROUP>, WORDS = GROUP / 32;    // words of eight codes that a lane takes of each row and group
  constexpr int COLS = S::COLS, DEPTH = S::DEPTH;
  extern __shared__ uint8_t smem_raw[];
  uint8_t* const smem = smem_raw + ((1024u - (smem_u32(smem_raw) & 1023u)) & 1023u);
  const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
  uint8_t* const mine = smem + warp * (DEPTH * S::SLOT);
  float2* const sz = reinterpret_cast<float2*>(smem + S::SCALE_AT + warp * S::SCALES);      // [MT][G][16] (scale, less)
  const uint32_t bars = smem_u32(smem + S::BAR_AT) + warp * (DEPTH * 8);
  volatile int* const abort_flag = reinterpret_cast<volatile int*>(smem + S::FLAG_AT);
  const int rows = p.M, x_slot = rows * S::X_ROW;
  uint8_t* const x_mine = smem + S::PART_AT + PARTS * rows * (COLS + 1) * 4 + warp * (DEPTH * x_slot);
  // the warp's parts of K: the first one, how many, and their stages
  const int tile = blockIdx.x, stages = (p.K + SPAN - 1) / SPAN, n_parts = (stages + p.part - 1) / p.part;
  constexpr int SHARE = PARTS / WARPS;
  const int part0 = warp * SHARE, s0 = part0 * p.part, n_st = max(0, min(stages - s0, SHARE * p.part));
  if (threadIdx.x == 0) {
    for (int i = 0; i < WARPS * DEPTH; ++i) mbar_init(smem_u32(smem + S::BAR_AT) + 8 * i, 1);
    *abort_flag = 0;
    asm volatile("fence.mbarrier_init.release.cluster;" ::: "memory");
  }
  __syncthreads();

  // Requests run ahead of the arithmetic.  A box is COLS rows of 128 bytes, 16-byte piece c at c ^ (row & 7), zeros behind the last row and behind K (A
  // has zeros there too, and the rows' sums are dropped).
  auto request_codes = [&](int i) {
    if (i < n_st && lane == 0) {
      mbar_expect_tx(bars + 8 * (i % DEPTH), S::SLOT + rows * 2 * min(SPAN, p.K - (s0 + i) * SPAN));
      load_box(smem_u32(mine) + i % DEPTH * S::SLOT, &codes, (s0 + i) * (SPAN / 4), tile * COLS, bars + 8 * (i % DEPTH));
    }
  };
  auto request_x = [&](int i) {
    if (i < n_st && lane < rows)
      bulk_load_1d(smem_u32(x_mine) + i % DEPTH * x_slot + lane * S::X_ROW, p.A + lane * p.lda + (s0 + i) * SPAN, 2 * min(SPAN, p.K - (s0 + i) * SPAN), bars + 8 * (i % DEPTH));
  };
  Scales<GROUP, MT> scales(p, (int64_t)tile * COLS + lane / G, s0 * G + lane % G);

  asm volatile("griddepcontrol.launch_dependents;" ::: "memory");
  // with the promise that nothing in flight writes the weights their first stages are on their way before the kernels ahead have finished
  if (!p.w_static) asm volatile("griddepcontrol.wait;" ::: "memory");
#pragma unroll
  for (int i = 0; i < DEPTH - 1; ++i) request_codes(i);
  if (n_st > 0) scales.fetch(p);
  if (p.w_static) asm volatile("griddepcontrol.wait;" ::: "memory");
  __syncwarp();
#pragma unroll
  for (int i = 0; i < DEPTH - 1; ++i) request_x(i);

  const int t = lane & 3, rr = lane >> 2;
  const int r = (rr >> 2) | (rr & 2) | (rr & 1) << 2;  // the lane's row of the upper eight: neighbours differ in the bits that the pieces' order uses
  const uint8_t* const x_at = x_mine + min(rr, rows - 1) * S::X_ROW + t * (GROUP / 2);       // columns behind the last row of A repeat it: nobody reads their sums
  // a lane's first word within a row's 128 bytes; a group's place further on only turns bits of it
  const uint32_t w_lane = r * 128 + ((((t * (GROUP / 8)) >> 4) ^ r) << 4) + (t * (GROUP / 8) & 15);
  uint32_t mask = 0x000f000fu, magic = F16 ? 0x64006400u : 0x43004300u;
  asm("" : "+r"(mask), "+r"(magic));
  float sum[MT][4];
  // TAIL: the last stage of K, of which `left` elements are there
  auto window = [&](int g, uint32_t at, const uint8_t* xs, const float2* s, int left, auto tail) {
    float acc[MT][4];
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
      uint4 v = *reinterpret_cast<const uint4*>(xs + g * (GROUP * 2) + 16 * x);
      if (decltype(tail)::value && g * GROUP + t * (GROUP / 4) + 8 * x >= left) v = make_uint4(0u, 0u, 0u, 0u);
      const uint32_t b0 = __byte_perm(v.x, v.z, 0x5410), b1 = __byte_perm(v.x, v.z, 0x7632), b2 = __byte_perm(v.y, v.w, 0x5410), b3 = __byte_perm(v.y, v.w, 0x7632);
#pragma unroll
      for (int a = 0; a < MT; ++a) {
        const uint32_t up = w[a][0][x], down = w[a][1][x], lu = __float_as_uint(f[a][0].y), ld = __float_as_uint(f[a][1].y);
        const uint32_t u0 = unpack<F16, 0>(up, mask, magic, lu), u1 = unpack<F16, 1>(up, mask, magic, lu), u2 = unpack<F16, 2>(up, mask, magic, lu), u3 = unpack<F16, 3>(up, mask, magic, lu);
        const uint32_t d0 = unpack<F16, 0>(down, mask, magic, ld), d1 = unpack<F16, 1>(down, mask, magic, ld), d2 = unpack<F16, 2>(down, mask, magic, ld), d3 = unpack<F16, 3>(down, mask, magic, ld);
        if (x == 0) mma16<F16, true>(acc[a], u0, d0, u1, d1, b0, b1);
        else mma16<F16, false>(acc[a], u0, d0, u1, d1, b0, b1);
        mma16<F16, false>(acc[a], u2, d2, u3, d3, b2, b3);
      }
    }
#pragma unroll
    for (int a = 0; a < MT; ++a)
#pragma unroll
      for (int e = 0; e < 4; ++e) sum[a][e] = f_fma(f[a][e >> 1].x, acc[a][e], sum[a][e]);
  };

#pragma unroll
  for (int a = 0; a < MT; ++a)
#pragma unroll
    for (int e = 0; e < 4; ++e) sum[a][e] = 0.0f;
  int in_part = 0, part = part0;
  auto stage = [&](int i, int left, auto tail) {
    scales.put(sz, F16);
    if (i + 1 < n_st) scales.fetch(p);
    request_codes(i + DEPTH - 1);
    __syncwarp();
    request_x(i + DEPTH - 1);
    const uint32_t slot = i % DEPTH;
    warp_mbar_wait(bars + 8 * slot, (i / DEPTH) & 1, abort_flag, &g_gemv_four_status_word, 0x4000u | slot);      // one that gives up lets the kernel run out
    __syncwarp();                                      // and every lane's scales are there
#pragma unroll
    for (int g = 0; g < G; ++g) {
      if (decltype(tail)::value && g * GROUP >= left) break;
      window(g, slot * S::SLOT + (w_lane ^ (g * (GROUP / 2))), x_at + slot * x_slot, sz + r + g * 16, left, tail);
    }
    __syncwarp();                                      // the slot and the scales are free
  };
  for (int i = 0; i < n_st; ++i) {
    const int left = p.K - (s0 + i) * SPAN;
    if (left >= SPAN) stage(i, left, std::false_type{});
    else stage(i, left, std::true_type{});
    if (++in_part == p.part || i + 1 == n_st) {
      // a part is done; all are joined at the end
      float* const to = reinterpret_cast<float*>(smem + S::PART_AT) + (part * rows + 2 * t) * (COLS + 1) + r;       // [rows][COLS + 1]
#pragma unroll
      for (int a = 0; a < MT; ++a)
#pragma unroll
        for (int e = 0; e < 4; ++e) {
          if (2 * t + (e & 1) < rows) to[(e & 1) * (COLS + 1) + 16 * a + 8 * (e >> 1)] = sum[a][e];
          sum[a][e] = 0.0f;
        }
      in_part = 0;
      ++part;
    }
  }
  __syncthreads();
  for (int x = threadIdx.x; x < rows * COLS; x += WARPS * 32) {
    const int col = x % COLS, row = x / COLS, n = tile * COLS + col;
    if (n >= p.N) continue;
    const float* from = reinterpret_cast<const float*>(smem + S::PART_AT) + row * (COLS + 1) + col;
    float q[PARTS];
#pragma unroll
    for (int i = 0; i < PARTS; ++i) q[i] = i < n_parts ? from[i * rows * (COLS + 1)] : 0.0f;
    const float v = f_add(join(q), 0.0f);
    store_scalar(p.C, p.c_dtype, (int64_t)row * p.ldc + n, apply_epilogue(v, p.epi, row, n));
  }
  if (*abort_flag) {                                   // a wait gave up: let copies in flight end
    const uint64_t t0 = globaltimer_ns();
    while (globaltimer_ns() - t0 < 200000ull) __nanosleep(1000);
  }
}

// ---------------------------------------------------------------- five rows and more
// The same sums for 8 NT rows of A.  Eight warps, each with a tile of 16 rows of weights of its own, work on the same stage, for which they share A's elements in shared
// memory (put there, and into the codes' order, once).  The parts of K are shared among the CTAs of a cluster, or are all one CTA's, and are joined over distributed shared
// memory, every CTA a share of the elements.  How many parts a CTA has (1, 2, 4 or all 8) is the choice with which the waves of CTAs take the fewest stages (below):
// 16 rows on 128256 x 4096, where many blocks fill the GPU, take 122 us with all parts in a CTA and 173 us with two; on 4096 x 14336, where eight CTAs for each block are
// needed, 17.1 us.  33 rows on 11009 x 4128 in groups of 32 take 32.4 us (79 with one warp a part and A's elements from global memory).  Reading A's elements two stages
// ahead instead of one changes nothing; more than 40 rows would leave room for one CTA of an SM only (64 rows on 28672 x 4096: 113 us, as twice 32 rows 94).
constexpr int RW = 8;                                  // warps
template <int GROUP, int NT>
struct Rows4 {
  static constexpr int ROWS = 8 * NT, COLS = 16 * RW, DEPTH = 3;
  static constexpr int SCALES = PER<GROUP> * 16 * 8;
  static constexpr int X = ROWS * 512;                 // a stage of A
  static constexpr int RING_AT = 2 * X, SCALE_AT = RING_AT + RW * DEPTH * STAGE, BAR_AT = SCALE_AT + RW * SCALES, FLAG_AT = BAR_AT + RW * DEPTH * 8, SMEM = 1024 + FLAG_AT + 16;
  static constexpr int SUMS = 2 * ROWS * (COLS + 1) * 4;   // over A's stages, at the end
  static_assert(SMEM <= 113 * 1024 && X % 1024 == 0 && BAR_AT % 8 == 0 && SUMS <= SCALE_AT, "two fit the SM");
};

template <bool F16, int GROUP, int NT>
__global__ void __launch_bounds__(RW * 32, 2) gemv_w4_rows_kernel(const __grid_constant__ CUtensorMap codes, const __grid_constant__ W4Params p) {
  using S = Rows4<GROUP, NT>;
  constexpr int G = PER<GROUP>, WORDS = GROUP / 32, COLS = S::COLS, DEPTH = S::DEPTH;
  extern __shared__ uint8_t smem_raw[];
  uint8_t* const smem = smem_raw + ((1024u - (smem_u32(smem_raw) & 1023u)) & 1023u);
  const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
  uint8_t* const mine = smem + S::RING_AT + warp * (DEPTH * STAGE);
  float2* const sz = reinterpret_cast<float2*>(smem + S::SCALE_AT + warp * S::SCALES);      // [G][16] (scale, less)
  const uint32_t bars = smem_u32(smem + S::BAR_AT) + warp * (DEPTH * 8);
  volatile int* const abort_flag = reinterpret_cast<volatile int*>(smem + S::FLAG_AT);
  const int m0 = (int)blockIdx.y * p.rows, rows = min(p.rows, p.M - m0);
  const int rank = (int)blockIdx.x % p.ctas, n_cta = (int)(blockIdx.x / p.ctas) * COLS, n0 = n_cta + 16 * warp;
  const int stages = (p.K + SPAN - 1) / SPAN, share = p.share, s0 = rank * share * p.part, n_st = max(0, min(stages - s0, share * p.part));
  if (threadIdx.x == 0) {
    for (int i = 0; i < RW * DEPTH; ++i) mbar_init(smem_u32(smem + S::BAR_AT) + 8 * i, 1);
    *abort_flag = 0;
    asm volatile("fence.mbarrier_init.release.cluster;" ::: "memory");
  }
  __syncthreads();

  // as above, a warp's own 16 rows of weights; warps behind the last row take part in the rest
  int r_i = 0;
  auto request = [&] {
    if (r_i >= n_st || n0 >= p.N) return;
    if (lane == 0) {
      mbar_expect_tx(bars + 8 * (r_i % DEPTH), STAGE);
      load_box(smem_u32(mine) + r_i % DEPTH * STAGE, &codes, (s0 + r_i) * (SPAN / 4), n0, bars + 8 * (r_i % DEPTH));
    }
    ++r_i;
  };
  Scales<GROUP, 1> scales(p, (int64_t)n0 + lane / G, s0 * G + lane % G);

  asm volatile("griddepcontrol.launch_dependents;" ::: "memory");
  if (!p.w_static) asm volatile("griddepcontrol.wait;" ::: "memory");
#pragma unroll
  for (int i = 0; i < DEPTH - 1; ++i) request();
  if (n_st > 0) scales.fetch(p);
  if (p.w_static) asm volatile("griddepcontrol.wait;" ::: "memory");

  // A's elements: a thread's 16-byte pieces are piece threadIdx % 32 of every eighth row.  Piece c of a row lies at c ^ turn(row), so that a quarter of a warp (two rows,
  // four places of a group) reads eight different ones; which bits that takes depends on how far apart the places are.
  auto turn = [](int row, int c) -> int {
    if (GROUP == 32) return (row & 1) << 2 | (row & 2) | (row >> 2 & 1);
    return (row & 7) ^ (GROUP == 128 ? (c >> 3 & 1) << 1 : 0);
  };
  const int x_row = threadIdx.x >> 5, x_piece = lane;
  const uint16_t* const x_src = p.A + (int64_t)m0 * p.lda + s0 * SPAN + 8 * x_piece;
  const uint32_t x_to = smem_u32(smem) + x_row * 512 + ((x_piece ^ turn(x_row, x_piece)) << 4);
  auto load_x = [&](int i) {
    const bool in_k = (s0 + i) * SPAN + 8 * x_piece < p.K;
#pragma unroll
    for (int j = 0; j < NT; ++j) {
      const bool there = in_k && x_row + 8 * j < rows;             // else zeros
      asm volatile("cp.async.cg.shared.global [%0], [%1], 16, %2;"
                   ::"r"(x_to + (i & 1) * S::X + j * 4096), "l"(x_src + (there ? (int64_t)(x_row + 8 * j) * p.lda + i * SPAN : 0)), "r"(there ? 16 : 0) : "memory");
    }
    asm volatile("cp.async.commit_group;" ::: "memory");
  };
  // ... into the codes' order: 0 4, 1 5, 2 6, 3 7
  auto order_x = [&](int i) {
    asm volatile("cp.async.wait_group 0;" ::: "memory");
    uint8_t* const at = smem + (i & 1) * S::X + x_row * 512 + ((x_piece ^ turn(x_row, x_piece)) << 4);
#pragma unroll
    for (int j = 0; j < NT; ++j) {
      uint4* const q = reinterpret_cast<uint4*>(at + j * 4096);
      const uint4 v = *q;
      *q = make_uint4(__byte_perm(v.x, v.z, 0x5410), __byte_perm(v.x, v.z, 0x7632), __byte_perm(v.y, v.w, 0x5410), __byte_perm(v.y, v.w, 0x7632));
    }
  };
  if (n_st > 0) { load_x(0); order_x(0); }
  __syncthreads();

  const int t = lane & 3, rr = lane >> 2;
  const int r = (rr >> 2) | (rr & 2) | (rr & 1) << 2;
  const uint32_t w_lane = r * 128 + ((((t * (GROUP / 8)) >> 4) ^ r) << 4) + (t * (GROUP / 8) & 15);
  // piece g (GROUP / 8) + t (GROUP / 32) + x of row rr: bits of x and, in groups of 32, of g are turned into it
  const int x_first = t * (GROUP / 32);
  const uint32_t x_lane = rr * 512 + ((x_first ^ turn(rr, x_first)) << 4);
  uint32_t mask = 0x000f000fu, magic = F16 ? 0x64006400u : 0x43004300u;
  asm("" : "+r"(mask), "+r"(magic));
  float sum[NT][4], saved[NT][4];
#pragma unroll
  for (int j = 0; j < NT; ++j)
#pragma unroll
    for (int e = 0; e < 4; ++e) sum[j][e] = saved[j][e] = 0.0f;
  int in_part = 0;
  bool first = true, second = false;
  float half[NT][4];
  for (int i = 0; i < n_st; ++i) {
    if (i + 1 < n_st) load_x(i + 1);
    scales.put(sz, F16);
    if (i + 1 < n_st) scales.fetch(p);
    request();
    const uint32_t slot = i % DEPTH;
    if (n0 < p.N) warp_mbar_wait(bars + 8 * slot, (i / DEPTH) & 1, abort_flag, &g_gemv_four_status_word, 0x4100u | slot);      // one that gives up lets the kernel run out
    __syncwarp();
    const int left = p.K - (s0 + i) * SPAN;
    const uint8_t* const xs = smem + (i & 1) * S::X;
#pragma unroll
    for (int g = 0; g < G; ++g) {
      if (g * GROUP >= left) break;
      uint32_t w[2][WORDS];
      float2 f[2];
#pragma unroll
      for (int u = 0; u < 2; ++u) {
        const uint8_t* from = mine + slot * STAGE + (w_lane ^ (g * (GROUP / 2))) + u * 1024;
        if constexpr (WORDS == 4) { const uint4 v = *reinterpret_cast<const uint4*>(from); w[u][0] = v.x; w[u][1] = v.y; w[u][2] = v.z; w[u][3] = v.w; }
        else if constexpr (WORDS == 2) { const uint2 v = *reinterpret_cast<const uint2*>(from); w[u][0] = v.x; w[u][1] = v.y; }
        else w[u][0] = *reinterpret_cast<const uint32_t*>(from);
        f[u] = sz[g * 16 + r + 8 * u];
      }
      float acc[NT][4];
#pragma unroll
      for (int x = 0; x < WORDS; ++x) {
        const uint32_t lu = __float_as_uint(f[0].y), ld = __float_as_uint(f[1].y);
        const uint32_t u0 = unpack<F16, 0>(w[0][x], mask, magic, lu), u1 = unpack<F16, 1>(w[0][x], mask, magic, lu), u2 = unpack<F16, 2>(w[0][x], mask, magic, lu), u3 = unpack<F16, 3>(w[0][x], mask, magic, lu);
        const uint32_t d0 = unpack<F16, 0>(w[1][x], mask, magic, ld), d1 = unpack<F16, 1>(w[1][x], mask, magic, ld), d2 = unpack<F16, 2>(w[1][x], mask, magic, ld), d3 = unpack<F16, 3>(w[1][x], mask, magic, ld);
        const uint32_t at = GROUP == 128 ? (x_lane ^ (x << 4)) + g * 256 : GROUP == 64 ? (x_lane ^ (x << 4)) + g * 128 : (x_lane ^ ((g & 1) << 6)) + (g >> 1) * 128;
#pragma unroll
        for (int j = 0; j < NT; ++j) {
          const uint4 b = *reinterpret_cast<const uint4*>(xs + at + j * 4096);
          if (x == 0) mma16<F16, true>(acc[j], u0, d0, u1, d1, b.x, b.y);
          else mma16<F16, false>(acc[j], u0, d0, u1, d1, b.x, b.y);
          mma16<F16, false>(acc[j], u2, d2, u3, d3, b.z, b.w);
        }
      }
#pragma unroll
      for (int j = 0; j < NT; ++j)
#pragma unroll
        for (int e = 0; e < 4; ++e) sum[j][e] = f_fma(f[e >> 1].x, acc[j][e], sum[j][e]);
    }
    if (++in_part == p.part && i + 1 < n_st) {
      // a part is done, and this CTA has another
#pragma unroll
      for (int j = 0; j < NT; ++j)
#pragma unroll
        for (int e = 0; e < 4; ++e) { saved[j][e] = first ? sum[j][e] : f_add(saved[j][e], sum[j][e]); sum[j][e] = 0.0f; }
      in_part = 0;
      first = false;
      if (i + 1 == 4 * p.part) {                       // the first half of all: share is PARTS
#pragma unroll
        for (int j = 0; j < NT; ++j)
#pragma unroll
          for (int e = 0; e < 4; ++e) half[j][e] = saved[j][e];
        first = second = true;
      }
    }
    if (i + 1 < n_st) order_x(i + 1);
    __syncthreads();                                   // the next stage of A is there, this one, the slot and the scales are free
  }
  // The part's sums, [rows][COLS + 1], or the two parts', or the half's, or the whole
  float* const sums = reinterpret_cast<float*>(smem);
  const bool both = !first && share == 2 && p.ctas > 1;
#pragma unroll
  for (int j = 0; j < NT; ++j)
#pragma unroll
    for (int e = 0; e < 4; ++e) {
      const int row = 8 * j + 2 * t + (e & 1);
      if (row >= rows) continue;
      float* const to = sums + row * (COLS + 1) + 16 * warp + r + 8 * (e >> 1);
      const float total = first ? sum[j][e] : both ? saved[j][e] : f_add(saved[j][e], sum[j][e]);
      *to = second ? f_add(half[j][e], total) : total;
      if (share == 2) to[rows * (COLS + 1)] = both ? sum[j][e] : 0.0f;
    }
  if (p.ctas > 1) asm volatile("barrier.cluster.arrive.release.aligned;\n\tbarrier.cluster.wait.acquire.aligned;" ::: "memory");
  else __syncthreads();
  for (int x = rank * (RW * 32) + threadIdx.x; x < rows * COLS; x += p.ctas * (RW * 32)) {
    const int row = x / COLS, col = x % COLS, n = n_cta + col;
    if (n >= p.N) continue;
    const uint32_t at = smem_u32(sums + row * (COLS + 1) + col);
    float q[PARTS], v;
    if (p.ctas > 1) {
#pragma unroll
      for (int i = 0; i < PARTS; ++i) {
        q[i] = 0.0f;
        if (i < p.ctas * (share == 2 ? 2 : 1)) {
          uint32_t there;
          asm volatile("mapa.shared::cluster.u32 %0, %1, %2;" : "=r"(there) : "r"(at + (share == 2 ? (i & 1) * rows * (COLS + 1) * 4 : 0)), "r"(share == 2 ? i >> 1 : i));
          asm volatile("ld.shared::cluster.f32 %0, [%1];" : "=f"(q[i]) : "r"(there) : "memory");
        }
      }
      v = share == 4 ? f_add(q[0], q[1]) : join(q);
    } else {
      v = sums[row * (COLS + 1) + col];
    }
    store_scalar(p.C, p.c_dtype, (int64_t)(m0 + row) * p.ldc + n, apply_epilogue(f_add(v, 0.0f), p.epi, m0 + row, n));
  }
  if (*abort_flag) {                                   // a wait gave up: let copies in flight end
    const uint64_t t0 = globaltimer_ns();
    while (globaltimer_ns() - t0 < 200000ull) __nanosleep(1000);
  }
  __syncwarp();
  if (p.ctas > 1) asm volatile("barrier.cluster.arrive.relaxed.aligned;\n\tbarrier.cluster.wait.acquire.aligned;" ::: "memory");      // nobody's sums go before all have read (and stored) them
}

template <bool F16, int GROUP, int NT>
cudaError_t launch_more(const rg_weights_four_t* W, W4Params p, cudaStream_t st) {
  using S = Rows4<GROUP, NT>;
  static DeviceOnce configured;
  const DeviceInfo dev = current_device();
  if (!configured.has(dev.dev)) {
    const cudaError_t e = cudaFuncSetAttribute(gemv_w4_rows_kernel<F16, GROUP, NT>, cudaFuncAttributeMaxDynamicSharedMemorySize, S::SMEM);
    if (e != cudaSuccess) return e;
    configured.set(dev.dev);
  }
  CUtensorMap codes;
  if (!make_tmap_4d(&codes, W->codes, RG_BF16, {p.K / 4, p.N, 1, 1}, {W->code_ld / 2, 0, 0}, {SPAN / 4, 16, 1, 1})) return cudaErrorInvalidValue;
  const int blocks = (p.N + S::COLS - 1) / S::COLS;
  const int parts = ((p.K + SPAN - 1) / SPAN + p.part - 1) / p.part;
  // Two CTAs an SM; a wave of them takes the time of its stages and, for its start and end, about that of three more.
  const int64_t slots = 2 * dev.sms, all = (int64_t)blocks * ((p.M + p.rows - 1) / p.rows);
  int64_t best = INT64_MAX;
  for (int share = 1; share <= PARTS; share *= 2) {
    const int64_t time = (all * ((parts + share - 1) / share) + slots - 1) / slots * (share * p.part + 3);
    if (time < best) { best = time; p.share = share; }
  }
  p.ctas = (parts + p.share - 1) / p.share;
  cudaLaunchConfig_t cfg = {};
  cfg.gridDim = dim3((unsigned)(blocks * p.ctas), (unsigned)((p.M + p.rows - 1) / p.rows), 1);
  cfg.blockDim = dim3(RW * 32, 1, 1);
  cfg.dynamicSmemBytes = S::SMEM;
  cfg.stream = st;
  cudaLaunchAttribute attr[2];
  attr[0].id = cudaLaunchAttributeProgrammaticStreamSerialization;
  attr[0].val.programmaticStreamSerializationAllowed = 1;
  attr[1].id = cudaLaunchAttributeClusterDimension;
  attr[1].val.clusterDim.x = (unsigned)p.ctas; attr[1].val.clusterDim.y = 1; attr[1].val.clusterDim.z = 1;
  cfg.attrs = attr;
  cfg.numAttrs = 2;
  return cudaLaunchKernelEx(&cfg, gemv_w4_rows_kernel<F16, GROUP, NT>, codes, p);
}

template <bool F16, int GROUP, int MT, int WARPS>
cudaError_t launch_tiles(const rg_weights_four_t* W, const W4Params& p, cudaStream_t st) {
  using S = Shape4<GROUP, MT, WARPS>;
  static DeviceOnce configured;
  const DeviceInfo dev = current_device();
  if (!configured.has(dev.dev)) {
    const cudaError_t e = cudaFuncSetAttribute(gemv_w4_kernel<F16, GROUP, MT, WARPS>, cudaFuncAttributeMaxDynamicSharedMemorySize, S::MOST);
    if (e != cudaSuccess) return e;
    configured.set(dev.dev);
  }
  CUtensorMap codes;                                   // four codes an element of 16 bits
  if (!make_tmap_4d(&codes, W->codes, RG_BF16, {p.K / 4, p.N, 1, 1}, {W->code_ld / 2, 0, 0}, {SPAN / 4, S::COLS, 1, 1})) return cudaErrorInvalidValue;
  const int tiles = (p.N + S::COLS - 1) / S::COLS;
  cudaLaunchConfig_t cfg = {};
  cfg.gridDim = dim3((unsigned)tiles, 1, 1);
  cfg.blockDim = dim3(WARPS * 32, 1, 1);
  cfg.dynamicSmemBytes = S::SMEM + p.M * S::ROW;
  cfg.stream = st;
  cudaLaunchAttribute attr[1];
  attr[0].id = cudaLaunchAttributeProgrammaticStreamSerialization;
  attr[0].val.programmaticStreamSerializationAllowed = 1;
  cfg.attrs = attr;
  cfg.numAttrs = 1;
  return cudaLaunchKernelEx(&cfg, gemv_w4_kernel<F16, GROUP, MT, WARPS>, codes, p);
}
// Tiles of 16 rows of weights with eight warps, while all of them fit the GPU at a time, two an SM (one row, groups of 128: 4096 x 14336 13.3 us, 18.7 in tiles of 32; 6144 x 4096, which
// does not fit: 10.1 and 8.5); then tiles of 32, for which A's elements are read and put in order once, with four warps, or with eight where four leave fewer than
// 12 an SM (8192 x 8192: 13.9 us with eight, 19.6 with four; 14336 x 4096: 15.7 with eight, 13.2 with four; 57344 x 8192: 63.2 with four, 79.5 with a warp a tile).  Three and four rows in
// groups of 32 fill shared memory first: four warps, three CTAs an SM, as soon as eight take more than one wave of two (10240 x 4096: 17.1 us with four, 19.6 and 22.3 with eight).
template <bool F16, int GROUP>
cudaError_t launch_few(const rg_weights_four_t* W, const W4Params& p, cudaStream_t st) {
  const int64_t sms = current_device().sms, wide = (p.N + 31) / 32;
  if ((p.N + 15) / 16 <= 2 * sms) return launch_tiles<F16, GROUP, 1, 8>(W, p, st);
  const bool eight = GROUP == 32 && p.M > 2 ? wide <= 2 * sms : wide * 4 < 12 * sms;
  return eight ? launch_tiles<F16, GROUP, 2, 8>(W, p, st) : launch_tiles<F16, GROUP, 2, 4>(W, p, st);
}
// Up to four rows the first kernel, but for sizes at which its tiles need a second wave of CTAs for lack of shared memory and the second kernel's need one.  Four rows in groups
// of 32, tiles that would have eight warps: one CTA fits an SM (4740 x 4096: 13.4 us, the second kernel 13.2; 8704 x 4096: 16.1 and 14.1; 8704 x 14336: 40.5 and 38.2); from 15/8 tiles
// an SM on clusters of the second kernel find no room in one wave either (9216 x 4096: 16.2 and 22.2).  Three or four rows in groups of 32, four in groups of 64, with four warps: three
// CTAs an SM, and the second kernel's 148 blocks are four tiles an SM (groups of 32, 18432 x 4096: 28.3 and 23.1 us, 16384 x 8192: 53.1 and 42.4; groups of 64: 19.7 and 17.8; 19072 x 4096 in groups
// of 32: 29.1 and 40.5; three rows in groups of 64, of which four fit: 16.4 and 17.8).
template <int GROUP>
bool takes_few(const W4Params& p) {
  if (p.M > FEW) return false;
  const int64_t sms = current_device().sms, wide = (p.N + 31) / 32;
  if (GROUP == 32 && p.M == 4 && (p.N + 15) / 16 > 2 * sms && wide * 8 <= 15 * sms) return false;
  return !((GROUP == 32 ? p.M > 2 : GROUP == 64 && p.M == 4) && wide > 3 * sms && wide <= 4 * sms);
}
template <bool F16, int GROUP>
cudaError_t launch_group(const rg_weights_four_t* W, W4Params p, cudaStream_t st) {
  if (takes_few<GROUP>(p)) return launch_few<F16, GROUP>(W, p, st);
  const int passes = (p.M + 39) / 40;                  // over the rows, as even as eights allow
  p.rows = ((p.M + passes - 1) / passes + 7) / 8 * 8;
  switch (p.rows / 8) {
    case 1: return launch_more<F16, GROUP, 1>(W, p, st);
    case 2: return launch_more<F16, GROUP, 2>(W, p, st);
    case 3: return launch_more<F16, GROUP, 3>(W, p, st);
    case 4: return launch_more<F16, GROUP, 4>(W, p, st);
    default: return launch_more<F16, GROUP, 5>(W, p, st);
  }
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

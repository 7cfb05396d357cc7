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
// A CTA takes 16 MT rows of weights, its eight warps a part of K each; every warp streams its own stages through shared memory by asynchronous copies.
#include <algorithm>

#include "rg_common.cuh"
#include "rg_internal.h"

namespace rg {

namespace {

constexpr int WARPS = 8, THREADS = WARPS * 32;
constexpr int SPAN = 256;                              // k of a stage: 128 bytes a row of weights

struct W4Params {
  const uint8_t* codes;
  const void* scales;
  const uint8_t* zeros;
  const uint16_t* A;
  void* C;
  int64_t code_ld, scale_ld, zero_ld, lda, ldc;
  int32_t M, N, K, groups;
  int32_t scale_dtype, c_dtype, w_static;
  int32_t part;                                        // stages of a part
  EpilogueArgs epi;
};

__device__ __forceinline__ void copy16(uint32_t dst, const void* src, bool there) {
  asm volatile("cp.async.cg.shared.global [%0], [%1], 16, %2;" ::"r"(dst), "l"(src), "r"(there ? 16 : 0) : "memory");
}
template <bool F16>
__device__ __forceinline__ uint32_t add2(uint32_t a, uint32_t b) {
  uint32_t d;
  if (F16) asm("add.rn.f16x2 %0, %1, %2;" : "=r"(d) : "r"(a), "r"(b));
  else asm("add.rn.bf16x2 %0, %1, %2;" : "=r"(d) : "r"(a), "r"(b));
  return d;
}
template <bool F16>
__device__ __forceinline__ void mma16(float (&c)[4], uint32_t a0, uint32_t a1, uint32_t a2, uint32_t a3, uint32_t b0, uint32_t b1) {
  if (F16)
    asm volatile("mma.sync.aligned.m16n8k16.row.col.f32.f16.f16.f32 {%0, %1, %2, %3}, {%4, %5, %6, %7}, {%8, %9}, {%0, %1, %2, %3};"
                 : "+f"(c[0]), "+f"(c[1]), "+f"(c[2]), "+f"(c[3]) : "r"(a0), "r"(a1), "r"(a2), "r"(a3), "r"(b0), "r"(b1));
  else
    asm volatile("mma.sync.aligned.m16n8k16.row.col.f32.bf16.bf16.f32 {%0, %1, %2, %3}, {%4, %5, %6, %7}, {%8, %9}, {%0, %1, %2, %3};"
                 : "+f"(c[0]), "+f"(c[1]), "+f"(c[2]), "+f"(c[3]) : "r"(a0), "r"(a1), "r"(a2), "r"(a3), "r"(b0), "r"(b1));
}
// Codes i and i + 4 of a word in the halves of a word, less the zero point: the mask puts them into the mantissa of 128 (bf16) or 1024 (fp16), and
// `less` is -(128 + z) or -(1024 + z) twice.
template <bool F16, int I>
__device__ __forceinline__ uint32_t unpack(uint32_t w, uint32_t less) {
  return add2<F16>(((w >> (4 * I)) & 0x000f000fu) | (F16 ? 0x64006400u : 0x43004300u), less);
}

// Bytes of a warp's ring stage for one 16-row tile, and of the scales and zero points that go with it
constexpr int STAGE = 16 * 128;
template <int GROUP> constexpr int PER = SPAN / GROUP;                 // groups of a stage

template <int GROUP, int MT>
struct Ring4 {
  static constexpr int DEPTH = MT == 1 ? 4 : 3;
  static constexpr int SCALES = 2 * PER<GROUP> * 16 * MT * 8;          // two stages of (scale, less) pairs
  static constexpr int WARP_BYTES = DEPTH * MT * STAGE + SCALES;
};

template <bool F16, int GROUP, int MT, int NT>
__global__ void __launch_bounds__(THREADS) gemv_w4_kernel(const __grid_constant__ W4Params p) {
  using R = Ring4<GROUP, MT>;
  constexpr int G = PER<GROUP>, WORDS = GROUP / 32;    // words of eight codes that a lane takes of each row and group
  extern __shared__ __align__(128) uint8_t smem[];
  const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
  uint8_t* const mine = smem + warp * R::WARP_BYTES;
  const uint32_t ring = (uint32_t)__cvta_generic_to_shared(mine);
  float2* const sz = reinterpret_cast<float2*>(mine + R::DEPTH * MT * STAGE);       // [2][MT][G][16] (scale, less)
  const int64_t n0 = (int64_t)blockIdx.x * (16 * MT);
  const int m0 = (int)blockIdx.y * (8 * NT);
  const int stages = (p.K + SPAN - 1) / SPAN, s0 = warp * p.part, n_st = max(0, min(stages - s0, p.part));

  // stage i of the part into slot i % DEPTH: 16-byte pieces of a row, piece c at c ^ (row & 7)
  auto request = [&](int i) {
    if (i < n_st) {
#pragma unroll
      for (int q = 0; q < 4 * MT; ++q) {
        const int row = (lane >> 3) + 4 * q, c = lane & 7;
        const int64_t n = n0 + row, byte = (int64_t)(s0 + i) * 128 + 16 * c;
        const bool there = n < p.N && 2 * byte < p.K;
        copy16(ring + (i % R::DEPTH) * (MT * STAGE) + row * 128 + ((c ^ (row & 7)) << 4), p.codes + (there ? n * p.code_ld + byte : 0), there);
      }
    }
    asm volatile("cp.async.commit_group;" ::: "memory");
  };
  // the scales and zero points of stage i, G * 16 MT of each: one lane's share
  constexpr int SHARE = G * 16 * MT / 32;
  float scale[SHARE];
  uint32_t zero[SHARE];
  auto fetch = [&](int i) {
#pragma unroll
    for (int q = 0; q < SHARE; ++q) {
      const int x = lane + 32 * q, row = x / G;
      const int64_t n = n0 + row, g = (int64_t)(s0 + i) * G + x % G;
      const bool there = i < n_st && n < p.N && g < p.groups;
      scale[q] = there ? load_scalar(p.scales, p.scale_dtype, n * p.scale_ld + g) : 0.0f;
      zero[q] = there && p.zeros ? p.zeros[n * p.zero_ld + g] : 8u;
    }
  };
  auto put = [&](int i) {
#pragma unroll
    for (int q = 0; q < SHARE; ++q) {
      const int x = lane + 32 * q, row = x / G, g = x % G;
      const uint32_t less = (F16 ? 0xe400u : 0xc300u) + (zero[q] & 15u);        // -(1024 + z), -(128 + z)
      sz[(i & 1) * (MT * G * 16) + ((row >> 4) * G + g) * 16 + (row & 15)] = make_float2(scale[q], __uint_as_float(less | less << 16));
    }
  };

  asm volatile("griddepcontrol.launch_dependents;" ::: "memory");
  // with the promise that nothing in flight writes the weights their first stages are on their way before the kernels ahead have finished
  if (!p.w_static) asm volatile("griddepcontrol.wait;" ::: "memory");
#pragma unroll
  for (int i = 0; i < R::DEPTH - 1; ++i) request(i);
  fetch(0);
  if (p.w_static) asm volatile("griddepcontrol.wait;" ::: "memory");

  const int t = lane & 3, rr = lane >> 2;
  const int r = (rr >> 2) | (rr & 2) | (rr & 1) << 2;  // the lane's row of the upper eight: neighbours differ in the bits that the pieces' order uses
  const uint16_t* a_row[NT];
#pragma unroll
  for (int j = 0; j < NT; ++j) a_row[j] = p.A + (int64_t)min(m0 + 8 * j + rr, p.M - 1) * p.lda;
  float sum[MT][NT][4];
#pragma unroll
  for (int a = 0; a < MT; ++a)
#pragma unroll
    for (int j = 0; j < NT; ++j)
#pragma unroll
      for (int e = 0; e < 4; ++e) sum[a][j][e] = 0.0f;

  for (int i = 0; i < n_st; ++i) {
    put(i);
    fetch(i + 1);
    request(i + R::DEPTH - 1);
    asm volatile("cp.async.wait_group %0;" ::"n"(R::DEPTH - 1) : "memory");
    __syncwarp();                                      // every lane's pieces and scales are there
    const int k0 = (s0 + i) * SPAN, windows = min(G, (p.K - k0 + GROUP - 1) / GROUP);
    const uint8_t* slot = mine + (i % R::DEPTH) * (MT * STAGE);
    const float2* s = sz + (i & 1) * (MT * G * 16);
#pragma unroll 1
    for (int g = 0; g < windows; ++g) {
      float acc[MT][NT][4];
#pragma unroll
      for (int a = 0; a < MT; ++a)
#pragma unroll
        for (int j = 0; j < NT; ++j)
#pragma unroll
          for (int e = 0; e < 4; ++e) acc[a][j][e] = 0.0f;
      // this lane's words of its rows: GROUP / 4 codes from k0 + g GROUP + t GROUP / 4 on
      uint32_t w[MT][2][WORDS];
      float2 f[MT][2];
      const int byte = g * (GROUP / 2) + t * (GROUP / 8);
#pragma unroll
      for (int a = 0; a < MT; ++a)
#pragma unroll
        for (int u = 0; u < 2; ++u) {
          const uint8_t* at = slot + a * STAGE + (r + 8 * u) * 128 + (((byte >> 4) ^ r) << 4) + (byte & 15);
          if constexpr (WORDS == 4) { const uint4 x = *reinterpret_cast<const uint4*>(at); w[a][u][0] = x.x; w[a][u][1] = x.y; w[a][u][2] = x.z; w[a][u][3] = x.w; }
          else if constexpr (WORDS == 2) { const uint2 x = *reinterpret_cast<const uint2*>(at); w[a][u][0] = x.x; w[a][u][1] = x.y; }
          else w[a][u][0] = *reinterpret_cast<const uint32_t*>(at);
          f[a][u] = s[(a * G + g) * 16 + r + 8 * u];
        }
      const int k = k0 + g * GROUP + t * (GROUP / 4);
#pragma unroll
      for (int x = 0; x < WORDS; ++x) {
        uint4 b[NT];
        const bool there = k + 8 * x < p.K;
#pragma unroll
        for (int j = 0; j < NT; ++j) b[j] = there && m0 + 8 * j + rr < p.M ? __ldg(reinterpret_cast<const uint4*>(a_row[j] + k + 8 * x)) : make_uint4(0u, 0u, 0u, 0u);
        // A's elements in the codes' order: 0 4, 1 5, 2 6, 3 7
        uint32_t b0[NT], b1[NT], b2[NT], b3[NT];
#pragma unroll
        for (int j = 0; j < NT; ++j) {
          b0[j] = __byte_perm(b[j].x, b[j].z, 0x5410); b1[j] = __byte_perm(b[j].x, b[j].z, 0x7632);
          b2[j] = __byte_perm(b[j].y, b[j].w, 0x5410); b3[j] = __byte_perm(b[j].y, b[j].w, 0x7632);
        }
#pragma unroll
        for (int a = 0; a < MT; ++a) {
          const uint32_t up = w[a][0][x], down = w[a][1][x], lu = __float_as_uint(f[a][0].y), ld = __float_as_uint(f[a][1].y);
          const uint32_t u0 = unpack<F16, 0>(up, lu), u1 = unpack<F16, 1>(up, lu), u2 = unpack<F16, 2>(up, lu), u3 = unpack<F16, 3>(up, lu);
          const uint32_t d0 = unpack<F16, 0>(down, ld), d1 = unpack<F16, 1>(down, ld), d2 = unpack<F16, 2>(down, ld), d3 = unpack<F16, 3>(down, ld);
#pragma unroll
          for (int j = 0; j < NT; ++j) {
            mma16<F16>(acc[a][j], u0, d0, u1, d1, b0[j], b1[j]);
            mma16<F16>(acc[a][j], u2, d2, u3, d3, b2[j], b3[j]);
          }
        }
      }
#pragma unroll
      for (int a = 0; a < MT; ++a)
#pragma unroll
        for (int j = 0; j < NT; ++j)
#pragma unroll
          for (int e = 0; e < 4; ++e) sum[a][j][e] = f_fma(f[a][e >> 1].x, acc[a][j][e], sum[a][j][e]);
    }
    __syncwarp();                                      // the slot and the scales are free
  }
  asm volatile("cp.async.wait_group 0;" ::: "memory");
  __syncthreads();                                     // the rings are no longer used: the parts' sums go over them
  constexpr int COLS = 16 * MT, ROWS = 8 * NT;
  float* parts = reinterpret_cast<float*>(smem);       // [WARPS][ROWS][COLS + 1]
  static_assert(WARPS * ROWS * (COLS + 1) * 4 <= WARPS * R::WARP_BYTES, "the sums fit the rings");
#pragma unroll
  for (int a = 0; a < MT; ++a)
#pragma unroll
    for (int j = 0; j < NT; ++j)
#pragma unroll
      for (int e = 0; e < 4; ++e) parts[(warp * ROWS + 8 * j + 2 * t + (e & 1)) * (COLS + 1) + 16 * a + r + 8 * (e >> 1)] = sum[a][j][e];
  __syncthreads();
  const int n_parts = (stages + p.part - 1) / p.part;
  for (int i = threadIdx.x; i < ROWS * COLS; i += THREADS) {
    const int row = i / COLS, col = i % COLS;
    const int64_t n = n0 + col;
    if (m0 + row >= p.M || n >= p.N) continue;
    float v = parts[row * (COLS + 1) + col];
    for (int q = 1; q < n_parts; ++q) v = f_add(v, parts[(q * ROWS + row) * (COLS + 1) + col]);
    store_scalar(p.C, p.c_dtype, (int64_t)(m0 + row) * p.ldc + n, apply_epilogue(v, p.epi, m0 + row, n));
  }
}

template <bool F16, int GROUP, int MT, int NT>
cudaError_t launch(const W4Params& p, cudaStream_t st) {
  static DeviceOnce configured;
  constexpr int SMEM = WARPS * Ring4<GROUP, MT>::WARP_BYTES;
  const DeviceInfo dev = current_device();
  if (!configured.has(dev.dev)) {
    const cudaError_t e = cudaFuncSetAttribute(gemv_w4_kernel<F16, GROUP, MT, NT>, cudaFuncAttributeMaxDynamicSharedMemorySize, SMEM);
    if (e != cudaSuccess) return e;
    configured.set(dev.dev);
  }
  cudaLaunchConfig_t cfg = {};
  cfg.gridDim = dim3((unsigned)((p.N + 16 * MT - 1) / (16 * MT)), (unsigned)((p.M + 8 * NT - 1) / (8 * NT)), 1);
  cfg.blockDim = dim3(THREADS, 1, 1);
  cfg.dynamicSmemBytes = SMEM;
  cfg.stream = st;
  cudaLaunchAttribute attr[1];
  attr[0].id = cudaLaunchAttributeProgrammaticStreamSerialization;
  attr[0].val.programmaticStreamSerializationAllowed = 1;
  cfg.attrs = attr;
  cfg.numAttrs = 1;
  return cudaLaunchKernelEx(&cfg, gemv_w4_kernel<F16, GROUP, MT, NT>, p);
}
template <bool F16, int GROUP>
cudaError_t launch_rows(const W4Params& p, cudaStream_t st) {
  if (p.M <= 8) return launch<F16, GROUP, 1, 1>(p, st);
  if (p.M <= 16) return launch<F16, GROUP, 1, 2>(p, st);
  return launch<F16, GROUP, 2, 4>(p, st);
}
template <bool F16>
cudaError_t launch_group(const W4Params& p, int group, cudaStream_t st) {
  return group == 32 ? launch_rows<F16, 32>(p, st) : group == 64 ? launch_rows<F16, 64>(p, st) : launch_rows<F16, 128>(p, st);
}

}  // namespace

// All arguments were validated by the caller.
rg_status_t launch_gemv_w4(const rg_weights_four_t* W, const rg_tensor_t* A, const rg_tensor_t* C, const rg_epilogue_t* epi, cudaStream_t st) {
  W4Params p{};
  p.codes = static_cast<const uint8_t*>(W->codes); p.scales = W->scales; p.zeros = static_cast<const uint8_t*>(W->zeros);
  p.code_ld = W->code_ld; p.scale_ld = W->scale_ld; p.zero_ld = W->zero_ld; p.scale_dtype = W->scale_dtype; p.w_static = W->w_static;
  p.A = static_cast<const uint16_t*>(A->ptr); p.C = C->ptr; p.lda = A->ld; p.ldc = C->ld; p.c_dtype = C->dtype;
  p.M = (int32_t)A->rows; p.N = (int32_t)W->rows; p.K = (int32_t)W->cols;
  p.groups = (p.K + W->group - 1) / W->group;
  const int stages = (p.K + SPAN - 1) / SPAN;
  p.part = (stages + WARPS - 1) / WARPS;
  if (epi) {
    p.epi.bias = epi->bias; p.epi.bias_dtype = epi->bias_dtype; p.epi.act = epi->act;
    p.epi.residual = epi->residual; p.epi.residual_dtype = epi->residual_dtype; p.epi.ldr = epi->ldr;
  }
  const cudaError_t e = A->dtype == RG_F16 ? launch_group<true>(p, W->group, st) : launch_group<false>(p, W->group, st);
  return e == cudaSuccess ? RG_OK : RG_ERR_CUDA;
}

}  // namespace rg

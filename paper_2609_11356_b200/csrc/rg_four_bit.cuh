// Values held in four bits: the cache's format (rg_cache_four_t) and the small arithmetic on it that several kernels share.
//
// A group is 16 consecutive elements of a head: codes c in -8..7, kept as c + 8, and a scale byte b that stands for s = (8 + b % 8) 2^(b / 8 - 22).
// c s has at most 4 + 4 significant bits and is 0 or 2^-19 .. 61440 in magnitude, so it is a bf16 and an fp16 number: nothing is rounded on the way back.
// Every byte is a finite scale: what lies in unused slots cannot be an infinity or a NaN.
//
// A block (one page of one head) is a row of tiles of 8 slots, tile_bytes(dim) = 4.5 dim bytes each:
//   codes   [dim / 32][8 slots][16 bytes]       a slot's 32 elements are four words, a word's nibbles elements 0 2 4 6 1 3 5 7 of its eight
//   scales  [dim / 32][8 slots][2 bytes]
// so that any run of whole tiles is one contiguous piece, neighbouring slots' words lie side by side (threads that hold neighbouring keys read shared
// memory without conflicts), and word >> 4 i & 0x000f000f is elements 2 i and 2 i + 1 in the halves of a word.
#pragma once
#include "rg_common.cuh"

namespace rg {

constexpr int GROUP4 = 16;
__host__ __device__ constexpr int tile4_bytes(int dim) { return 9 * dim / 2; }
// a slot's word group of 32 elements (chunk) within its tile
__host__ __device__ constexpr int codes4_at(int chunk, int slot) { return (chunk * 8 + slot) * 16; }
__host__ __device__ constexpr int scales4_at(int dim, int chunk, int slot) { return 4 * dim + (chunk * 8 + slot) * 2; }

__device__ __forceinline__ float scale4(uint32_t b) { return __uint_as_float((b << 20) + (108u << 23)); }      // (1 + b % 8 / 8) 2^(b / 8 - 19)

// The smallest scale that the largest magnitude of a group reaches with 7.5 steps (the largest there is, if none does).  7.5 s is exact in fp32; the
// quotient's rounding is put right by comparing.
__device__ __forceinline__ uint32_t scale4_byte(float amax) {
  const float y = f_mul(amax, 0x1.111112p-3f);                     // amax / 7.5
  int b = (int)((__float_as_uint(y) + 0xfffffu) >> 20) - (108 << 3);
  b = min(max(b, 0), 255);
  if (b > 0 && f_mul(7.5f, scale4(b - 1)) >= amax) --b;
  else if (b < 255 && f_mul(7.5f, scale4(b)) < amax) ++b;
  return (uint32_t)b;
}

// Eight codes of 16-bit numbers, as they lie in a word, for a scale that reaches their largest magnitude; inv = 1 / s.  x inv is off by less than 2^-20 (6.04e-7,
// all eight mantissas of s and 11 bits of x gone through), so it may miss a border between two codes; it is rounded to a multiple of 2^-15 first, which puts what is next to
// a border exactly there, and then to an integer, ties to even.  That is exact: x / s is a border or at least 2^-12 from one (11 bits of x against the four of s).  The integer stands in the
// low bits of a float above 2^23 (the 8 is added there), which is multiplied to its nibble; what stands above the codes adds up to a constant.  Codes of 8
// become 7 by a minimum in front.
__device__ __forceinline__ uint32_t codes4(const float* x, float inv) {
  uint32_t w = 0u - 0x4b400000u * 0x11111111u;                     // 0x4b400000 in every nibble's place
#pragma unroll
  for (int e = 0; e < 8; ++e) {
    const float t = f_add(f_add(f_mul(x[e], inv), 384.0f), -384.0f);
    w += __float_as_uint(f_add(fminf(t, 7.25f), 12582920.0f)) << (4 * (e >> 1) + 16 * (e & 1));
  }
  return w;
}
// The same for numbers in 64 bits.  x inv is off by less than 2^-44 (1 / s by 2^-48 of it, x / s at most 7.5) and rounded to a multiple of 2^-40.
__device__ __forceinline__ uint32_t codes4(const double* x, double inv) {
  uint32_t w = 0u;
#pragma unroll
  for (int e = 0; e < 8; ++e) {
    const double t = __dadd_rn(__dadd_rn(__dmul_rn(x[e], inv), 6144.0), -6144.0);
    w |= min((uint32_t)__double2loint(__dadd_rn(t, 6755399441055752.0)), 15u) << (4 * (e >> 1) + 16 * (e & 1));      // 1.5 2^52 + 8
  }
  return w;
}
__device__ __forceinline__ double inverse4(float s) {              // 1 / s to 2^-47
  const double d = (double)s, r = (double)__frcp_rn(s);
  return __fma_rn(r, __fma_rn(-d, r, 1.0), r);
}
// The largest magnitude of eight numbers in 64 bits, as far as scale4_byte goes by it: 20 bits, the last of which stands for all that follow (7.5 s has eight
// bits).  Upper halves of doubles, which order as they do.
__device__ __forceinline__ uint32_t magnitude4(const double* x) {
  uint32_t m = 0u;
#pragma unroll
  for (int e = 0; e < 8; ++e) m = max(m, ((uint32_t)__double2hiint(x[e]) & 0x7fffffffu) | min((uint32_t)__double2loint(x[e]), 1u));
  return m;
}
__device__ __forceinline__ float magnitude4_value(uint32_t m) { return __double2float_rn(__hiloint2double((int)m, 0)); }

}  // namespace rg

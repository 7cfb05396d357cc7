// Values held in four bits: the cache's format (rg_cache_four_t) and the small arithmetic on it that several kernels share.
//
// A group is 16 consecutive elements of a head: codes c in -8..7, kept as c + 8, and a scale byte b that stands for s = (8 + b % 8) 2^(b / 8 - 22).
// c s has at most 4 + 4 significant bits and lies in 2^-22 .. 61440, so it is a bf16 and an fp16 number: nothing is rounded on the way back.
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

// The code of x, plus 8: the integer nearest to x / s, ties to even, kept within -8..7; inv = 1 / s.  The product x inv may land on the wrong side of a
// border; the remainder x - q s is exact and tells.  NaN becomes 0.  `near`: x is so close to a border that half a unit of its last place, or a few, decide.
__device__ __forceinline__ uint32_t code4(float x, float s, float inv, bool& near) {
  x = x == x ? x : 0.0f;
  const float q = rintf(fminf(fmaxf(f_mul(x, inv), -8.0f), 8.0f)), rem = f_fma(-q, s, x), half = f_mul(0.5f, s);
  near |= fabsf(f_add(fabsf(rem), -half)) <= f_mul(fabsf(x), 0x1p-22f);
  int c = (int)q;
  const bool odd = c & 1;
  if (rem > half || (odd && rem == half)) ++c;
  if (rem < -half || (odd && rem == -half)) --c;
  return (uint32_t)(min(max(c, -8), 7) + 8);
}
// Whether the scale of a group with this largest magnitude hangs on its last few bits.
__device__ __forceinline__ bool scale4_near(float amax) { return ((__float_as_uint(f_mul(amax, 0x1.111112p-3f)) + 16u) & 0xfffffu) <= 32u; }

}  // namespace rg

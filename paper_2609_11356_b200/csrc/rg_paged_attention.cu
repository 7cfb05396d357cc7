// Attention of new rows over a paged cache (rg_paged_attention).
//
// Rows of one key head, (token, query head of the group), fill the 128 lanes of a tensor-core tile; keys are walked in
// blocks of 128 places.  Per row and block, with c = scale * log2(e):
//   s_t = q . k_t                             d/16 tcgen05.mma steps from a zero accumulator, ascending
//   m'  = max_t s_t;  if (m' - m) c > 8:  a = 2^((m - m') c), m = m', l = a l, O = a O      (else m, l and O stay)
//   p_t = 2^(s_t c - m c), or 2^((s_t - m) c) where m c is large;  l += sum of p_t;  O += P V       P = p narrowed, 8 steps on the same accumulator
// and at the end O * (1 / l).  A running maximum that may lag by 2^8 costs nothing in precision (p is a floating-point number
// below 2^8) and saves nearly every rescaling of O, which lives in tensor memory.  P is narrowed because the tensor core takes two
// operands of one 16-bit type (fp16: 2^7 P, see shift_of): half a step of it on every weight, 0.0023 off in all for bf16 where 32-bit weights are
// 0.0017 off by the result's own rounding (fp16: 0.00029 and 0.00021); the sum l takes the weights before that.
//
// The sum is kept for each quarter of a block's keys (32 of them, added as a butterfly adds them) and the four are joined at the end.  All of it is one
// fixed order in both kernels below, and neither knows which other rows there are: a block that a row does not see adds exact zeros, so
// a row has the same bits as a single token, in a chunk, in any batch and on any pages.
//
// paged_attention_wide_kernel, for many rows: two tiles of 128 rows, one CTA an SM; while one tile's softmax runs the tensor core works for the other.
//   softmax (4 warps a tile)  scores from tensor memory into registers, probabilities back over them as the first operand
//                             of the next product; row r of a tile is TMEM lane r, so maxima and sums need no exchange
//   producer                  work items, page numbers, then one TMA box for each page piece (a lane each): K and V blocks into one ring
//   MMA                       S_t = Q_t K_j^T and O_t += P_t V_j for the CTA's tiles in turn
//   fixer                     hands each arrived slot to the MMA warp; in blocks where some row is masked it first turns V elements
//                             that are not finite into zeros (0 * NaN would reach every row of the tile).  For rows that do see such an element
//                             the result is put right once they are stored (rare, from global memory).
//   A chunk of 4096 rows on 16384 keys, 32 heads of 128 on 8 key heads: 0.94-0.97 ms called on rotating inputs, 1.0 PFLOP/s (0.85 ms, 1.13 PFLOP/s as a graph
//   of ten on one input).  What bounds it: 512 items on 148 SMs are
//   four turns of which the last is half empty (0.86), and a tile's chain of product, commit, 112 hardware exponentials a lane and quarter-rate
//   unit, product (about 3500 cycles for the two tiles' 2048 of the tensor core).  Tried there, as graphs: all exponentials on the hardware unit 950 us,
//   an eighth by the polynomial 896, a quarter 906-925, three eighths 985; two threads a row (16 softmax warps) 1070; scores read twice instead of held in
//   registers 1090.
// paged_attention_few_kernel, for single tokens and drafts: further down.
// The grid is persistent: the work items (sequence, tile, part, key head) are counted out of the sequences' lengths on the device, so
// nothing is read back and a captured graph follows the lengths of the day.
#include <cuda.h>

#include <algorithm>

#include "rg_common.cuh"
#include "rg_internal.h"
#include "rg_ptx.cuh"

namespace rg {

__device__ unsigned int g_paged_attn_status_word = 0;      // waits that gave up
__device__ unsigned int g_paged_attn_page_word = 0;        // pages and lengths outside the cache

namespace {

constexpr int BLK = 128;                       // keys of a block
constexpr float LAG = 8.0f;                    // how far, in powers of two, a score may exceed the running maximum
constexpr int ITEMS = 4;                       // work items that the producer can be ahead
constexpr int FLAGS = 8;                       // masked blocks' items that the fixer can be ahead of the softmax warps (below half the ring's slots)

// ---------------------------------------------------------------- PTX
__device__ __forceinline__ void pa_tma_4d(uint32_t dst, const CUtensorMap* map, int32_t x, int32_t y, int32_t z, int32_t w, uint32_t bar) {
  asm volatile("cp.async.bulk.tensor.4d.shared::cluster.global.mbarrier::complete_tx::bytes [%0], [%1, {%2, %3, %4, %5}], [%6];"
               ::"r"(dst), "l"(reinterpret_cast<uint64_t>(map)), "r"(x), "r"(y), "r"(z), "r"(w), "r"(bar) : "memory");
}
__device__ __forceinline__ void pa_fence_before() { asm volatile("tcgen05.fence::before_thread_sync;" ::: "memory"); }
__device__ __forceinline__ void pa_fence_after() { asm volatile("tcgen05.fence::after_thread_sync;" ::: "memory"); }
__device__ __forceinline__ void pa_commit(uint32_t bar) {
  asm volatile("tcgen05.commit.cta_group::1.mbarrier::arrive::one.shared::cluster.b64 [%0];" ::"r"(bar) : "memory");
}
// both operands in shared memory
__device__ __forceinline__ void pa_mma_ss(uint32_t d, uint64_t a, uint64_t b, uint32_t idesc, uint32_t acc) {
  asm volatile("{\n\t.reg .pred p;\n\tsetp.ne.b32 p, %4, 0;\n\ttcgen05.mma.cta_group::1.kind::f16 [%0], %1, %2, %3, p;\n\t}"
               ::"r"(d), "l"(a), "l"(b), "r"(idesc), "r"(acc) : "memory");
}
// first operand in tensor memory (two 16-bit elements a column)
__device__ __forceinline__ void pa_mma_ts(uint32_t d, uint32_t a, uint64_t b, uint32_t idesc, uint32_t acc) {
  asm volatile("{\n\t.reg .pred p;\n\tsetp.ne.b32 p, %4, 0;\n\ttcgen05.mma.cta_group::1.kind::f16 [%0], [%1], %2, %3, p;\n\t}"
               ::"r"(d), "r"(a), "l"(b), "r"(idesc), "r"(acc) : "memory");
}
__device__ __forceinline__ void pa_ld32(uint32_t taddr, uint32_t* r) {
  asm volatile(
      "tcgen05.ld.sync.aligned.32x32b.x32.b32 "
      "{%0, %1, %2, %3, %4, %5, %6, %7, %8, %9, %10, %11, %12, %13, %14, %15, "
      "%16, %17, %18, %19, %20, %21, %22, %23, %24, %25, %26, %27, %28, %29, %30, %31}, [%32];"
      : "=r"(r[0]), "=r"(r[1]), "=r"(r[2]), "=r"(r[3]), "=r"(r[4]), "=r"(r[5]), "=r"(r[6]), "=r"(r[7]), "=r"(r[8]), "=r"(r[9]), "=r"(r[10]),
        "=r"(r[11]), "=r"(r[12]), "=r"(r[13]), "=r"(r[14]), "=r"(r[15]), "=r"(r[16]), "=r"(r[17]), "=r"(r[18]), "=r"(r[19]), "=r"(r[20]),
        "=r"(r[21]), "=r"(r[22]), "=r"(r[23]), "=r"(r[24]), "=r"(r[25]), "=r"(r[26]), "=r"(r[27]), "=r"(r[28]), "=r"(r[29]), "=r"(r[30]), "=r"(r[31])
      : "r"(taddr) : "memory");
}
__device__ __forceinline__ void pa_st16(uint32_t taddr, const uint32_t* r) {
  asm volatile("tcgen05.st.sync.aligned.32x32b.x16.b32 [%16], {%0, %1, %2, %3, %4, %5, %6, %7, %8, %9, %10, %11, %12, %13, %14, %15};"
               ::"r"(r[0]), "r"(r[1]), "r"(r[2]), "r"(r[3]), "r"(r[4]), "r"(r[5]), "r"(r[6]), "r"(r[7]), "r"(r[8]), "r"(r[9]), "r"(r[10]),
                 "r"(r[11]), "r"(r[12]), "r"(r[13]), "r"(r[14]), "r"(r[15]), "r"(taddr) : "memory");
}
__device__ __forceinline__ void pa_st32(uint32_t taddr, const uint32_t* r) {
  asm volatile(
      "tcgen05.st.sync.aligned.32x32b.x32.b32 [%32], "
      "{%0, %1, %2, %3, %4, %5, %6, %7, %8, %9, %10, %11, %12, %13, %14, %15, "
      "%16, %17, %18, %19, %20, %21, %22, %23, %24, %25, %26, %27, %28, %29, %30, %31};"
      ::"r"(r[0]), "r"(r[1]), "r"(r[2]), "r"(r[3]), "r"(r[4]), "r"(r[5]), "r"(r[6]), "r"(r[7]), "r"(r[8]), "r"(r[9]), "r"(r[10]),
        "r"(r[11]), "r"(r[12]), "r"(r[13]), "r"(r[14]), "r"(r[15]), "r"(r[16]), "r"(r[17]), "r"(r[18]), "r"(r[19]), "r"(r[20]),
        "r"(r[21]), "r"(r[22]), "r"(r[23]), "r"(r[24]), "r"(r[25]), "r"(r[26]), "r"(r[27]), "r"(r[28]), "r"(r[29]), "r"(r[30]), "r"(r[31]), "r"(taddr)
      : "memory");
}
__device__ __forceinline__ void pa_wait_st() { asm volatile("tcgen05.wait::st.sync.aligned;" ::: "memory"); }
// The library's bounded wait, made by a whole warp and without a function call (a kernel that moves registers between its warps cannot have one).
__device__ __forceinline__ bool pa_wait(uint32_t bar, uint32_t parity, volatile int* abort_flag, uint32_t code) {
  if (__all_sync(0xffffffffu, mbar_try_wait(bar, parity))) return true;
  uint64_t t0 = 0;
  for (uint32_t turn = 1;; ++turn) {
    if (__all_sync(0xffffffffu, mbar_try_wait(bar, parity))) return true;
    if ((turn & 255u) == 0) {
      const uint64_t now = globaltimer_ns();
      if (t0 == 0) t0 = now;
      const bool late = now - t0 > WAIT_LIMIT_NS;
      if (late) { *abort_flag = 1; atomicCAS(&g_paged_attn_status_word, 0u, code); }
      if (__any_sync(0xffffffffu, late || *abort_flag)) return false;
    }
  }
}
__device__ __forceinline__ float pa_ex2(float x) {
  float y;
  asm("ex2.approx.ftz.f32 %0, %1;" : "=f"(y) : "f"(x));
  return y;
}
__device__ __forceinline__ float max3(float a, float b, float c) {
  float r;
  asm("max.NaN.f32 %0, %1, %2, %3;" : "=f"(r) : "f"(a), "f"(b), "f"(c));
  return r;
}

// 128-byte swizzled operand: rows of 128 bytes, groups of 8 rows 1024 bytes apart; `lead` is the distance between 64-element
// column groups, which only the transposed (MN-major) operand uses
__device__ __forceinline__ uint64_t pa_desc(uint32_t smem_addr, uint32_t lead) {
  uint64_t d = 0;
  d |= static_cast<uint64_t>((smem_addr & 0x3ffffu) >> 4);
  d |= static_cast<uint64_t>(lead >> 4) << 16;
  d |= static_cast<uint64_t>(1024 >> 4) << 32;
  d |= static_cast<uint64_t>(1) << 46;
  d |= static_cast<uint64_t>(2) << 61;
  return d;
}
// 16-bit x 16-bit -> fp32, M = 128, N = n; `transposed`: that operand is MN-major
__host__ __device__ constexpr uint32_t pa_idesc(int n, bool bf16, bool a_transposed, bool b_transposed) {
  return (1u << 4) | (bf16 ? (1u << 7) | (1u << 10) : 0u) | (a_transposed ? 1u << 15 : 0u) | (b_transposed ? 1u << 16 : 0u) | (static_cast<uint32_t>(n >> 3) << 17) | (8u << 24);
}

// ---------------------------------------------------------------- arguments and work items
// Division of numbers below 2^31 by a fixed one: n * ceil(2^(31 + s) / d) / 2^(31 + s), s = ceil(log2 d).  (The hardware has none: a
// division is some 40 instructions in a row, and eight of them stood in front of a single token's first copy.)
struct Div {
  uint32_t d, mul, shift;                // mul = 0: by one
  static Div by(uint32_t d) {
    uint32_t s = 0;
    while ((uint64_t(1) << s) < d) ++s;
    return {d, d > 1 ? (uint32_t)(((uint64_t(1) << (31 + s)) + d - 1) / d) : 0u, s ? s - 1 : 0u};
  }
};
__device__ __forceinline__ int32_t operator/(int32_t n, const Div& v) { return v.mul ? (int32_t)(__umulhi((uint32_t)n, v.mul) >> v.shift) : n; }

struct Params {
  const int32_t *table, *seq_lens, *cu_q;
  int64_t table_ld, max_len, tokens;
  int32_t n_seqs, page_size, pages;
  int32_t hq, hkv, group, d;
  Div by_split, by_hkv, by_hq, by_page, by_group, by_tile;   // by_tile: a CTA's tokens
  int32_t tile_tokens, cta_tokens;       // tokens of one tile: floor(rows of a tile / group); of a CTA: one tile's or two tiles'
  int32_t box;                           // keys of one TMA box
  int32_t split, segments, causal, levels;
  int32_t window;
  float scale, c;                        // c = scale * log2(e)
  void* out;
  int64_t o_tok, o_head;
  int32_t o_dtype, o_vec;
  float* lse;
  int64_t lse_ld;
  float* part_o;                         // [rows][segments][d], a row being token * hq + head
  float2* part_ml;                       // [rows][segments]
  const uint16_t* v;                     // for elements that are not finite
  int64_t v_page, v_slot, v_head;
};

struct alignas(16) Item {
  int32_t seq, head, seg;
  int32_t tok;                           // first token of the CTA's rows
  int32_t n_tok;                         // tokens of this CTA; 0: no more items
  int32_t pos;                           // place of the first one
  int32_t len, lo, hi;                   // keys some row sees, within this part: lo .. hi (hi < lo: none)
  int32_t b0, b1;                        // blocks
  int32_t multi;                         // the sequence has several parts: results go to the workspace
};
static_assert(sizeof(Item) == 48, "three 16-byte words");

// How a sequence's rows see its keys.
struct SeqView {
  int32_t tok, len, first, n;            // first row, length, place of the first row, rows
};
__device__ __forceinline__ SeqView view_of(const Params& p, int s, bool* bad) {
  SeqView v;
  const int32_t b = min(max(p.cu_q[s], 0), (int32_t)p.tokens), e = min(max(p.cu_q[s + 1], b), (int32_t)p.tokens), len = p.seq_lens[s];
  v.tok = b; v.n = e - b;
  v.len = min(max(len, 0), (int32_t)p.max_len);
  v.first = v.len - v.n;
  *bad = v.n > 0 && (v.len != len || v.first < 0);
  return v;
}
// last key that the row at `place` sees, and the first one
__device__ __forceinline__ int32_t last_seen(const Params& p, int32_t place, int32_t len) { return place < 0 ? -1 : p.causal ? place : len - 1; }
__device__ __forceinline__ int32_t first_seen(const Params& p, int32_t place) { return p.window ? max(0, place - p.window + 1) : 0; }
// parts of a sequence's rows: first one and how many
__device__ __forceinline__ void parts_of(const Params& p, const SeqView& v, int32_t* g0, int32_t* n) {
  const int32_t hi = last_seen(p, v.len - 1, v.len), lo = first_seen(p, max(v.first, 0));
  *g0 = 0; *n = 1;
  if (p.split && hi >= lo) { *g0 = lo / p.by_split; *n = hi / p.by_split - *g0 + 1; }
}

// The items of this CTA out of the list level, sequence, tile (the last, longest first), part, head.  Every CTA takes one of each gridDim.x of
// them, from the front and from the back in turn.  A level holds the tiles that see a like number of keys, the most first: work of unlike
// size then comes out even (9 prompts' chunks of 45 to 986 rows: the busiest CTA has 1.08 times the mean's work, with sequences just
// taken in turn 1.44).  Parts are alike and many sequences even out by themselves: one level.  32 sequences at a time, one a lane.  The
// producer walks the list and hands the items to the other warps in shared memory.
struct Walk {
  uint32_t next, step[2];                // number of the next item, counted from the first item of the lane group, and how far the ones after it are
  uint32_t before, count, total;         // this lane's sequence: items before it in the group, its own; the group's
  int32_t base, level, levels;           // first sequence of the group
  int32_t least, most;                   // keys of the shortest and of the longest tile, about
  uint32_t left;                         // items of the list from the next one on (levels only): behind the last none is looked for
  int32_t t_end;                         // this lane's sequence: end of its tiles of the level
  SeqView mine;                          // this lane's sequence
  // keys that tile i sees, about, and never fewer than the tile before: tiles that see fewer than x
  __device__ __forceinline__ int32_t below(const Params& p, int tile_tokens, int32_t tiles, int32_t x) const {
    const int32_t cap = p.window ? p.window + tile_tokens : INT32_MAX;
    if (!p.causal || x > cap) return x > (p.causal ? cap : mine.len) ? tiles : 0;
    return min(max(max(x - mine.first + tile_tokens - 1, 0) / p.by_tile - 1, 0), tiles);
  }
  __device__ __forceinline__ void look_up(const Params& p) {
    const int s = base + (threadIdx.x & 31);
    mine = SeqView{0, 0, 0, 0};
    if (s < p.n_seqs) {
      bool bad;
      mine = view_of(p, s, &bad);
      if (bad) atomicCAS(&g_paged_attn_page_word, 0u, (unsigned)RG_PAGE_CODE_ATTEND);
    }
  }
  __device__ __forceinline__ void load(const Params& p, int tile_tokens) {
    const int lane = threadIdx.x & 31;
    if (p.n_seqs > 32 || levels == 1) look_up(p);
    int32_t g0, n;
    parts_of(p, mine, &g0, &n);
    const int32_t tiles = (mine.n + tile_tokens - 1) / p.by_tile;
    int32_t t0 = 0;
    t_end = tiles;
    if (levels > 1 && mine.n > 0) {
      const int64_t range = (int64_t)most - least + 1;
      if (level > 0) t0 = below(p, tile_tokens, tiles, least + (int32_t)(range * level / levels));
      if (level + 1 < levels) t_end = max(t0, below(p, tile_tokens, tiles, least + (int32_t)(range * (level + 1) / levels)));
    }
    count = (uint32_t)(t_end - t0) * n * p.hkv;
    uint32_t sum = count;
#pragma unroll
    for (int x = 1; x < 32; x <<= 1) {
      const uint32_t up = __shfl_up_sync(0xffffffffu, sum, x);
      if (lane >= x) sum += up;
    }
    before = sum - count;
    total = __shfl_sync(0xffffffffu, sum, 31);
  }
  __device__ __forceinline__ void start(const Params& p, int tile_tokens) {
    most = 0;
    least = INT32_MAX;
    left = UINT32_MAX;
    levels = p.levels;
    if (levels > 1) {
      left = 0;
      for (base = 0; base < p.n_seqs; base += 32) {
        look_up(p);
        const int32_t cap = p.causal && p.window ? p.window + tile_tokens : INT32_MAX, first = p.causal ? mine.first + tile_tokens : mine.len;
        most = max(most, __reduce_max_sync(0xffffffffu, mine.n ? min(p.causal ? mine.len + tile_tokens : mine.len, cap) : 0));
        least = min(least, __reduce_min_sync(0xffffffffu, mine.n ? min(first, cap) : INT32_MAX));
        left += __reduce_add_sync(0xffffffffu, (uint32_t)((mine.n + tile_tokens - 1) / p.by_tile) * p.hkv);
      }
      least = min(least, most);
      if (left <= gridDim.x) levels = 1;                           // an item each: nothing to even out
      left -= min(left, blockIdx.x);
    }
    base = 0;
    level = levels - 1;
    next = blockIdx.x;
    step[0] = 2 * (gridDim.x - 1 - blockIdx.x) + 1;
    step[1] = 2 * blockIdx.x + 1;
    load(p, tile_tokens);
  }
  __device__ __forceinline__ bool get(const Params& p, int tile_tokens, Item& it) {
    if (left == 0) return false;
    while (next >= total) {
      next -= total;
      base += 32;
      if (base >= p.n_seqs) {
        base = 0;
        if (--level < 0) return false;
      }
      load(p, tile_tokens);
    }
    const int owner = __ffs(__ballot_sync(0xffffffffu, next >= before && next < before + count)) - 1;
    const uint32_t local = next - __shfl_sync(0xffffffffu, before, owner);
    next += step[0];
    left -= p.levels > 1 ? min(left, step[0]) : 0;
    const uint32_t swap = step[0];
    step[0] = step[1];
    step[1] = swap;
    it.seq = base + owner;
    SeqView v;
    v.tok = __shfl_sync(0xffffffffu, mine.tok, owner); v.len = __shfl_sync(0xffffffffu, mine.len, owner);
    v.n = __shfl_sync(0xffffffffu, mine.n, owner);
    v.first = v.len - v.n;
    int32_t g0, n;
    parts_of(p, v, &g0, &n);
    const int32_t rest = (int32_t)local / p.by_hkv, turn = n > 1 ? rest / n : rest;
    it.head = (int32_t)local - rest * p.hkv;
    it.seg = rest - turn * n;
    const int32_t tile = __shfl_sync(0xffffffffu, t_end, owner) - 1 - turn;
    const int32_t t0 = tile * tile_tokens;
    it.n_tok = min(tile_tokens, v.n - t0);
    it.tok = v.tok + t0;
    it.pos = v.first + t0;
    it.len = v.len;
    it.multi = n > 1;
    it.hi = last_seen(p, it.pos + it.n_tok - 1, v.len);
    it.lo = first_seen(p, max(it.pos, 0));
    it.seg += g0;
    if (p.split) {
      it.lo = max(it.lo, it.seg * p.split);
      it.hi = (int32_t)min((int64_t)it.hi, (int64_t)(it.seg + 1) * p.split - 1);
    }
    it.b0 = it.lo / BLK;
    it.b1 = it.hi >= it.lo ? it.hi / BLK + 1 : it.b0;
    return true;
  }
};

// whether some row of the item does not see all of block b
__device__ __forceinline__ bool masked_block(const Params& p, const Item& it, int b) {
  const int32_t k0 = b * BLK;
  return k0 + BLK - 1 > last_seen(p, it.pos, it.len) || (p.window && k0 < it.pos + it.n_tok - p.window);
}

// ---------------------------------------------------------------- one row, one block
// 2^x for x <= LAG + 7 or NaN by its own steps: the nearest integer by a magic addition, a polynomial of degree 5 for the rest (equal to 1
// at 0; largest relative error 1.7e-7, fitted by iteratively reweighted least squares), the integer added to the exponent; 0 below -125.
// Two at a time.  The integer sum at the end (and not a multiplication) keeps the assembler from contracting it with the addition that
// follows.  NaN comes out as some number: a row with a NaN among its scores is marked in its sum.
__device__ __forceinline__ float2 poly_ex2(float2 x) {
  const float2 magic = make_float2(12582912.0f, 12582912.0f), unmagic = make_float2(-12582912.0f, -12582912.0f);
  const float2 t = __fadd2_rn(x, magic), n = __fadd2_rn(t, unmagic);
  const float2 f = __ffma2_rn(n, make_float2(-1.0f, -1.0f), x);
  float2 q = make_float2(0x1.5bba14p-10f, 0x1.5bba14p-10f);
  q = __ffma2_rn(q, f, make_float2(0x1.3cea88p-7f, 0x1.3cea88p-7f));
  q = __ffma2_rn(q, f, make_float2(0x1.c6b752p-5f, 0x1.c6b752p-5f));
  q = __ffma2_rn(q, f, make_float2(0x1.ebf9bcp-3f, 0x1.ebf9bcp-3f));
  q = __ffma2_rn(q, f, make_float2(0x1.62e42ap-1f, 0x1.62e42ap-1f));
  q = __ffma2_rn(q, f, make_float2(1.0f, 1.0f));
  const float a = __int_as_float(__float_as_int(q.x) + (__float_as_int(t.x) << 23)), b = __int_as_float(__float_as_int(q.y) + (__float_as_int(t.y) << 23));
  return make_float2(x.x < -125.0f ? 0.0f : a, x.y < -125.0f ? 0.0f : b);
}

constexpr int QW = 32;                         // scores are taken 32 keys at a time: a quarter of a block, with a sum of its own

// A quarter of a row's scores from tensor memory; what follows cannot be moved in front of the wait.
__device__ __forceinline__ void load_quarter(uint32_t taddr, uint32_t (&s)[QW]) {
  pa_ld32(taddr, s);
  asm volatile("tcgen05.wait::ld.sync.aligned;"
               : "+r"(s[0]), "+r"(s[1]), "+r"(s[2]), "+r"(s[3]), "+r"(s[4]), "+r"(s[5]), "+r"(s[6]), "+r"(s[7]), "+r"(s[8]), "+r"(s[9]), "+r"(s[10]), "+r"(s[11]),
                 "+r"(s[12]), "+r"(s[13]), "+r"(s[14]), "+r"(s[15]), "+r"(s[16]), "+r"(s[17]), "+r"(s[18]), "+r"(s[19]), "+r"(s[20]), "+r"(s[21]), "+r"(s[22]),
                 "+r"(s[23]), "+r"(s[24]), "+r"(s[25]), "+r"(s[26]), "+r"(s[27]), "+r"(s[28]), "+r"(s[29])
               :: "memory");
  asm volatile("" : "+r"(s[30]), "+r"(s[31]) :: "memory");
}

// Waits for loads from tensor memory; what uses a row's scores cannot be moved in front of the wait.
__device__ __forceinline__ void wait_scores(uint32_t (&s)[BLK]) {
  asm volatile("tcgen05.wait::ld.sync.aligned;" ::: "memory");
#pragma unroll
  for (int i = 0; i < BLK; i += 16)
    asm volatile("" : "+r"(s[i]), "+r"(s[i + 1]), "+r"(s[i + 2]), "+r"(s[i + 3]), "+r"(s[i + 4]), "+r"(s[i + 5]), "+r"(s[i + 6]), "+r"(s[i + 7]), "+r"(s[i + 8]),
                 "+r"(s[i + 9]), "+r"(s[i + 10]), "+r"(s[i + 11]), "+r"(s[i + 12]), "+r"(s[i + 13]), "+r"(s[i + 14]), "+r"(s[i + 15]));
}

// The largest of a quarter's scores, NaN if one is.
__device__ __forceinline__ float quarter_max(const uint32_t* s) {
  float a = __uint_as_float(s[0]), b = __uint_as_float(s[1]);
#pragma unroll
  for (int i = 2; i + 3 < QW; i += 4) { a = max3(a, __uint_as_float(s[i]), __uint_as_float(s[i + 1])); b = max3(b, __uint_as_float(s[i + 2]), __uint_as_float(s[i + 3])); }
  a = max3(a, __uint_as_float(s[QW - 2]), __uint_as_float(s[QW - 1]));
  return max3(a, b, b);
}

// Whether the block's maximum mb moves the running one (from -inf: any number does; -inf and NaN never), and the factor that sums and O take then.
__device__ __forceinline__ bool rises(float m, float mb, float c) { return f_mul(f_add(mb, -m), c) > LAG; }
__device__ __forceinline__ float move_max(float& m, float mb, float c) {
  const float alpha = pa_ex2(f_mul(f_add(m, -mb), c));
  m = mb;
  return alpha;
}
// What a row's scores take on the way to their exponents: x = (s - off) c + shift.  The product m c is rounded once for all of a row's keys, and what it
// is off by, up to half its last place, multiplies every weight: nothing while it is below 2^-8, but at 2^31 weights pass fp16's range or
// vanish, and from 2^128 on there is no product.  Rows that far out take their maximum off first; s - m is exact where it matters.
// In fp16 all weights of a row, its sum and O are 2^7 times as large until the end (below 2^15, the maximum's lag included): a weight's half step is then 2^-32
// of the largest weight or less and not 2^-25, which lost everything below that: 60000 keys of weight 2^-26 next to one of 1 are a thousandth of the result.
constexpr float FAR = 65536.0f;
template <int DT> constexpr float UP = DT == RG_F16 ? 7.0f : 0.0f;
template <int DT> constexpr float DOWN = DT == RG_F16 ? 0x1p-7f : 1.0f;
template <int DT>
__device__ __forceinline__ bool shift_of(float m, float c, float& shift, float& off) {
  shift = m == -INFINITY ? 0.0f : -f_mul(m, c);
  off = 0.0f;
  const bool far = fabsf(shift) >= FAR && m != INFINITY;       // an infinite maximum: the row is NaN
  if (far) { off = m; shift = 0.0f; }
  if (DT == RG_F16) shift = f_add(shift, UP<DT>);
  return far;
}

// The exponentials of two scores.  Which of the two forms a key takes follows from its place alone: the last 4 of every 32 the polynomial,
// which takes them off the hardware unit (16 results a cycle and SM, where a block of both tiles wants 32768 in 2048 cycles of the tensor core).
constexpr int POLY_FROM = 28;
template <bool POLY>
__device__ __forceinline__ float2 prob2(float2 s, float c, float shift0, float shift1) {
  const float2 x = __ffma2_rn(s, make_float2(c, c), make_float2(shift0, shift1));
  return POLY ? poly_ex2(x) : make_float2(pa_ex2(x.x), pa_ex2(x.y));
}

// Probabilities of a quarter, narrowed two to a word (masked scores are -inf and give exact zeros); returns their fp32 sum, in the order of a
// butterfly over the 32 keys: key with key + 16 first, neighbours last.
template <int DT>
__device__ __forceinline__ float quarter_probs(const uint32_t* s, uint32_t* packed, float c, float shift) {
  float2 t[8];
#pragma unroll
  for (int i = 0; i < 8; ++i) {
    const int j = i + 8;
    const float2 a = prob2<false>(make_float2(__uint_as_float(s[2 * i]), __uint_as_float(s[2 * i + 1])), c, shift, shift);
    const float2 sj = make_float2(__uint_as_float(s[2 * j]), __uint_as_float(s[2 * j + 1]));
    const float2 b = 2 * j >= POLY_FROM ? prob2<true>(sj, c, shift, shift) : prob2<false>(sj, c, shift, shift);
    packed[i] = pack_16x2(a.x, a.y, DT);
    packed[j] = pack_16x2(b.x, b.y, DT);
    t[i] = __fadd2_rn(a, b);
  }
#pragma unroll
  for (int n = 4; n >= 1; n >>= 1)
#pragma unroll
    for (int i = 0; i < n; ++i) t[i] = __fadd2_rn(t[i], t[i + n]);
  return f_add(t[0].x, t[0].y);
}
// A quarter's running sum.  A NaN or an infinity among the block's scores makes the row NaN; nothing above -inf so far: no sum.
__device__ __forceinline__ float add_quarter(float l, float alpha, float total, float m, float mb) {
  total = mb != mb || mb == INFINITY ? __int_as_float(0x7fffffff) : m == -INFINITY ? 0.0f : total;
  return f_fma(l, alpha, total);
}
__device__ __forceinline__ float join_quarters(float a, float b, float c, float d) { return f_add(f_add(a, b), f_add(c, d)); }

template <int N>
__device__ __forceinline__ void pa_ld_cols(uint32_t taddr, uint32_t (&r)[N]);
template <>
__device__ __forceinline__ void pa_ld_cols<8>(uint32_t taddr, uint32_t (&r)[8]) {
  asm volatile("tcgen05.ld.sync.aligned.32x32b.x8.b32 {%0, %1, %2, %3, %4, %5, %6, %7}, [%8];\n\ttcgen05.wait::ld.sync.aligned;"
               : "=r"(r[0]), "=r"(r[1]), "=r"(r[2]), "=r"(r[3]), "=r"(r[4]), "=r"(r[5]), "=r"(r[6]), "=r"(r[7]) : "r"(taddr) : "memory");
}
template <>
__device__ __forceinline__ void pa_ld_cols<16>(uint32_t taddr, uint32_t (&r)[16]) {
  asm volatile("tcgen05.ld.sync.aligned.32x32b.x16.b32 {%0, %1, %2, %3, %4, %5, %6, %7, %8, %9, %10, %11, %12, %13, %14, %15}, [%16];\n\ttcgen05.wait::ld.sync.aligned;"
               : "=r"(r[0]), "=r"(r[1]), "=r"(r[2]), "=r"(r[3]), "=r"(r[4]), "=r"(r[5]), "=r"(r[6]), "=r"(r[7]), "=r"(r[8]), "=r"(r[9]), "=r"(r[10]),
                 "=r"(r[11]), "=r"(r[12]), "=r"(r[13]), "=r"(r[14]), "=r"(r[15]) : "r"(taddr) : "memory");
}
template <>
__device__ __forceinline__ void pa_ld_cols<32>(uint32_t taddr, uint32_t (&r)[32]) { load_quarter(taddr, r); }
template <int N>
__device__ __forceinline__ void pa_st_cols(uint32_t taddr, const uint32_t (&r)[N]) {
  if constexpr (N == 32) pa_st32(taddr, r);
  else if constexpr (N == 16) pa_st16(taddr, r);
  else
    asm volatile("tcgen05.st.sync.aligned.32x32b.x8.b32 [%8], {%0, %1, %2, %3, %4, %5, %6, %7};"
                 ::"r"(r[0]), "r"(r[1]), "r"(r[2]), "r"(r[3]), "r"(r[4]), "r"(r[5]), "r"(r[6]), "r"(r[7]), "r"(taddr) : "memory");
}

// O = alpha O for one lane's columns (16 at a time: half of a row's scores are in registers meanwhile, and 32 made the compiler spill some)
template <int HDP>
__device__ __forceinline__ void rescale(uint32_t t_o, float alpha) {
#pragma unroll 1
  for (int q = 0; q < HDP / 16; ++q) {
    uint32_t o[16];
    pa_ld_cols<16>(t_o + 16u * q, o);
#pragma unroll
    for (int i = 0; i < 16; ++i) o[i] = __float_as_uint(f_mul(__uint_as_float(o[i]), alpha));
    pa_st16(t_o + 16u * q, o);
  }
}

// Which 16-bit elements of two words are not finite, a bit each at 15 and 31.
template <int DT>
__device__ __forceinline__ uint32_t not_finite_in(uint32_t x) {
  constexpr uint32_t EXP = DT == RG_BF16 ? 0x7f807f80u : 0x7c007c00u, ONE = DT == RG_BF16 ? 0x00800080u : 0x04000400u;      // exponent fields, and what makes a full one carry
  return ((x & EXP) + ONE) & 0x80008000u;
}

// The fixer's work on a block of V in shared memory (n 16-byte words, 128-byte rows of 64 elements, box after box): elements that are not finite
// become zero.  Whether one of them belongs to a key of lo .. hi.
template <int DT>
__device__ __forceinline__ bool fix_values(uint4* base, uint32_t n, int32_t key0, int32_t lo, int32_t hi) {
  bool seen = false;
#pragma unroll 4
  for (uint32_t i = threadIdx.x & 31; i < n; i += 32) {
    uint4 w = base[i];
    if (not_finite_in<DT>(w.x) | not_finite_in<DT>(w.y) | not_finite_in<DT>(w.z) | not_finite_in<DT>(w.w)) {
      auto clean = [&](uint32_t x) { return x & ~((not_finite_in<DT>(x) >> 15) * 0xffffu); };
      w.x = clean(w.x); w.y = clean(w.y); w.z = clean(w.z); w.w = clean(w.w);
      base[i] = w;
      const int32_t key = key0 + (int32_t)(i / 8 % BLK);
      seen |= key >= lo && key <= hi;
    }
  }
  asm volatile("fence.proxy.async.shared::cta;" ::: "memory");
  return __any_sync(0xffffffffu, seen);
}

// A key's values for one key head, or null where its page is not in the cache.
__device__ __forceinline__ const uint16_t* value_row(const Params& p, const Item& it, int32_t key) {
  const int32_t page = key / p.by_page;
  const int64_t id = p.table[(int64_t)it.seq * p.table_ld + page];
  return id < 0 || id >= p.pages ? nullptr : p.v + id * p.v_page + (int64_t)(key - page * p.page_size) * p.v_slot + it.head * p.v_head;
}

// Elements of O for which a row sees an element of V that is not finite are made anew once the rest is stored, from global memory: the sum of those
// elements (an infinity, or NaN).  The product does not do: in a block that is masked for its tile the fixer has taken them out, in any other they were
// multiplied by a weight that may have come out as 0 (NaN for an infinity), and which of the two a block is depends on the rows that came with this one.
// The warp goes through columns 32 q .. 32 q + 31 of V, 32 keys at a time, in masked blocks only or in `all`.  A lane first holds a key, the kinds of its
// elements as a bit for each column, then a row, which sees keys lo .. hi (none: lo > hi) and has its results from `at` on in the output or in a part.
// 0.8 us for 32 keys and 32 columns, 4 where every value is infinite (the 4096-row chunk takes 6 ms with one infinity, 28 with nothing else, 1 with NaN
// alone); the waits of the other warps, 2 s, allow for four million keys of infinities in a part.
template <int DT>
__device__ __forceinline__ void put_odd_values(const Params& p, const Item& it, bool all, int q, int32_t lo, int32_t hi, bool writes, int64_t at) {
  const int n = min(QW, p.d - 32 * q);
  const uint32_t full = n == 32 ? 0xffffffffu : (1u << n) - 1;
  uint32_t up = 0, down = 0, nan = 0;                              // the row's columns that see an infinity, a negative one, a NaN
#pragma unroll 1
  for (int32_t k0 = it.lo & ~31; k0 <= it.hi; k0 += 32) {
    if (!all && !masked_block(p, it, k0 / BLK)) continue;
    const int32_t key = k0 + (threadIdx.x & 31);
    const uint16_t* v = key >= it.lo && key <= it.hi ? value_row(p, it, key) : nullptr;
    uint32_t hit = 0, key_up = 0, key_down = 0, key_nan = 0;
#pragma unroll
    for (int w = 0; w < QW / 8; ++w) {
      const uint4 x = v && w < n / 8 ? *reinterpret_cast<const uint4*>(v + 32 * q + 8 * w) : make_uint4(0u, 0u, 0u, 0u);
      hit |= not_finite_in<DT>(x.x) | not_finite_in<DT>(x.y) | not_finite_in<DT>(x.z) | not_finite_in<DT>(x.w);
    }
#pragma unroll 1
    for (int w = 0; hit && w < n / 8; ++w) {
      const uint4 x = *reinterpret_cast<const uint4*>(v + 32 * q + 8 * w);
      const uint32_t word[4] = {x.x, x.y, x.z, x.w};
#pragma unroll
      for (int i = 0; i < 4; ++i) {
        const uint32_t odd = not_finite_in<DT>(word[i]);
        if (!odd) continue;
#pragma unroll
        for (int half = 0; half < 2; ++half) {
          if (!(odd >> (15 + 16 * half) & 1u)) continue;
          const uint32_t e = word[i] >> (16 * half) & 0xffffu, bit = 1u << (8 * w + 2 * i + half);
          if (e & (DT == RG_BF16 ? 0x7fu : 0x3ffu)) key_nan |= bit;
          else if (e >> 15) key_down |= bit;
          else key_up |= bit;
        }
      }
    }
#pragma unroll 1
    for (uint32_t left = __ballot_sync(0xffffffffu, (key_up | key_down | key_nan) != 0); left; left &= left - 1) {
      const int lane = __ffs(left) - 1;
      const uint32_t a = __shfl_sync(0xffffffffu, key_up, lane), b = __shfl_sync(0xffffffffu, key_down, lane), c = __shfl_sync(0xffffffffu, key_nan, lane);
      if (k0 + lane >= lo && k0 + lane <= hi) { up |= a; down |= b; nan |= c; }
    }
    if (!__any_sync(0xffffffffu, lo <= hi && (nan | (up & down)) != full)) break;      // NaN everywhere: nothing changes any more
  }
  __syncwarp();                                                    // the elements were stored before, by other lanes or as parts of words
  asm volatile("" ::: "memory");
  void* base = it.multi ? static_cast<void*>(p.part_o) : p.out;
  nan |= up & down;
#pragma unroll 1
  for (uint32_t left = writes ? up | down | nan : 0u; left; left &= left - 1) {
    const int i = __ffs(left) - 1;
    store_scalar(base, it.multi ? (int)RG_F32 : p.o_dtype, at + 32 * q + i, nan >> i & 1u ? __int_as_float(0x7fffffff) : up >> i & 1u ? INFINITY : -INFINITY);
  }
}

// A position in a ring of N barriers.
template <int N>
struct Ring {
  uint32_t slot = 0, phase = 0;
  __device__ __forceinline__ void step() { if (++slot == N) { slot = 0; phase ^= 1u; } }
};

// ---------------------------------------------------------------- the kernel for many rows
template <int HDP>
struct Wide {
  static constexpr int DB = HDP / 64;                              // 64-column boxes of a head
  static constexpr int NT = 2, SOFT = 4 * NT;                      // tiles of 128 rows, softmax warps
  static constexpr int PRODUCER = SOFT, MMA = SOFT + 1, FIXER = SOFT + 2, WARPS = SOFT + 3, THREADS = (SOFT + 4) * 32;   // the last warp does nothing
  static constexpr uint32_t Q_BOX = 128 * 128, Q_TILE = DB * Q_BOX;
  static constexpr uint32_t KV_BOX = BLK * 128, SLOT = DB * KV_BOX;
  static constexpr int SLOTS = HDP == 128 ? 5 : 10;
  static constexpr uint32_t COLS = 512;                            // tensor memory: S_t, and P_t over it, at 128 t, O_t at 128 (2 + t)
  static constexpr uint32_t KV_AT = NT * Q_TILE, ITEM_AT = KV_AT + SLOTS * SLOT, BAR_AT = ITEM_AT + ITEMS * sizeof(Item), N_BAR = 12 + 3 * SLOTS + 2 * ITEMS,
                            FLAG_AT = BAR_AT + 8 * N_BAR, LAST = FLAG_AT + 4 * (2 + FLAGS);
  static constexpr size_t SMEM = 1024 + LAST;
  static_assert(SMEM <= 232448 && SLOTS / 2 + 1 < FLAGS, "fits the SM; the fixer cannot be a whole turn of flags ahead");
};

template <int HDP, int DT>
__global__ void __launch_bounds__(Wide<HDP>::THREADS, 1)
paged_attention_wide_kernel(const __grid_constant__ CUtensorMap tmap_q, const __grid_constant__ CUtensorMap tmap_k, const __grid_constant__ CUtensorMap tmap_v,
                       const __grid_constant__ Params p) {
  using F = Wide<HDP>;
  constexpr int DB = F::DB, SLOTS = F::SLOTS, NT = F::NT;
  constexpr uint32_t IDESC_S = pa_idesc(BLK, DT == RG_BF16, false, false), IDESC_O = pa_idesc(HDP, DT == RG_BF16, false, true);

  extern __shared__ uint8_t smem_raw[];
  const uint32_t smem_base = (smem_u32(smem_raw) + 1023u) & ~1023u;
  uint8_t* smem_gen = smem_raw + (smem_base - smem_u32(smem_raw));
  const uint32_t sQ = smem_base, sKV = smem_base + F::KV_AT;
  Item* items = reinterpret_cast<Item*>(smem_gen + F::ITEM_AT);
  const uint32_t bar0 = smem_base + F::BAR_AT;
  const uint32_t b_q_full = bar0, b_q_empty = bar0 + 8, b_s = bar0 + 16, b_o_full = bar0 + 32, b_o_empty = bar0 + 48, b_p = bar0 + 64, b_full = bar0 + 96;   // one a tile from b_s on; b_p: and half of the keys
  const uint32_t b_ready = b_full + 8 * SLOTS, b_empty = b_ready + 8 * SLOTS, b_item = b_empty + 8 * SLOTS, b_free = b_item + 8 * ITEMS;
  uint32_t* tmem_slot = reinterpret_cast<uint32_t*>(smem_gen + F::FLAG_AT);
  volatile int* abort_flag = reinterpret_cast<volatile int*>(tmem_slot + 1);
  volatile int* not_finite = reinterpret_cast<volatile int*>(tmem_slot + 2);          // [FLAGS]

  const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
  if (threadIdx.x == 0) {
    mbar_init(b_q_full, 1); mbar_init(b_q_empty, 1);
    for (int t = 0; t < 2; ++t) { mbar_init(b_s + 8 * t, 1); mbar_init(b_p + 16 * t, 4); mbar_init(b_p + 16 * t + 8, 4); mbar_init(b_o_full + 8 * t, 1); mbar_init(b_o_empty + 8 * t, 4); }
    for (int s = 0; s < SLOTS; ++s) { mbar_init(b_full + 8 * s, 1); mbar_init(b_ready + 8 * s, 1); mbar_init(b_empty + 8 * s, 1); }
    for (int s = 0; s < ITEMS; ++s) { mbar_init(b_item + 8 * s, 1); mbar_init(b_free + 8 * s, F::WARPS - 1); }
    *abort_flag = 0;
    asm volatile("fence.mbarrier_init.release.cluster;" ::: "memory");
  }
  if (warp == F::MMA) {
    asm volatile("tcgen05.alloc.cta_group::1.sync.aligned.shared::cta.b32 [%0], %1;" ::"r"(smem_u32(tmem_slot)), "r"(F::COLS) : "memory");
    asm volatile("tcgen05.relinquish_alloc_permit.cta_group::1.sync.aligned;" ::: "memory");
  }
  pa_fence_before();
  __syncthreads();
  pa_fence_after();
  const uint32_t tmem = *tmem_slot;
  asm volatile("griddepcontrol.wait;" ::: "memory");               // the set-up ran under the tail of the kernel in front; from here on its results are read
  if (p.segments > 1) asm volatile("griddepcontrol.launch_dependents;" ::: "memory");
  const int cta_tokens = p.cta_tokens;

  // Next item, for the warps that get it from the producer; false: none left, or a wait gave up.
  Ring<ITEMS> ir;
  auto next_item = [&](Item& it, bool& alive) -> bool {
    if (!pa_wait(b_item + 8 * ir.slot, ir.phase, abort_flag, 0x2000u)) { alive = false; return false; }
    it = items[ir.slot];
    __syncwarp();
    if (lane == 0) mbar_arrive(b_free + 8 * ir.slot);
    ir.step();
    return it.n_tok > 0;
  };
  Item it;
  bool alive = true;
  // A softmax thread holds a row's 128 scores: its warps take registers from the other four (168 a thread at launch: 2 * 216 + 72 = 3 * 168).
  if (warp >= F::SOFT) {
  asm volatile("setmaxnreg.dec.sync.aligned.u32 72;");
  if (warp == F::PRODUCER) {
    // ------------------------------------------------------------ producer
    const int pieces = BLK / p.box;                                // TMA boxes along the keys of a block
    const int piece = lane & (pieces - 1), col = lane / pieces;          // col < DB: this lane issues a box
    Ring<SLOTS> kv;
    uint32_t q_phase = 1;
    Walk walk;
    walk.start(p, cta_tokens);
    while (alive) {
      const bool more = walk.get(p, cta_tokens, it);
      if (!more) it.n_tok = 0;
      alive = pa_wait(b_free + 8 * ir.slot, ir.phase ^ 1u, abort_flag, 0x2080u);
      if (!alive) break;
      if (lane == 0) { items[ir.slot] = it; mbar_arrive(b_item + 8 * ir.slot); }
      ir.step();
      if (!more) break;
      if (it.b1 == it.b0) continue;
      const int32_t* row = p.table + (int64_t)it.seq * p.table_ld;
      auto wanted = [&](int b) -> bool { const int32_t k = b * BLK + piece * p.box; return col < DB && k <= it.hi && k + p.box > it.lo; };
      auto entry = [&](int b) -> int32_t { return row[(b * BLK + piece * p.box) / p.by_page]; };
      int32_t ahead = wanted(it.b0) ? entry(it.b0) : 0;
      alive = pa_wait(b_q_empty, q_phase, abort_flag, 0x2100u);
      if (!alive) break;
      q_phase ^= 1u;
      const int tiles = it.n_tok > p.tile_tokens ? 2 : 1;
      if (lane == 0) mbar_expect_tx(b_q_full, (uint32_t)(tiles * DB * p.tile_tokens * p.group) * 128u);
      __syncwarp();
      if (lane < tiles * DB) {
        const int t = lane / DB, b = lane % DB;
        pa_tma_4d(sQ + t * F::Q_TILE + b * F::Q_BOX, &tmap_q, b * 64, 0, it.tok + t * p.tile_tokens, it.head, b_q_full);
      }
      for (int b = it.b0; b < it.b1 && alive; ++b) {
        const bool mine = wanted(b);
        int32_t page = ahead;
        if (b + 1 < it.b1 && wanted(b + 1)) ahead = entry(b + 1);  // looked up a block ahead of its use
        if (mine && (page < 0 || page >= p.pages)) {               // not a page: the copy from behind the last one fills in zeros
          if (col == 0) atomicCAS(&g_paged_attn_page_word, 0u, (unsigned)RG_PAGE_CODE_ATTEND);
          page = p.pages;
        }
        const int32_t key = b * BLK + piece * p.box, at = key - key / p.by_page * p.page_size;
        const uint32_t bytes = (uint32_t)__popc(__ballot_sync(0xffffffffu, mine)) * (uint32_t)p.box * 128u;
#pragma unroll
        for (int which = 0; which < 2; ++which) {
          alive = pa_wait(b_empty + 8 * kv.slot, kv.phase ^ 1u, abort_flag, 0x2200u | kv.slot);
          if (!alive) break;
          if (lane == 0) mbar_expect_tx(b_full + 8 * kv.slot, bytes);
          __syncwarp();
          if (mine) pa_tma_4d(sKV + kv.slot * F::SLOT + col * F::KV_BOX + piece * p.box * 128, which ? &tmap_v : &tmap_k, col * 64, at, it.head, page, b_full + 8 * kv.slot);
          kv.step();
        }
      }
    }
  } else if (warp == F::MMA) {
    // ------------------------------------------------------------ MMA issuer: the warp walks converged, an elected lane issues
    const bool leader = elect_one();
    Ring<SLOTS> kv;
    uint32_t q_phase = 0, p_phase[2] = {0, 0}, o_phase[2] = {1, 1};
    // Waits for the next slot; its address comes out warp-uniform, so that the descriptors stay in uniform registers.
    auto next_slot = [&](uint32_t& bar) -> uint32_t {
      const uint32_t slot = __shfl_sync(0xffffffffu, kv.slot, 0);
      alive = pa_wait(b_ready + 8 * slot, kv.phase, abort_flag, 0x2300u | slot);
      if (alive) alive = pa_wait(b_full + 8 * slot, kv.phase, abort_flag, 0x2380u | slot);
      pa_fence_after();
      bar = b_empty + 8 * slot;
      kv.step();
      return __shfl_sync(0xffffffffu, sKV + slot * F::SLOT, 0);
    };
    auto scores = [&](int t, uint32_t sK) {
#pragma unroll
      for (int b = 0; b < DB; ++b) {
        const uint64_t a = pa_desc(sQ + t * F::Q_TILE + b * F::Q_BOX, 16), k = pa_desc(sK + b * F::KV_BOX, 16);
#pragma unroll
        for (int e = 0; e < 4; ++e) if (leader) pa_mma_ss(tmem + 128u * t, a + 2u * e, k + 2u * e, IDESC_S, (b | e) ? 1u : 0u);
      }
      if (leader) pa_commit(b_s + 8 * t);
    };
    while (alive && next_item(it, alive)) {
      const int nb = __shfl_sync(0xffffffffu, it.b1 - it.b0, 0);
      if (nb == 0) continue;
      const int tiles = __shfl_sync(0xffffffffu, it.n_tok, 0) > p.tile_tokens ? 2 : 1;
      alive = pa_wait(b_q_full, q_phase, abort_flag, 0x2400u);
      q_phase ^= 1u;
      if (!alive) break;
      uint32_t k_bar, v_bar, sK = next_slot(k_bar);
      if (!alive) break;
      for (int t = 0; t < tiles; ++t) scores(t, sK);
      if (leader) { pa_commit(k_bar); if (nb == 1) pa_commit(b_q_empty); }
      for (int j = 0; j < nb && alive; ++j) {
        const bool more = j + 1 < nb;
        const uint32_t sV = next_slot(v_bar);
        if (!alive) break;
#pragma unroll
        for (int t = 0; t < NT; ++t) {
          if (t >= tiles) break;
          alive = pa_wait(b_p + 16 * t, p_phase[t], abort_flag, 0x2500u | t);
          if (alive && j == 0) { alive = pa_wait(b_o_empty + 8 * t, o_phase[t], abort_flag, 0x2580u | t); o_phase[t] ^= 1u; }
          if (!alive) break;
          pa_fence_after();
          const uint64_t v = pa_desc(sV, F::KV_BOX);
#pragma unroll
          for (int half = 0; half < 2; ++half) {                   // the first 64 keys' product runs while the others' probabilities are computed
            if (half) { alive = pa_wait(b_p + 16 * t + 8, p_phase[t], abort_flag, 0x2540u | t); p_phase[t] ^= 1u; if (!alive) break; pa_fence_after(); }
#pragma unroll
            for (int e = 0; e < 4; ++e)
              if (leader) pa_mma_ts(tmem + 128u * (NT + t), tmem + 128u * t + 32u * half + 8u * e, v + (uint64_t)((4 * half + e) * (2048 >> 4)), IDESC_O, (j | half | e) ? 1u : 0u);
          }
          if (!alive) break;
          if (!more && leader) pa_commit(b_o_full + 8 * t);
          if (more) {
            if (t == 0) sK = next_slot(k_bar);
            if (!alive) break;
            scores(t, sK);
          }
        }
        if (!alive) break;
        if (leader) {
          pa_commit(v_bar);
          if (more) pa_commit(k_bar);
          if (j + 2 == nb) pa_commit(b_q_empty);
        }
      }
    }
  } else if (warp == F::FIXER) {
    // ------------------------------------------------------------ fixer
    Ring<SLOTS> kv;
    uint32_t flags = 0;
    while (alive && next_item(it, alive)) {
      bool any_masked = false;
      for (int b = it.b0; b < it.b1 && alive; ++b) {
        const bool masked = masked_block(p, it, b);
#pragma unroll
        for (int which = 0; which < 2; ++which) {
          alive = pa_wait(b_full + 8 * kv.slot, kv.phase, abort_flag, 0x2600u | kv.slot);
          if (!alive) break;
          if (which == 1 && masked) {
            const bool seen = fix_values<DT>(reinterpret_cast<uint4*>(smem_gen + F::KV_AT + kv.slot * F::SLOT), F::SLOT / 16, b * BLK, it.lo, it.hi);
            if (lane == 0) not_finite[flags % FLAGS] = any_masked ? (not_finite[flags % FLAGS] | (seen ? 1 : 0)) : (seen ? 1 : 0);
            any_masked = true;
          }
          __syncwarp();
          if (lane == 0) mbar_arrive(b_ready + 8 * kv.slot);
          kv.step();
        }
      }
      if (any_masked) ++flags;
    }
  }
  } else {
    // ------------------------------------------------------------ softmax and output rows
    asm volatile("setmaxnreg.inc.sync.aligned.u32 216;");
    const int t = warp >> 2;                                       // tile
    const int r = (warp & 3) * 32 + lane;                          // row of the tile, and its lane in tensor memory
    const uint32_t t_s = tmem + (static_cast<uint32_t>((warp & 3) * 32) << 16) + 128u * t, t_o = t_s + 128u * NT;
    const int my_tok = r / p.by_group, my_head = r - my_tok * p.group;
    uint32_t s_phase = 0, o_phase = 0, flags = 0;
    while (alive && next_item(it, alive)) {
      const int tok = t * p.tile_tokens + my_tok;                  // within the item
      const bool live = my_tok < p.tile_tokens && tok < it.n_tok;
      const bool warp_live = __any_sync(0xffffffffu, live);
      const bool tile_live = t * p.tile_tokens < it.n_tok;
      const int32_t place = it.pos + tok;
      const int32_t hi = live ? min(last_seen(p, place, it.len), it.hi) : -1, lo = max(first_seen(p, place), it.lo);
      float m = -INFINITY, l[4] = {0.0f, 0.0f, 0.0f, 0.0f}, shift = 0.0f;
      bool far = false;
      bool any_masked = masked_block(p, it, it.b0) && it.b1 > it.b0;
      if (it.b1 > it.b0 + 1) any_masked |= masked_block(p, it, it.b1 - 1);      // what is masked lies at the ends
      if (tile_live) {
        for (int b = it.b0; b < it.b1; ++b) {
          const bool masked = masked_block(p, it, b);
          alive = pa_wait(b_s + 8 * t, s_phase, abort_flag, 0x2700u | t);
          if (!alive) break;
          const int first = lo - b * BLK, last = hi - b * BLK;     // columns of the block that the row sees
          pa_fence_after();
          if (warp_live) {
            uint32_t s[BLK];
#pragma unroll
            for (int q = 0; q < 4; ++q) pa_ld32(t_s + 32u * q, s + 32 * q);
            wait_scores(s);
            if (masked) {
#pragma unroll
              for (int i = 0; i < BLK; ++i) s[i] = i >= first && i <= last ? s[i] : 0xff800000u;
            }
            const float mb = max3(max3(quarter_max(s), quarter_max(s + 32), quarter_max(s + 64)), quarter_max(s + 96), -INFINITY);
            // rare, and in one branch: the maximum moves, or the row is far (as a branch of its own behind the maximum's, the far rows took 3 % of a long chunk)
            const bool up = rises(m, mb, p.c), moved = __any_sync(0xffffffffu, up || far);
            float alpha = 1.0f;
            if (moved) {
              if (up) alpha = move_max(m, mb, p.c);
              float off;
              far = shift_of<DT>(m, p.c, shift, off);
              if (far) {
#pragma unroll
                for (int i = 0; i < BLK; ++i) s[i] = __float_as_uint(f_add(__uint_as_float(s[i]), -off));
              }
            }
            // probabilities go over scores, which have been read
#pragma unroll
            for (int q = 0; q < 4; ++q) {
              uint32_t packed[QW / 2];
              l[q] = add_quarter(l[q], alpha, quarter_probs<DT>(s + 32 * q, packed, p.c, shift), m, mb);
              pa_st16(t_s + 16u * q, packed);
              if (q == 1) {
                // the scores of this block are complete, so the product of the block before is too: O may be rescaled
                if (moved && b > it.b0) rescale<HDP>(t_o, alpha);
                pa_wait_st();
                pa_fence_before();
                __syncwarp();
                if (lane == 0) mbar_arrive(b_p + 16 * t);
              }
            }
            pa_wait_st();
            pa_fence_before();
          } else if (lane == 0) {
            mbar_arrive(b_p + 16 * t);
          }
          s_phase ^= 1u;
          __syncwarp();
          if (lane == 0) mbar_arrive(b_p + 16 * t + 8);
        }
        if (!alive) break;
      }
      const int slot_flag = flags % FLAGS;
      if (any_masked) ++flags;
      if (!tile_live) continue;
      const bool blocks = it.b1 > it.b0;
      const float sum = join_quarters(l[0], l[1], l[2], l[3]);
      bool add_back = false;
      if (blocks) {
        alive = pa_wait(b_o_full + 8 * t, o_phase, abort_flag, 0x2780u | t);
        o_phase ^= 1u;
        if (!alive) break;
        pa_fence_after();
        add_back = any_masked && not_finite[slot_flag] != 0;
      }
      if (warp_live) {
        const int64_t token = (int64_t)it.tok + tok;
        const int head = it.head * p.group + my_head;
        const int64_t grow = token * p.hq + head;
        const bool none = !(sum > 0.0f) && sum == sum;             // no key seen
        const float inv = it.multi ? DOWN<DT> : none ? 0.0f : __frcp_rn(sum);
        float* part = it.multi ? p.part_o + (grow * p.segments + it.seg) * p.d : nullptr;
        bool odd = false;
#pragma unroll 1
        for (int q = 0; q < HDP / QW; ++q) {
          if (32 * q >= p.d) break;
          uint32_t raw[QW];
          __syncwarp();
          if (blocks) load_quarter(t_o + 32u * q, raw);
          float o[QW];
#pragma unroll
          for (int i = 0; i < QW; ++i) o[i] = none || !blocks ? 0.0f : f_mul(__uint_as_float(raw[i]), inv);
          float z = 0.0f;
#pragma unroll
          for (int i = 0; i < QW; ++i) z = f_fma(o[i], 0.0f, z);
          odd |= !(z == 0.0f);                                     // O is not finite here
          const int n = live ? min(QW, p.d - 32 * q) : 0;
          if (n == 0) {
          } else if (it.multi) {
#pragma unroll
            for (int i = 0; i < QW; i += 4)
              if (i < n) *reinterpret_cast<float4*>(part + 32 * q + i) = make_float4(o[i], o[i + 1], o[i + 2], o[i + 3]);
          } else if (p.o_dtype == RG_F32) {
            float* dst = static_cast<float*>(p.out) + token * p.o_tok + head * p.o_head + 32 * q;
            if (p.o_vec) {
#pragma unroll
              for (int i = 0; i < QW; i += 4) if (i < n) *reinterpret_cast<float4*>(dst + i) = make_float4(o[i], o[i + 1], o[i + 2], o[i + 3]);
            } else {
#pragma unroll
              for (int i = 0; i < QW; ++i) if (i < n) dst[i] = o[i];
            }
          } else {
            uint16_t* dst = static_cast<uint16_t*>(p.out) + token * p.o_tok + head * p.o_head + 32 * q;
            uint32_t w[QW / 2];
#pragma unroll
            for (int i = 0; i < QW / 2; ++i) w[i] = pack_16x2(o[2 * i], o[2 * i + 1], DT);
            if (p.o_vec) {
#pragma unroll
              for (int i = 0; i < QW / 2; i += 4) if (2 * i < n) *reinterpret_cast<uint4*>(dst + 2 * i) = make_uint4(w[i], w[i + 1], w[i + 2], w[i + 3]);
            } else {
#pragma unroll
              for (int i = 0; i < QW / 2; ++i) if (2 * i < n) { dst[2 * i] = (uint16_t)(w[i] & 0xffffu); dst[2 * i + 1] = (uint16_t)(w[i] >> 16); }
            }
          }
        }
        const bool some = live && sum > 0.0f;                      // the row sees keys, and no NaN among its scores
        odd = __any_sync(0xffffffffu, odd && some);
        if (odd || add_back) {
#pragma unroll 1
          for (int q = 0; 32 * q < p.d; ++q)
            put_odd_values<DT>(p, it, odd, q, some ? lo : INT32_MAX, hi, some, it.multi ? (grow * p.segments + it.seg) * p.d : token * p.o_tok + head * p.o_head);
        }
        if (live) {
          if (it.multi) p.part_ml[grow * p.segments + it.seg] = make_float2(m, f_mul(sum, DOWN<DT>));
          else if (p.lse) p.lse[token * p.lse_ld + head] = none ? -INFINITY : f_add(f_mul(m, p.scale), logf(f_mul(sum, DOWN<DT>)));
        }
      }
      if (blocks) {
        pa_fence_before();
        __syncwarp();
        if (lane == 0) mbar_arrive(b_o_empty + 8 * t);
      }
    }
  }

  // ---------------------------------------------------------------- teardown
  __syncthreads();
  if (*abort_flag) {                                               // a wait gave up: let copies and products in flight end
    const uint64_t t0 = globaltimer_ns();
    while (globaltimer_ns() - t0 < 200000ull) __nanosleep(1000);
    __syncthreads();
  }
  if (warp == F::MMA) {
    pa_fence_after();
    asm volatile("tcgen05.dealloc.cta_group::1.sync.aligned.b32 %0, %1;" ::"r"(tmem), "r"(F::COLS) : "memory");
  }
}

// ---------------------------------------------------------------- the form for few rows
// Single tokens and drafts: up to ROWS rows of a key head.  The operands change places: a block's keys are the 128 rows of the first product and
// the head's elements the 128 rows of the second, the queries the narrow side (N = 16 or 32) of both, so that the tensor core reads every K and
// V element from shared memory once and little else:
//   S' = K_j Q^T       lane = key, column = row of queries
//   O' += V_j^T P^T    lane = element of the head, column = row of queries; V is read transposed, P from shared memory
// A softmax thread is one key of the block and holds its score with every row; maxima and sums over the keys go through butterflies
// in which lanes trade rows (after five steps a lane holds one row's value), and the four warps' maxima through shared memory.
// What bounds it: the K and V bytes.  64 sequences of up to 8192 keys, 8 key heads of 128 (1.14 GB): 196 us a call, 5.8 TB/s; 4 of up to 61000 (0.76 GB): 132 us,
// 5.8 TB/s; one of 8192 (34 MB): 13 us, of which the copies are 5 (launch, item and page look-up, the chain of two blocks and the join are latency).
// With the queries as the 128 rows instead (the other form, 4 of them filled) the 64 sequences took 234 us on the device, and 278 with each row's keys dealt to
// four warps: the tensor core then reads 128 mostly empty rows from shared memory for every step.
template <int HDP, int ROWS>
struct Few {
  static constexpr int DB = HDP / 64;
  static constexpr int PRODUCER = 4, MMA = 5, FIXER = 6, WARPS = 7, THREADS = WARPS * 32;
  static constexpr int N = ROWS < 16 ? 16 : ROWS;                  // narrow side of the products
  static constexpr uint32_t Q_BOX = N * 128, P_BOX = N * 128, P_BUF = 2 * P_BOX;      // rows of 64 elements, 64 keys
  static constexpr uint32_t KV_BOX = BLK * 128, SLOT = DB * KV_BOX;
  static constexpr int SLOTS = HDP == 128 ? 3 : 5;
  static constexpr uint32_t COLS = 128;                            // tensor memory: S' of even and odd blocks at 0 and 32, O' of even and odd items at 64 and 96
  static constexpr uint32_t Q_AT = SLOTS * SLOT, P_AT = Q_AT + DB * Q_BOX, ITEM_AT = P_AT + 2 * P_BUF, BAR_AT = ITEM_AT + ITEMS * sizeof(Item),
                            N_BAR = 12 + 3 * SLOTS + 2 * ITEMS, FLAG_AT = BAR_AT + 8 * N_BAR, MAX_AT = (FLAG_AT + 4 * (2 + FLAGS) + 15) & ~15u, SUM_AT = MAX_AT + 2 * 128 * 4,
                            LAST = SUM_AT + 2 * 128 * 4;
  static constexpr size_t SMEM = 1024 + LAST;
  static_assert(SMEM <= 115712 && SLOTS / 2 + 1 < FLAGS, "two CTAs fit the SM; the fixer cannot be a whole turn of flags ahead");
};

// Butterfly over the warp's lanes for ROWS values a lane, lanes trading halves of what they still hold: lane i ends with the whole value of
// row i >> (5 - log2 ROWS).  Every level combines lane i's value with lane i ^ x's, x = 16, 8, 4, 2, 1.
template <int ROWS, bool MAX>
__device__ __forceinline__ float reduce_rows(float (&v)[ROWS]) {
  const int lane = threadIdx.x & 31;
  int n = ROWS;
#pragma unroll
  for (int x = 16; x; x >>= 1) {
    if (n > 1) {
      n >>= 1;
      const bool upper = lane & x;
#pragma unroll
      for (int i = 0; i < ROWS / 2; ++i) {
        if (i >= n) break;
        const float keep = upper ? v[i + n] : v[i], send = upper ? v[i] : v[i + n];
        const float got = __shfl_xor_sync(0xffffffffu, send, x);
        v[i] = MAX ? max3(keep, got, got) : f_add(keep, got);
      }
    } else {
      const float got = __shfl_xor_sync(0xffffffffu, v[0], x);
      v[0] = MAX ? max3(v[0], got, got) : f_add(v[0], got);
    }
  }
  return v[0];
}

template <int HDP, int ROWS, int DT>
__global__ void __launch_bounds__(Few<HDP, ROWS>::THREADS, 2)
paged_attention_few_kernel(const __grid_constant__ CUtensorMap tmap_q, const __grid_constant__ CUtensorMap tmap_k, const __grid_constant__ CUtensorMap tmap_v,
                           const __grid_constant__ Params p) {
  using F = Few<HDP, ROWS>;
  constexpr int DB = F::DB, SLOTS = F::SLOTS;
  constexpr uint32_t IDESC_S = pa_idesc(F::N, DT == RG_BF16, false, false), IDESC_O = pa_idesc(F::N, DT == RG_BF16, true, false);

  extern __shared__ uint8_t smem_raw[];
  const uint32_t smem_base = (smem_u32(smem_raw) + 1023u) & ~1023u;
  uint8_t* smem_gen = smem_raw + (smem_base - smem_u32(smem_raw));
  const uint32_t sKV = smem_base, sQ = smem_base + F::Q_AT, sP = smem_base + F::P_AT;
  Item* items = reinterpret_cast<Item*>(smem_gen + F::ITEM_AT);
  const uint32_t bar0 = smem_base + F::BAR_AT;
  const uint32_t b_q_full = bar0, b_q_empty = bar0 + 8, b_x = bar0 + 16, b_y = bar0 + 24, b_s = bar0 + 32, b_p = bar0 + 48, b_pv = bar0 + 64, b_o_empty = bar0 + 80, b_full = bar0 + 96;   // two each from b_s to b_o_empty
  const uint32_t b_ready = b_full + 8 * SLOTS, b_empty = b_ready + 8 * SLOTS, b_item = b_empty + 8 * SLOTS, b_free = b_item + 8 * ITEMS;
  uint32_t* tmem_slot = reinterpret_cast<uint32_t*>(smem_gen + F::FLAG_AT);
  volatile int* abort_flag = reinterpret_cast<volatile int*>(tmem_slot + 1);
  volatile int* not_finite = reinterpret_cast<volatile int*>(tmem_slot + 2);          // [FLAGS]
  float* xm = reinterpret_cast<float*>(smem_gen + F::MAX_AT);                          // [2][4][32]: the warps' maxima of a block, by its parity
  float* xl = reinterpret_cast<float*>(smem_gen + F::SUM_AT);                          // [2][4][32]: their sums, by the item's parity

  const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
  if (threadIdx.x == 0) {
    mbar_init(b_q_full, 1); mbar_init(b_q_empty, 1); mbar_init(b_x, 4); mbar_init(b_y, 4);
    for (int t = 0; t < 2; ++t) { mbar_init(b_s + 8 * t, 1); mbar_init(b_p + 8 * t, 4); mbar_init(b_pv + 8 * t, 1); mbar_init(b_o_empty + 8 * t, 4); }
    for (int s = 0; s < SLOTS; ++s) { mbar_init(b_full + 8 * s, 1); mbar_init(b_ready + 8 * s, 1); mbar_init(b_empty + 8 * s, 1); }
    for (int s = 0; s < ITEMS; ++s) { mbar_init(b_item + 8 * s, 1); mbar_init(b_free + 8 * s, F::WARPS - 1); }
    *abort_flag = 0;
    asm volatile("fence.mbarrier_init.release.cluster;" ::: "memory");
  }
  if (warp == F::MMA) {
    asm volatile("tcgen05.alloc.cta_group::1.sync.aligned.shared::cta.b32 [%0], %1;" ::"r"(smem_u32(tmem_slot)), "r"(F::COLS) : "memory");
    asm volatile("tcgen05.relinquish_alloc_permit.cta_group::1.sync.aligned;" ::: "memory");
  }
  pa_fence_before();
  __syncthreads();
  pa_fence_after();
  const uint32_t tmem = *tmem_slot;
  asm volatile("griddepcontrol.wait;" ::: "memory");               // the set-up ran under the tail of the kernel in front; from here on its results are read
  if (p.segments > 1) asm volatile("griddepcontrol.launch_dependents;" ::: "memory");

  Ring<ITEMS> ir;
  auto next_item = [&](Item& it, bool& alive) -> bool {
    if (!pa_wait(b_item + 8 * ir.slot, ir.phase, abort_flag, 0x3000u)) { alive = false; return false; }
    it = items[ir.slot];
    __syncwarp();
    if (lane == 0) mbar_arrive(b_free + 8 * ir.slot);
    ir.step();
    return it.n_tok > 0;
  };
  Item it;
  bool alive = true;

  if (warp == F::PRODUCER) {
    // ------------------------------------------------------------ producer: K_0, K_1, V_0, K_2, V_1, ..., as they are used
    const int pieces = BLK / p.box;
    const int piece = lane & (pieces - 1), col = lane / pieces;
    Ring<SLOTS> kv;
    uint32_t q_phase = 1;
    Walk walk;
    walk.start(p, p.tile_tokens);
    while (alive) {
      const bool more = walk.get(p, p.tile_tokens, it);
      if (!more) it.n_tok = 0;
      alive = pa_wait(b_free + 8 * ir.slot, ir.phase ^ 1u, abort_flag, 0x3080u);
      if (!alive) break;
      if (lane == 0) { items[ir.slot] = it; mbar_arrive(b_item + 8 * ir.slot); }
      ir.step();
      if (!more) break;
      if (it.b1 == it.b0) continue;
      const int32_t* row = p.table + (int64_t)it.seq * p.table_ld;
      auto wanted = [&](int b) -> bool { const int32_t k = b * BLK + piece * p.box; return col < DB && b < it.b1 && k <= it.hi && k + p.box > it.lo; };
      auto entry = [&](int b) -> int32_t { return row[(b * BLK + piece * p.box) / p.by_page]; };
      int32_t page = wanted(it.b0) ? entry(it.b0) : 0, next = wanted(it.b0 + 1) ? entry(it.b0 + 1) : 0;      // looked up a block ahead of their use
      alive = pa_wait(b_q_empty, q_phase, abort_flag, 0x3100u);
      if (!alive) break;
      q_phase ^= 1u;
      if (lane == 0) mbar_expect_tx(b_q_full, (uint32_t)(DB * p.tile_tokens * p.group) * 128u);
      __syncwarp();
      if (lane < DB) pa_tma_4d(sQ + lane * F::Q_BOX, &tmap_q, lane * 64, 0, it.tok, it.head, b_q_full);
      auto copy = [&](const CUtensorMap* map, int b, int32_t& id) {
        const bool mine = wanted(b);
        if (mine && (id < 0 || id >= p.pages)) {                   // not a page: the copy from behind the last one fills in zeros
          if (col == 0) atomicCAS(&g_paged_attn_page_word, 0u, (unsigned)RG_PAGE_CODE_ATTEND);
          id = p.pages;
        }
        const int32_t key = b * BLK + piece * p.box, at = key - key / p.by_page * p.page_size;
        const uint32_t bytes = (uint32_t)__popc(__ballot_sync(0xffffffffu, mine)) * (uint32_t)p.box * 128u;
        alive = pa_wait(b_empty + 8 * kv.slot, kv.phase ^ 1u, abort_flag, 0x3200u | kv.slot);
        if (!alive) return;
        if (lane == 0) mbar_expect_tx(b_full + 8 * kv.slot, bytes);
        __syncwarp();
        if (mine) pa_tma_4d(sKV + kv.slot * F::SLOT + col * F::KV_BOX + piece * p.box * 128, map, col * 64, at, it.head, id, b_full + 8 * kv.slot);
        kv.step();
      };
      copy(&tmap_k, it.b0, page);
      for (int b = it.b0; b < it.b1 && alive; ++b) {
        const int32_t later = wanted(b + 2) ? entry(b + 2) : 0;
        if (b + 1 < it.b1) copy(&tmap_k, b + 1, next);
        if (alive) copy(&tmap_v, b, page);
        page = next;
        next = later;
      }
    }
  } else if (warp == F::MMA) {
    // ------------------------------------------------------------ MMA issuer
    const bool leader = elect_one();
    Ring<SLOTS> kv;
    uint32_t q_phase = 0, block = 0, n_item = 0;
    auto next_slot = [&](uint32_t& bar) -> uint32_t {
      const uint32_t slot = __shfl_sync(0xffffffffu, kv.slot, 0);
      alive = pa_wait(b_ready + 8 * slot, kv.phase, abort_flag, 0x3300u | slot);
      if (alive) alive = pa_wait(b_full + 8 * slot, kv.phase, abort_flag, 0x3380u | slot);
      pa_fence_after();
      bar = b_empty + 8 * slot;
      kv.step();
      return __shfl_sync(0xffffffffu, sKV + slot * F::SLOT, 0);
    };
    // The scores of block number c go to columns 32 (c & 1): those of c - 2 have been read, since the product of c - 2 was issued.
    auto scores = [&](uint32_t c, uint32_t sK, uint32_t k_bar) {
#pragma unroll
      for (int b = 0; b < DB; ++b) {
        const uint64_t k = pa_desc(sK + b * F::KV_BOX, 16), q = pa_desc(sQ + b * F::Q_BOX, 16);
#pragma unroll
        for (int e = 0; e < 4; ++e) if (leader) pa_mma_ss(tmem + 32u * (c & 1), k + 2u * e, q + 2u * e, IDESC_S, (b | e) ? 1u : 0u);
      }
      if (leader) { pa_commit(b_s + 8 * (c & 1)); pa_commit(k_bar); }
    };
    while (alive && next_item(it, alive)) {
      const int nb = __shfl_sync(0xffffffffu, it.b1 - it.b0, 0);
      if (nb == 0) continue;
      alive = pa_wait(b_q_full, q_phase, abort_flag, 0x3400u);
      q_phase ^= 1u;
      if (!alive) break;
      uint32_t bar, sK = next_slot(bar);
      if (!alive) break;
      scores(block, sK, bar);
      if (nb == 1 && leader) pa_commit(b_q_empty);
      const uint32_t t_o = tmem + 64u + 32u * (n_item & 1);
      for (int j = 0; j < nb; ++j, ++block) {
        if (j + 1 < nb) {
          sK = next_slot(bar);
          if (!alive) break;
          scores(block + 1, sK, bar);
          if (j + 2 == nb && leader) pa_commit(b_q_empty);
        }
        const uint32_t sV = next_slot(bar);
        if (alive) alive = pa_wait(b_p + 8 * (block & 1), (block >> 1) & 1, abort_flag, 0x3500u);
        if (alive && j == 0) alive = pa_wait(b_o_empty + 8 * (n_item & 1), ((n_item >> 1) & 1) ^ 1u, abort_flag, 0x3580u);
        if (!alive) break;
        pa_fence_after();
        // heads of up to 64 elements: the upper 64 lanes repeat the lower ones (distance 0 between the column groups), nobody reads them
        const uint64_t v = pa_desc(sV, HDP == 128 ? F::KV_BOX : 0), pr = pa_desc(sP + (block & 1) * F::P_BUF, 16);
#pragma unroll
        for (int e = 0; e < BLK / 16; ++e)
          if (leader) pa_mma_ss(t_o, v + (uint64_t)(e * (2048 >> 4)), pr + (uint64_t)((e >> 2) * (F::P_BOX >> 4) + 2 * (e & 3)), IDESC_O, (j | e) ? 1u : 0u);
        if (leader) { pa_commit(b_pv + 8 * (block & 1)); pa_commit(bar); }
      }
      ++n_item;
    }
  } else if (warp == F::FIXER) {
    // ------------------------------------------------------------ fixer
    Ring<SLOTS> kv;
    uint32_t flags = 0;
    while (alive && next_item(it, alive)) {
      bool any_masked = false;
      const int nb = it.b1 - it.b0;
      for (int i = 0; i < 2 * nb && alive; ++i) {                  // K_0, K_1, V_0, K_2, V_1, ..., V of the last two
        const bool is_v = i == 2 * nb - 1 || (i >= 2 && !(i & 1));
        const int b = it.b0 + (i == 2 * nb - 1 ? nb - 1 : (i >> 1) - 1);
        alive = pa_wait(b_full + 8 * kv.slot, kv.phase, abort_flag, 0x3600u | kv.slot);
        if (!alive) break;
        if (is_v && masked_block(p, it, b)) {
          const bool seen = fix_values<DT>(reinterpret_cast<uint4*>(smem_gen + kv.slot * F::SLOT), F::SLOT / 16, b * BLK, it.lo, it.hi);
          if (lane == 0) not_finite[flags % FLAGS] = any_masked ? (not_finite[flags % FLAGS] | (seen ? 1 : 0)) : (seen ? 1 : 0);
          any_masked = true;
        }
        __syncwarp();
        if (lane == 0) mbar_arrive(b_ready + 8 * kv.slot);
        kv.step();
      }
      if (any_masked) ++flags;
    }
  } else {
    // ------------------------------------------------------------ softmax and output rows
    constexpr int SH = ROWS == 8 ? 2 : ROWS == 16 ? 1 : 0;         // lane i looks after row i >> SH
    const int r = lane >> SH;
    const int my_tok = r / p.by_group;
    const uint32_t t_lane = tmem + (static_cast<uint32_t>(warp * 32) << 16);
    uint32_t block = 0, n_item = 0, flags = 0;
    uint8_t* p_row = smem_gen + F::P_AT + (warp >> 1) * F::P_BOX + (lane & 7) * 2;     // this key's place in the rows of P: 16-byte pieces of 8 keys, swizzled
    const int p_piece = (warp & 1) * 4 + (lane >> 3);
    while (alive && next_item(it, alive)) {
      const bool live = my_tok < it.n_tok && my_tok < p.tile_tokens;
      const int32_t place = it.pos + my_tok;
      const int32_t hi = live ? min(last_seen(p, place, it.len), it.hi) : -1, lo = max(first_seen(p, place), it.lo);
      const bool blocks = it.b1 > it.b0;
      const uint32_t t_o = t_lane + 64u + 32u * (n_item & 1);
      float m = -INFINITY, l = 0.0f;                               // of row r; l over this warp's keys
      bool any_masked = blocks && (masked_block(p, it, it.b0) || masked_block(p, it, it.b1 - 1));       // what is masked lies at the ends
      for (int b = it.b0; b < it.b1; ++b, ++block) {
        const uint32_t buf = block & 1, phase = (block >> 1) & 1;
        alive = pa_wait(b_s + 8 * buf, phase, abort_flag, 0x3700u);
        if (!alive) break;
        pa_fence_after();
        uint32_t s[ROWS];
        pa_ld_cols<ROWS>(t_lane + 32u * buf, s);
        const bool masked = masked_block(p, it, b);
        const int32_t key = b * BLK + warp * 32 + lane;
        if (masked) {
#pragma unroll
          for (int i = 0; i < ROWS; ++i) {
            const int32_t from = __shfl_sync(0xffffffffu, lo, i << SH), to = __shfl_sync(0xffffffffu, hi, i << SH);
            s[i] = key >= from && key <= to ? s[i] : 0xff800000u;
          }
        }
        float v[ROWS];
#pragma unroll
        for (int i = 0; i < ROWS; ++i) v[i] = __uint_as_float(s[i]);
        float* x = xm + buf * 128;                                 // a warp is at most one block ahead of another
        x[warp * 32 + lane] = reduce_rows<ROWS, true>(v);
        __syncwarp();
        if (lane == 0) mbar_arrive(b_x);
        alive = pa_wait(b_x, block & 1, abort_flag, 0x3640u);
        if (!alive) break;
        const float mb = max3(max3(x[lane], x[32 + lane], x[64 + lane]), x[96 + lane], x[96 + lane]);
        const float alpha = rises(m, mb, p.c) ? move_max(m, mb, p.c) : 1.0f;
        float shift, off;
        if (__any_sync(0xffffffffu, shift_of<DT>(m, p.c, shift, off))) {
#pragma unroll
          for (int i = 0; i < ROWS; ++i) s[i] = __float_as_uint(f_add(__uint_as_float(s[i]), -__shfl_sync(0xffffffffu, off, i << SH)));
        }
        uint8_t* row = p_row + buf * F::P_BUF;
#pragma unroll
        for (int i = 0; i < ROWS; i += 2) {
          const float s0 = __shfl_sync(0xffffffffu, shift, i << SH), s1 = __shfl_sync(0xffffffffu, shift, (i + 1) << SH);
          const float2 sc = make_float2(__uint_as_float(s[i]), __uint_as_float(s[i + 1]));
          const float2 eh = prob2<false>(sc, p.c, s0, s1), ep = prob2<true>(sc, p.c, s0, s1);
          const float2 e = lane >= POLY_FROM ? ep : eh;
          v[i] = e.x; v[i + 1] = e.y;
          const uint32_t w = pack_16x2(e.x, e.y, DT);
          *reinterpret_cast<uint16_t*>(row + i * 128 + ((p_piece ^ (i & 7)) << 4)) = (uint16_t)(w & 0xffffu);
          *reinterpret_cast<uint16_t*>(row + (i + 1) * 128 + ((p_piece ^ ((i + 1) & 7)) << 4)) = (uint16_t)(w >> 16);
        }
        asm volatile("fence.proxy.async.shared::cta;" ::: "memory");
        if (b > it.b0 && __any_sync(0xffffffffu, live && alpha != 1.0f)) {
          // O' takes the factor once the product of the block before is complete; the one of this block waits for this warp
          alive = pa_wait(b_pv + 8 * (buf ^ 1), ((block - 1) >> 1) & 1, abort_flag, 0x3680u);
          if (!alive) break;
          pa_fence_after();
          uint32_t o[ROWS];
          pa_ld_cols<ROWS>(t_o, o);
#pragma unroll
          for (int i = 0; i < ROWS; ++i) o[i] = __float_as_uint(f_mul(__uint_as_float(o[i]), __shfl_sync(0xffffffffu, alpha, i << SH)));
          pa_st_cols<ROWS>(t_o, o);
          pa_wait_st();
        }
        pa_fence_before();
        __syncwarp();
        if (lane == 0) mbar_arrive(b_p + 8 * buf);
        l = add_quarter(l, alpha, reduce_rows<ROWS, false>(v), m, mb);
      }
      if (!alive) break;
      const int slot_flag = flags % FLAGS;
      if (any_masked) ++flags;
      float sum = 0.0f;
      bool add_back = false;
      if (blocks) {
        float* x = xl + (n_item & 1) * 128;
        x[warp * 32 + lane] = l;
        __syncwarp();
        if (lane == 0) mbar_arrive(b_y);
        alive = pa_wait(b_y, n_item & 1, abort_flag, 0x3740u);
        if (!alive) break;
        sum = join_quarters(x[lane], x[32 + lane], x[64 + lane], x[96 + lane]);
        alive = pa_wait(b_pv + 8 * ((block - 1) & 1), ((block - 1) >> 1) & 1, abort_flag, 0x3780u);      // the last block's product
        if (!alive) break;
        pa_fence_after();
        add_back = any_masked && not_finite[slot_flag] != 0;
      }
      const bool none = !(sum > 0.0f) && sum == sum;               // no key seen
      const float inv = it.multi ? DOWN<DT> : none ? 0.0f : __frcp_rn(sum);
      const int col = warp * 32 + lane;                            // element of the head
      const int n_rows = it.n_tok * p.group;
      if (warp * 32 < p.d) {
        uint32_t raw[ROWS];
        if (blocks) pa_ld_cols<ROWS>(t_o, raw);
        float o[ROWS];
#pragma unroll
        for (int i = 0; i < ROWS; ++i) {
          const bool zero = __shfl_sync(0xffffffffu, (int)none, i << SH) || !blocks;
          const float f = __shfl_sync(0xffffffffu, inv, i << SH);
          o[i] = zero ? 0.0f : f_mul(__uint_as_float(raw[i]), f);
        }
        const bool some = live && sum > 0.0f;                      // lane's row sees keys, and no NaN among its scores
        const uint32_t some_rows = __ballot_sync(0xffffffffu, some);
        bool odd = false;                                          // whether O is not finite in one of them
#pragma unroll
        for (int i = 0; i < ROWS; ++i) odd |= (some_rows >> (i << SH) & 1u) && !(f_add(o[i], -o[i]) == 0.0f);
        if (col < p.d) {
          int tok = 0, head = 0;
#pragma unroll
          for (int i = 0; i < ROWS; ++i) {
            if (i < n_rows) {
              const int64_t token = (int64_t)it.tok + tok;
              const int h = it.head * p.group + head;
              if (it.multi) p.part_o[((token * p.hq + h) * p.segments + it.seg) * p.d + col] = o[i];
              else store_scalar(p.out, p.o_dtype, token * p.o_tok + h * p.o_head + col, o[i]);
              if (++head == p.group) { head = 0; ++tok; }
            }
          }
        }
        odd = __any_sync(0xffffffffu, odd);
        if (odd || add_back) {
          const int64_t token = (int64_t)it.tok + my_tok;
          const int h = it.head * p.group + r - my_tok * p.group;
          put_odd_values<DT>(p, it, odd, warp, some ? lo : INT32_MAX, hi, some && (lane & ((1 << SH) - 1)) == 0,
                             it.multi ? ((token * p.hq + h) * p.segments + it.seg) * p.d : token * p.o_tok + h * p.o_head);
        }
      }
      if (warp == 0 && live && (lane & ((1 << SH) - 1)) == 0) {
        const int64_t token = (int64_t)it.tok + my_tok;
        const int h = it.head * p.group + r - my_tok * p.group;
        if (it.multi) p.part_ml[(token * p.hq + h) * p.segments + it.seg] = make_float2(m, f_mul(sum, DOWN<DT>));
        else if (p.lse) p.lse[token * p.lse_ld + h] = none ? -INFINITY : f_add(f_mul(m, p.scale), logf(f_mul(sum, DOWN<DT>)));
      }
      if (blocks) {
        pa_fence_before();
        __syncwarp();
        if (lane == 0) mbar_arrive(b_o_empty + 8 * (n_item & 1));
        ++n_item;
      }
    }
  }

  // ---------------------------------------------------------------- teardown
  __syncthreads();
  if (*abort_flag) {                                               // a wait gave up: let copies and products in flight end
    const uint64_t t0 = globaltimer_ns();
    while (globaltimer_ns() - t0 < 200000ull) __nanosleep(1000);
    __syncthreads();
  }
  if (warp == F::MMA) {
    pa_fence_after();
    asm volatile("tcgen05.dealloc.cta_group::1.sync.aligned.b32 %0, %1;" ::"r"(tmem), "r"(F::COLS) : "memory");
  }
}

// Joins the parts of a row: parts of one sixteen (by their number) in ascending order, then the sixteens in ascending order.  A warp sums a
// sixteen, four columns a lane and sixteen loads in flight; WARPS of them take the sixteens of one row in turn.  With WARPS = 1 (no sequence can have
// more than 16 parts) every warp of a CTA has a row of its own: 2048 rows of up to 16 parts; a single long row would leave most of them without work.
constexpr int JOIN_THREADS = 256;
template <int WARPS>
__global__ void __launch_bounds__(JOIN_THREADS) join_parts_kernel(const __grid_constant__ Params p) {
  __shared__ float4 s_o[WARPS > 1 ? WARPS : 1][32];
  __shared__ float s_l[WARPS > 1 ? WARPS : 1], s_m[WARPS > 1 ? WARPS : 1];
  const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
  asm volatile("griddepcontrol.wait;" ::: "memory");               // the parts are the kernel's in front
  const int32_t grow = WARPS > 1 ? (int32_t)blockIdx.x : (int32_t)blockIdx.x * (JOIN_THREADS / 32) + warp;
  if (grow >= (int32_t)(p.tokens * p.hq)) return;
  const int32_t token = grow / p.by_hq;
  const int head = grow - token * p.hq;
  // the row's sequence: the first that ends behind it.  Its lengths come with the search.
  SeqView v = {0, 0, 0, 0};
  bool found = false;
  for (int base = 0; base < p.n_seqs && !found; base += 32) {
    bool bad;
    if (base + lane < p.n_seqs) v = view_of(p, base + lane, &bad);
    else v = SeqView{INT32_MAX, 0, 0, 0};
    const uint32_t hit = __ballot_sync(0xffffffffu, v.tok <= token && token < v.tok + v.n);
    found = hit != 0;
    const int owner = found ? __ffs(hit) - 1 : 0;
    v.tok = __shfl_sync(0xffffffffu, v.tok, owner); v.len = __shfl_sync(0xffffffffu, v.len, owner);
    v.first = __shfl_sync(0xffffffffu, v.first, owner); v.n = __shfl_sync(0xffffffffu, v.n, owner);
  }
  if (!found) return;
  int32_t g0, n;
  parts_of(p, v, &g0, &n);
  if (n <= 1) return;                                              // written by the main kernel
  const int32_t place = v.first + (token - v.tok), hi = last_seen(p, place, v.len), lo = first_seen(p, max(place, 0));
  const int ga = hi >= lo ? lo / p.by_split : 0, gb = hi >= lo ? hi / p.by_split + 1 : 0;
  const float2* ml = p.part_ml + (int64_t)grow * p.segments;
  const bool mine = 4 * lane < p.d;
  const float* po = p.part_o + (int64_t)grow * p.segments * p.d + 4 * lane;
  // a sixteen's products, maxima and sums; the first one of each warp is on its way before the row's maximum is known
  float4 x[16];
  float2 xml;
  auto fetch = [&](int base) {
    const int first = 16 * (base + (WARPS > 1 ? warp : 0)), g = first + (lane & 15);
    xml = g >= ga && g < gb ? ml[g] : make_float2(-INFINITY, 0.0f);
#pragma unroll
    for (int i = 0; i < 16; ++i)
      x[i] = mine && first + i >= ga && first + i < gb ? *reinterpret_cast<const float4*>(po + (int64_t)(first + i) * p.d) : make_float4(0.0f, 0.0f, 0.0f, 0.0f);
  };
  fetch(ga / 16);
  float m = xml.x;
  for (int g = ga / 16 * 16 + 16 * WARPS + (WARPS > 1 ? (int)threadIdx.x : lane); g < gb; g += WARPS > 1 ? JOIN_THREADS : 32) m = fmaxf(m, ml[g].x);
#pragma unroll
  for (int k = 16; k; k >>= 1) m = fmaxf(m, __shfl_xor_sync(0xffffffffu, m, k));
  if (WARPS > 1) {
    if (lane == 0) s_m[warp] = m;
    __syncthreads();
#pragma unroll
    for (int w = 0; w < WARPS; ++w) m = fmaxf(m, s_m[w]);
  }
  float l = 0.0f;
  float4 o = make_float4(0.0f, 0.0f, 0.0f, 0.0f);
  for (int base = ga / 16; base * 16 < gb; base += WARPS) {        // sixteens base .. base + WARPS - 1
    if (base != ga / 16) fetch(base);
    const float w = xml.x == -INFINITY ? 0.0f : pa_ex2(f_mul(f_add(xml.x, -m), p.c)), wl = f_mul(w, xml.y);
    float4 a = make_float4(0.0f, 0.0f, 0.0f, 0.0f);
    float al = 0.0f;
#pragma unroll
    for (int i = 0; i < 16; ++i) {
      const float wi = __shfl_sync(0xffffffffu, w, i);
      al = f_add(al, __shfl_sync(0xffffffffu, wl, i));
      a.x = f_fma(wi, x[i].x, a.x); a.y = f_fma(wi, x[i].y, a.y); a.z = f_fma(wi, x[i].z, a.z); a.w = f_fma(wi, x[i].w, a.w);
    }
    if (WARPS > 1) {
      s_o[warp][lane] = a;
      if (lane == 0) s_l[warp] = al;
      __syncthreads();
      if (warp == 0) {
#pragma unroll
        for (int k = 0; k < WARPS; ++k) {                          // a sixteen without parts is zeros
          const float4 y = s_o[k][lane];
          o.x = f_add(o.x, y.x); o.y = f_add(o.y, y.y); o.z = f_add(o.z, y.z); o.w = f_add(o.w, y.w);
          l = f_add(l, s_l[k]);
        }
      }
      __syncthreads();
    } else {
      o.x = f_add(o.x, a.x); o.y = f_add(o.y, a.y); o.z = f_add(o.z, a.z); o.w = f_add(o.w, a.w);
      l = f_add(l, al);
    }
  }
  if (WARPS > 1 && warp) return;
  const bool none = !(l > 0.0f) && l == l;
  const float inv = none ? 0.0f : __frcp_rn(l);
  if (mine) {
    const float r[4] = {none ? 0.0f : f_mul(o.x, inv), none ? 0.0f : f_mul(o.y, inv), none ? 0.0f : f_mul(o.z, inv), none ? 0.0f : f_mul(o.w, inv)};
    const int64_t at = (int64_t)token * p.o_tok + head * p.o_head + 4 * lane;
    if (p.o_vec && p.o_dtype == RG_F32) *reinterpret_cast<float4*>(static_cast<float*>(p.out) + at) = make_float4(r[0], r[1], r[2], r[3]);
    else if (p.o_vec) *reinterpret_cast<uint2*>(static_cast<uint16_t*>(p.out) + at) = make_uint2(pack_16x2(r[0], r[1], p.o_dtype), pack_16x2(r[2], r[3], p.o_dtype));
    else {
#pragma unroll
      for (int i = 0; i < 4; ++i) store_scalar(p.out, p.o_dtype, at + i, r[i]);
    }
  }
  if (p.lse && lane == 0) p.lse[(int64_t)token * p.lse_ld + head] = none ? -INFINITY : f_add(f_mul(m, p.scale), logf(l));
}
template <int WARPS>
cudaError_t launch_join(const Params& p, cudaStream_t st) {
  const int64_t rows = p.tokens * p.hq;
  cudaLaunchConfig_t cfg = {};
  cfg.gridDim = dim3((unsigned)(WARPS > 1 ? rows : (rows + JOIN_THREADS / 32 - 1) / (JOIN_THREADS / 32)), 1, 1);
  cfg.blockDim = dim3(JOIN_THREADS, 1, 1);
  cfg.stream = st;
  cudaLaunchAttribute attr[1];
  attr[0].id = cudaLaunchAttributeProgrammaticStreamSerialization;     // its launch runs under the main kernel, which it waits for
  attr[0].val.programmaticStreamSerializationAllowed = 1;
  cfg.attrs = attr;
  cfg.numAttrs = 1;
  return cudaLaunchKernelEx(&cfg, join_parts_kernel<WARPS>, p);
}

// ---------------------------------------------------------------- host
template <typename F, typename Kernel>
cudaError_t launch_form(Kernel kernel, DeviceOnce& configured, int ctas_per_sm, const CUtensorMap& q, const CUtensorMap& k, const CUtensorMap& v, const Params& p, int64_t most,
                        cudaStream_t st) {
  const DeviceInfo dev = current_device();
  if (!configured.has(dev.dev)) {
    cudaError_t e = cudaFuncSetAttribute(kernel, cudaFuncAttributeMaxDynamicSharedMemorySize, (int)F::SMEM);
    if (e != cudaSuccess) return e;
    configured.set(dev.dev);
  }
  cudaLaunchConfig_t cfg = {};
  cfg.gridDim = dim3((unsigned)std::min<int64_t>(most, (int64_t)dev.sms * ctas_per_sm), 1, 1);
  cfg.blockDim = dim3(F::THREADS, 1, 1);
  cfg.dynamicSmemBytes = F::SMEM;
  cfg.stream = st;
  cudaLaunchAttribute attr[1];
  attr[0].id = cudaLaunchAttributeProgrammaticStreamSerialization;
  attr[0].val.programmaticStreamSerializationAllowed = 1;
  cfg.attrs = attr;
  cfg.numAttrs = 1;
  return cudaLaunchKernelEx(&cfg, kernel, q, k, v, p);
}
template <int HDP, int DT>
cudaError_t launch_wide(const CUtensorMap& q, const CUtensorMap& k, const CUtensorMap& v, const Params& p, int64_t most, cudaStream_t st) {
  static DeviceOnce configured;
  return launch_form<Wide<HDP>>(paged_attention_wide_kernel<HDP, DT>, configured, 1, q, k, v, p, most, st);
}
template <int HDP, int ROWS, int DT>
cudaError_t launch_few(const CUtensorMap& q, const CUtensorMap& k, const CUtensorMap& v, const Params& p, int64_t most, cudaStream_t st) {
  static DeviceOnce configured;
  return launch_form<Few<HDP, ROWS>>(paged_attention_few_kernel<HDP, ROWS, DT>, configured, 2, q, k, v, p, most, st);
}
template <int DT>
cudaError_t launch_any(int rows, const CUtensorMap& q, const CUtensorMap& k, const CUtensorMap& v, const Params& p, int64_t most, cudaStream_t st) {
  if (p.d <= 64) {
    switch (rows) {
      case 8: return launch_few<64, 8, DT>(q, k, v, p, most, st);
      case 16: return launch_few<64, 16, DT>(q, k, v, p, most, st);
      case 32: return launch_few<64, 32, DT>(q, k, v, p, most, st);
    }
    return launch_wide<64, DT>(q, k, v, p, most, st);
  }
  switch (rows) {
    case 8: return launch_few<128, 8, DT>(q, k, v, p, most, st);
    case 16: return launch_few<128, 16, DT>(q, k, v, p, most, st);
  }
  return launch_wide<128, DT>(q, k, v, p, most, st);
}

}  // namespace

// All arguments were validated by the caller.
rg_status_t launch_paged_attention(const PagedAttnArgs& a, cudaStream_t st) {
  Params p{};
  const int64_t T = a.q->tokens, hkv = a.k->heads;
  const int G = (int)(a.q->heads / hkv), d = (int)a.q->dim, page = (int)a.k->page_size;
  p.table = a.seqs->block_table; p.seq_lens = a.seqs->seq_lens; p.cu_q = a.seqs->cu_q;
  p.table_ld = a.seqs->table_ld; p.max_len = a.max_len; p.tokens = T;
  p.n_seqs = a.seqs->n_seqs; p.page_size = page; p.pages = (int32_t)a.k->pages;
  p.hq = (int32_t)a.q->heads; p.hkv = (int32_t)hkv; p.group = G; p.d = d;
  p.split = (int32_t)a.split; p.segments = a.segments; p.causal = a.causal; p.window = (int32_t)a.window;
  p.scale = a.scale; p.c = a.scale * 1.44269504f;
  p.out = a.out->ptr; p.o_tok = a.out->token_stride; p.o_head = a.out->head_stride; p.o_dtype = a.out->dtype;
  const int per16 = a.out->dtype == RG_F32 ? 4 : 8;
  p.o_vec = (reinterpret_cast<uintptr_t>(a.out->ptr) & 15) == 0 && p.o_tok % per16 == 0 && p.o_head % per16 == 0;
  p.lse = a.lse; p.lse_ld = a.lse_ld;
  p.part_o = static_cast<float*>(a.ws);
  if (a.ws) p.part_ml = reinterpret_cast<float2*>(p.part_o + T * p.hq * (int64_t)a.segments * d);
  p.v = static_cast<const uint16_t*>(a.v->ptr); p.v_page = a.v->page_stride; p.v_slot = a.v->slot_stride; p.v_head = a.v->head_stride;

  const int64_t need = a.max_q * G;
  const int most_rows = d <= 64 ? 32 : 16;
  const int rows = need <= 8 ? 8 : need <= 16 ? 16 : need <= most_rows ? most_rows : 128;
  const bool narrow = rows < 128;
  p.tile_tokens = rows / G;
  int box = page & -page;                                  // the largest power of two that divides the page size: boxes never cross pages
  p.box = box = box < BLK ? box : BLK;

  CUtensorMap tq, tk, tv;
  const int64_t pages = p.pages > 0 ? p.pages : 1;
  const void* kp = p.pages > 0 ? a.k->ptr : a.q->ptr;      // no pages: nothing is read, but a map wants an address
  const void* vp = p.pages > 0 ? a.v->ptr : a.q->ptr;
  if (!make_tmap_4d(&tq, a.q->ptr, a.q->dtype, {d, G, T, hkv}, {a.q->head_stride, a.q->token_stride, G * a.q->head_stride}, {64, G, p.tile_tokens, 1}) ||
      !make_tmap_4d(&tk, kp, a.q->dtype, {d, page, hkv, pages}, {a.k->slot_stride, a.k->head_stride, a.k->page_stride}, {64, box, 1, 1}) ||
      !make_tmap_4d(&tv, vp, a.q->dtype, {d, page, hkv, pages}, {a.v->slot_stride, a.v->head_stride, a.v->page_stride}, {64, box, 1, 1}))
    return RG_ERR_CUDA;

  p.by_split = Div::by(p.split ? p.split : 1); p.by_hkv = Div::by(p.hkv); p.by_hq = Div::by(p.hq); p.by_page = Div::by(page); p.by_group = Div::by(G);
  // Two tiles share the keys that a CTA reads and the tensor core works for one while the other's softmax runs; but where all tiles find an SM
  // each, one tile alone is done sooner (about 2600 cycles a block against 3500).  4 query heads a key head, so 32 tokens a tile, on 1500 keys: 16 tiles 31.9 us
  // alone and 36.1 in twos, 64 tiles 33.3 and 37.3, 128 tiles 32.8 and 36.2; 152 tiles 60.6 and 43.5, 256 tiles 73.9 and 49.0.
  auto items_of = [&](int64_t tokens) { return std::min<int64_t>(T, (T + tokens - 1) / tokens + p.n_seqs) * hkv * a.segments; };
  p.cta_tokens = narrow || items_of(p.tile_tokens) <= current_device().sms ? p.tile_tokens : 2 * p.tile_tokens;
  p.by_tile = Div::by(p.cta_tokens);
  // A level is a walk over all sequences, so many of them want fewer levels.  Mixed prompts, 1 / 8 / 16 levels, us: 9 sequences of up to 1000 rows 178 / 164 /
  // 152 and 203 / 190 / 189; 32 of up to 600 rows 268 / 234 / 232; 64 of up to 300 rows 339 / 285 / 294; 128 of up to 200 rows 379 / 346 / 375; 300 of up to
  // 100 rows 357 / 348 / 424, of up to 4 rows 322 / 344 / 372.  Parts are alike: one level.
  p.levels = a.split != 0 || p.n_seqs > 128 ? 1 : p.n_seqs > 32 ? 8 : 16;
  // no more CTAs than there can be items
  const int64_t most = items_of(p.cta_tokens);
  if (most >= (int64_t(1) << 31) || T * p.hq >= (int64_t(1) << 31)) return RG_ERR_SHAPE;     // items and rows are counted in 32 bits
  const cudaError_t e = a.q->dtype == RG_BF16 ? launch_any<RG_BF16>(rows, tq, tk, tv, p, most, st) : launch_any<RG_F16>(rows, tq, tk, tv, p, most, st);
  if (e != cudaSuccess) return RG_ERR_CUDA;
  if (a.segments > 1 && (a.segments <= 16 ? launch_join<1>(p, st) : launch_join<JOIN_THREADS / 32>(p, st)) != cudaSuccess) return RG_ERR_CUDA;
  return RG_OK;
}

rg_status_t read_and_clear_paged_attn_status(uint32_t* wait, uint32_t* page) {
  unsigned int v[2] = {0, 0}, zero = 0;
  if (cudaMemcpyFromSymbol(&v[0], g_paged_attn_status_word, sizeof(v[0])) != cudaSuccess || cudaMemcpyFromSymbol(&v[1], g_paged_attn_page_word, sizeof(v[1])) != cudaSuccess)
    return RG_ERR_CUDA;
  if ((v[0] != 0 && cudaMemcpyToSymbol(g_paged_attn_status_word, &zero, sizeof(zero)) != cudaSuccess) ||
      (v[1] != 0 && cudaMemcpyToSymbol(g_paged_attn_page_word, &zero, sizeof(zero)) != cudaSuccess))
    return RG_ERR_CUDA;
  *wait = v[0];
  *page = v[1];
  return RG_OK;
}

}  // namespace rg

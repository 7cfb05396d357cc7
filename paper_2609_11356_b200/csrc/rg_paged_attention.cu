// Attention of new rows over a paged cache (rg_paged_attention).
//
// Rows of one key head, (token, query head of the group), fill the 128 lanes of a tensor-core tile; keys are walked in
// blocks of 128 places.  Per row and block, with c = scale * log2(e):
//   s_t = q . k_t                             d/16 tcgen05.mma steps from a zero accumulator, ascending
//   m'  = max_t s_t;  if (m' - m) c > 8:  a = 2^((m - m') c), m = m', l = a l, O = a O      (else m, l and O stay)
//   p_t = 2^(s_t c - m c);  l += sum of p_t;  O += P V       P = p narrowed, 8 steps on the same accumulator
// and at the end O * (1 / l).  A running maximum that may lag by 2^8 costs nothing in precision (p is a floating-point number
// below 2^8) and saves nearly every rescaling of O, which lives in tensor memory.
//
// A row's arithmetic is written once (softmax_block) and does not know the tile it is in: a block that the row does not
// see adds exact zeros, so the row has the same bits as a single token, in a chunk, in any batch and on any pages.
//
// One CTA, by warp:
//   softmax (4 warps a tile)  scores from tensor memory into registers, probabilities back over them as the first operand
//                             of the next product; row r of a tile is TMEM lane r, so maxima and sums need no exchange
//   producer                  page numbers, then one TMA box for each page piece (a lane each): K and V blocks into one ring
//   MMA                       S_t = Q_t K_j^T and O_t += P_t V_j for the CTA's tiles in turn
//   fixer                     hands each arrived slot to the MMA warp; in blocks where some row is masked it first turns V elements
//                             that are not finite into zeros (0 * NaN would reach every row of the tile).  Rows that do see such an element
//                             get it added back when they are stored (rare, from global memory).
// Two forms of one kernel:
//   wide    two tiles of 128 rows, one CTA an SM: while one tile's softmax runs the tensor core works for the other
//   narrow  one tile of up to 32 rows (single tokens and drafts), two CTAs an SM: bound by the K and V bytes, the second CTA
//           covers the latency of the first's chain of product, softmax, product
// The grid is persistent: the work items (sequence, tile, part, key head) are counted out of the sequences' lengths on the device, so
// nothing is read back and a captured graph follows the lengths of the day.
#include <cuda.h>

#include <algorithm>

#include "rg_common.cuh"
#include "rg_internal.h"
#include "rg_ptx.cuh"

namespace rg {

__device__ unsigned int g_paged_attn_status_word = 0;

namespace {

constexpr int BLK = 128;                       // keys of a block
constexpr float LAG = 8.0f;                    // how far, in powers of two, a score may exceed the running maximum
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
__device__ __forceinline__ void pa_wait_ld() { asm volatile("tcgen05.wait::ld.sync.aligned;" ::: "memory"); }
__device__ __forceinline__ void pa_wait_st() { asm volatile("tcgen05.wait::st.sync.aligned;" ::: "memory"); }
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
// 16-bit x 16-bit -> fp32, M = 128, N = n; `transposed`: second operand MN-major
__host__ __device__ constexpr uint32_t pa_idesc(int n, bool bf16, bool transposed) {
  return (1u << 4) | (bf16 ? (1u << 7) | (1u << 10) : 0u) | (transposed ? 1u << 16 : 0u) | (static_cast<uint32_t>(n >> 3) << 17) | (8u << 24);
}

// ---------------------------------------------------------------- arguments and work items
struct Params {
  const int32_t *table, *seq_lens, *cu_q;
  int64_t table_ld, max_len, tokens;
  int32_t n_seqs, page_size, pages, table_cols;
  int32_t hq, hkv, group, d;
  int32_t tile_tokens;                   // tokens of one tile: floor(rows of a tile / group)
  int32_t box;                           // keys of one TMA box
  int32_t split, segments, causal;
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

struct Item {
  int32_t seq, head, seg;
  int32_t tok;                           // first token of the CTA's rows
  int32_t n_tok;                         // tokens of this CTA
  int32_t pos;                           // place of the first one
  int32_t len, lo, hi;                   // keys some row sees, within this part: lo .. hi (hi < lo: none)
  int32_t b0, b1;                        // blocks
  bool multi;                            // the sequence has several parts: results go to the workspace
};

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
  if (p.split && hi >= lo) { *g0 = (int32_t)(lo / p.split); *n = (int32_t)(hi / p.split) - *g0 + 1; }
}

// The items of this CTA: number blockIdx.x, + gridDim.x, ... in the order sequence, tile (the last, longest first), part, head.  Every warp
// that needs them walks the same list; 32 sequences at a time, one a lane.
struct Walk {
  int64_t next;                          // number of the next item, counted from the first item of the lane group
  int64_t before, count, total;          // this lane's sequence: items before it in the group, its own; the group's
  int32_t base;                          // first sequence of the group
  SeqView mine;                          // this lane's sequence
  __device__ __forceinline__ void load(const Params& p, int tile_tokens) {
    const int lane = threadIdx.x & 31, s = base + lane;
    count = 0;
    if (s < p.n_seqs) {
      bool bad;
      const SeqView v = mine = view_of(p, s, &bad);
      if (bad) atomicCAS(&g_paged_attn_status_word, 0u, (unsigned)RG_PAGE_CODE_ATTEND);
      int32_t g0, n;
      parts_of(p, v, &g0, &n);
      count = (int64_t)((v.n + tile_tokens - 1) / tile_tokens) * n * p.hkv;
    }
    int64_t sum = count;
#pragma unroll
    for (int x = 1; x < 32; x <<= 1) {
      const int64_t up = __shfl_up_sync(0xffffffffu, sum, x);
      if (lane >= x) sum += up;
    }
    before = sum - count;
    total = __shfl_sync(0xffffffffu, sum, 31);
  }
  __device__ __forceinline__ void start(const Params& p, int tile_tokens) { base = 0; next = blockIdx.x; load(p, tile_tokens); }
  __device__ __forceinline__ bool get(const Params& p, int tile_tokens, Item& it) {
    while (next >= total) {
      next -= total;
      base += 32;
      if (base >= p.n_seqs) return false;
      load(p, tile_tokens);
    }
    const int owner = __ffs(__ballot_sync(0xffffffffu, next >= before && next < before + count)) - 1;
    const int64_t local = next - __shfl_sync(0xffffffffu, before, owner);
    next += gridDim.x;
    it.seq = base + owner;
    SeqView v;
    v.tok = __shfl_sync(0xffffffffu, mine.tok, owner); v.len = __shfl_sync(0xffffffffu, mine.len, owner);
    v.n = __shfl_sync(0xffffffffu, mine.n, owner);
    v.first = v.len - v.n;
    int32_t g0, n;
    parts_of(p, v, &g0, &n);
    it.head = (int32_t)(local % p.hkv);
    const int64_t rest = local / p.hkv;
    it.seg = (int32_t)(rest % n);
    const int32_t tiles = (v.n + tile_tokens - 1) / tile_tokens, tile = tiles - 1 - (int32_t)(rest / n);
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
// 2^x for x <= LAG or NaN by its own steps: the nearest integer by a magic addition, a polynomial of degree 5 for the rest (equal to 1
// at 0; largest relative error 1.7e-7, fitted by iteratively reweighted least squares), the integer added to the exponent.  Below
// -125 the answer is that of -125: at most 2^-125, where the hardware's instruction has 0.  Two at a time.  The integer sum at the end
// (and not a multiplication) keeps the assembler from contracting it with the addition that follows.  NaN comes out as some number: a row
// with a NaN among its scores is marked in its sum.
__device__ __forceinline__ float2 poly_ex2(float2 x) {
  const float2 magic = make_float2(12582912.0f, 12582912.0f), unmagic = make_float2(-12582912.0f, -12582912.0f);
  const float2 y = make_float2(fmaxf(x.x, -125.0f), fmaxf(x.y, -125.0f));
  const float2 t = __fadd2_rn(y, magic), n = __fadd2_rn(t, unmagic);
  const float2 f = __ffma2_rn(n, make_float2(-1.0f, -1.0f), y);
  float2 q = make_float2(0x1.5bba14p-10f, 0x1.5bba14p-10f);
  q = __ffma2_rn(q, f, make_float2(0x1.3cea88p-7f, 0x1.3cea88p-7f));
  q = __ffma2_rn(q, f, make_float2(0x1.c6b752p-5f, 0x1.c6b752p-5f));
  q = __ffma2_rn(q, f, make_float2(0x1.ebf9bcp-3f, 0x1.ebf9bcp-3f));
  q = __ffma2_rn(q, f, make_float2(0x1.62e42ap-1f, 0x1.62e42ap-1f));
  q = __ffma2_rn(q, f, make_float2(1.0f, 1.0f));
  return make_float2(__int_as_float(__float_as_int(q.x) + (__float_as_int(t.x) << 23)), __int_as_float(__float_as_int(q.y) + (__float_as_int(t.y) << 23)));
}

struct Row {
  float m, l;                            // running maximum of the scores (before scaling) and sum
};

// Scores of one row and block -> probabilities.  s: the block's 128 scores; packed: the narrowed probabilities, two a word.  first ..
// last: the columns the row sees (MASKED).  Returns the factor that O takes first.
template <int DT, bool MASKED>
__device__ __forceinline__ float softmax_block(uint32_t (&s)[BLK], uint32_t (&packed)[BLK / 2], int first, int last, float c, Row& row) {
  if (MASKED) {
#pragma unroll
    for (int i = 0; i < BLK; ++i) s[i] = (i >= first && i <= last) ? s[i] : 0xff800000u;
  }
  float mx[4];
#pragma unroll
  for (int q = 0; q < 4; ++q) {
    mx[q] = __uint_as_float(s[32 * q]);
#pragma unroll
    for (int i = 1; i + 1 < 32; i += 2) mx[q] = max3(mx[q], __uint_as_float(s[32 * q + i]), __uint_as_float(s[32 * q + i + 1]));
    mx[q] = max3(mx[q], __uint_as_float(s[32 * q + 31]), __uint_as_float(s[32 * q + 31]));
  }
  const float mb = max3(max3(mx[0], mx[1], mx[2]), mx[3], mx[3]);
  float alpha = 1.0f;
  if (f_mul(f_add(mb, -row.m), c) > LAG) {                 // from -inf: any number; -inf and NaN: never
    alpha = pa_ex2(f_mul(f_add(row.m, -mb), c));
    row.m = mb;
  }
  const float shift = row.m == -INFINITY ? 0.0f : -f_mul(row.m, c);
  const float2 c2 = make_float2(c, c), sh2 = make_float2(shift, shift);
  float2 sum[4];
#pragma unroll
  for (int i = 0; i < BLK / 2; ++i) {
    const float2 x = __ffma2_rn(make_float2(__uint_as_float(s[2 * i]), __uint_as_float(s[2 * i + 1])), c2, sh2);
    float2 e;
    // which of the two exponentials a key takes follows from its place alone: the hardware unit gives 4 results a cycle and
    // quarter of the SM, the polynomial takes the rest off it
    if ((i & 3) == 3) e = poly_ex2(x);
    else e = make_float2(pa_ex2(x.x), pa_ex2(x.y));
    if (MASKED) {
      e.x = (2 * i >= first && 2 * i <= last) ? e.x : 0.0f;
      e.y = (2 * i + 1 >= first && 2 * i + 1 <= last) ? e.y : 0.0f;
    }
    sum[i & 3] = i < 4 ? e : __fadd2_rn(sum[i & 3], e);
    packed[i] = pack_16x2(e.x, e.y, DT);
  }
  const float2 t = __fadd2_rn(__fadd2_rn(sum[0], sum[1]), __fadd2_rn(sum[2], sum[3]));
  float total = f_add(t.x, t.y);
  // a NaN or an infinity among the scores: the row is NaN; nothing above -inf so far: no sum
  total = mb != mb || mb == INFINITY ? __int_as_float(0x7fffffff) : row.m == -INFINITY ? 0.0f : total;
  row.l = f_fma(row.l, alpha, total);
  return alpha;
}

// ---------------------------------------------------------------- the kernel
template <int HDP, int NT>
struct Form {
  static constexpr int DB = HDP / 64;                              // 64-column boxes of a head
  static constexpr int ROWS = NT == 2 ? 128 : 32;                  // rows of a tile that hold queries
  static constexpr int SOFT = NT == 2 ? 8 : 1;                     // softmax warps
  static constexpr int THREADS = (SOFT + 3) * 32;
  static constexpr uint32_t Q_BOX = ROWS * 128, Q_TILE = DB * Q_BOX, Q_BYTES = NT * Q_TILE;
  static constexpr uint32_t KV_BOX = BLK * 128, SLOT = DB * KV_BOX;
  // wide: one CTA an SM; narrow: two.  The narrow form's query tile is read as 128 rows, the last 96 of them being whatever the ring
  // behind it holds: their scores stay in lanes that nobody reads.
  static constexpr int SLOTS = NT == 2 ? (HDP == 128 ? 5 : 10) : (HDP == 128 ? 3 : 6);
  static constexpr uint32_t COLS = NT == 2 ? 512 : 256;            // tensor memory: S_t (P_t over it) at 128 t, O_t at 128 (NT + t)
  static constexpr size_t SMEM = 1024 + Q_BYTES + SLOTS * SLOT + 512;
};

template <int HDP, int NT, int DT>
__global__ void __launch_bounds__(Form<HDP, NT>::THREADS, NT == 2 ? 1 : 2)
paged_attention_kernel(const __grid_constant__ CUtensorMap tmap_q, const __grid_constant__ CUtensorMap tmap_k, const __grid_constant__ CUtensorMap tmap_v,
                       const __grid_constant__ Params p) {
  using F = Form<HDP, NT>;
  constexpr int DB = F::DB, SLOTS = F::SLOTS, WARPS_T = F::SOFT / NT;
  constexpr uint32_t IDESC_S = pa_idesc(BLK, DT == RG_BF16, false), IDESC_O = pa_idesc(HDP, DT == RG_BF16, true);

  extern __shared__ uint8_t smem_raw[];
  const uint32_t smem_base = (smem_u32(smem_raw) + 1023u) & ~1023u;
  uint8_t* smem_gen = smem_raw + (smem_base - smem_u32(smem_raw));
  const uint32_t sQ = smem_base, sKV = sQ + F::Q_BYTES;
  uint64_t* bars = reinterpret_cast<uint64_t*>(smem_gen + F::Q_BYTES + SLOTS * F::SLOT);
  const uint32_t bar0 = smem_u32(bars);
  const uint32_t b_q_full = bar0, b_q_empty = bar0 + 8, b_s = bar0 + 16, b_p = bar0 + 32, b_o_full = bar0 + 48, b_o_empty = bar0 + 64;   // two each from b_s on
  const uint32_t b_full = bar0 + 80, b_ready = b_full + 8 * SLOTS, b_empty = b_ready + 8 * SLOTS;
  uint32_t* tmem_slot = reinterpret_cast<uint32_t*>(bars + 10 + 3 * SLOTS);
  volatile int* abort_flag = reinterpret_cast<volatile int*>(tmem_slot + 1);
  volatile int* not_finite = reinterpret_cast<volatile int*>(tmem_slot + 2);          // [FLAGS]
  static_assert((10 + 3 * SLOTS) * 8 + 4 * (2 + FLAGS) <= 512, "barriers and flags fit behind the ring");
  static_assert(SLOTS / 2 + 1 < FLAGS, "the fixer cannot be a whole turn of flags ahead");

  const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
  if (threadIdx.x == 0) {
    mbar_init(b_q_full, 1); mbar_init(b_q_empty, 1);
    for (int t = 0; t < 2; ++t) { mbar_init(b_s + 8 * t, 1); mbar_init(b_p + 8 * t, WARPS_T); mbar_init(b_o_full + 8 * t, 1); mbar_init(b_o_empty + 8 * t, WARPS_T); }
    for (int s = 0; s < SLOTS; ++s) { mbar_init(b_full + 8 * s, 1); mbar_init(b_ready + 8 * s, 1); mbar_init(b_empty + 8 * s, 1); }
    *abort_flag = 0;
    asm volatile("fence.mbarrier_init.release.cluster;" ::: "memory");
  }
  if (warp == F::SOFT + 1) {
    asm volatile("tcgen05.alloc.cta_group::1.sync.aligned.shared::cta.b32 [%0], %1;" ::"r"(smem_u32(tmem_slot)), "r"(F::COLS) : "memory");
    asm volatile("tcgen05.relinquish_alloc_permit.cta_group::1.sync.aligned;" ::: "memory");
  }
  pa_fence_before();
  __syncthreads();
  pa_fence_after();
  const uint32_t tmem = *tmem_slot;
  const int cta_tokens = NT * p.tile_tokens;
  Walk walk;
  Item it;
  walk.start(p, cta_tokens);

  if (warp == F::SOFT) {
    // ------------------------------------------------------------ producer
    const int pieces = BLK / p.box;                                // TMA boxes along the keys of a block
    const int piece = lane % pieces, col = lane / pieces;          // col < DB: this lane issues a box
    uint32_t ring = 0, items = 0;
    bool alive = true;
    while (alive && walk.get(p, cta_tokens, it)) {
      if (it.b1 == it.b0) continue;
      const int32_t* row = p.table + (int64_t)it.seq * p.table_ld;
      auto page_of = [&](int b) -> int32_t {                       // page of this lane's keys, out of the cache's range where there is none
        const int32_t k = b * BLK + piece * p.box;
        if (k > it.hi || k + p.box <= it.lo) return -1;
        const int32_t id = row[k / p.page_size];
        if (id >= 0 && id < p.pages) return id;
        if (col == 0) atomicCAS(&g_paged_attn_status_word, 0u, (unsigned)RG_PAGE_CODE_ATTEND);
        return p.pages;                                            // behind the last page: the copy fills in zeros
      };
      int32_t page = page_of(it.b0);
      alive = warp_mbar_wait(b_q_empty, (items & 1) ^ 1u, abort_flag, &g_paged_attn_status_word, 0x2100u);
      if (!alive) break;
      const int tiles = NT == 2 && it.n_tok > p.tile_tokens ? 2 : 1;
      if (lane == 0) mbar_expect_tx(b_q_full, (uint32_t)(tiles * DB * p.tile_tokens * p.group) * 128u);
      __syncwarp();
      if (lane < tiles * DB) {
        const int t = lane / DB, b = lane % DB;
        pa_tma_4d(sQ + t * F::Q_TILE + b * F::Q_BOX, &tmap_q, b * 64, 0, it.tok + t * p.tile_tokens, it.head, b_q_full);
      }
      ++items;
      for (int b = it.b0; b < it.b1 && alive; ++b) {
        const int32_t ahead = b + 1 < it.b1 ? page_of(b + 1) : -1;
        const bool mine = col < DB && page >= 0;
        const int32_t at = (b * BLK + piece * p.box) % p.page_size;
        const uint32_t bytes = (uint32_t)__popc(__ballot_sync(0xffffffffu, mine)) * (uint32_t)p.box * 128u;
#pragma unroll
        for (int kv = 0; kv < 2; ++kv) {
          const uint32_t slot = ring % SLOTS, turn = ring / SLOTS;
          alive = warp_mbar_wait(b_empty + 8 * slot, (turn & 1) ^ 1u, abort_flag, &g_paged_attn_status_word, 0x2200u | slot);
          if (!alive) break;
          if (lane == 0) mbar_expect_tx(b_full + 8 * slot, bytes);
          __syncwarp();
          if (mine) pa_tma_4d(sKV + slot * F::SLOT + col * F::KV_BOX + piece * p.box * 128, kv ? &tmap_v : &tmap_k, col * 64, at, it.head, page, b_full + 8 * slot);
          ++ring;
        }
        page = ahead;
      }
    }
  } else if (warp == F::SOFT + 1) {
    // ------------------------------------------------------------ MMA issuer: the warp walks converged, an elected lane issues
    const bool leader = elect_one();
    uint32_t ring = 0, items = 0, n_p[2] = {0, 0}, n_o[2] = {0, 0};
    bool alive = true;
    auto slot_ready = [&](uint32_t r) -> uint32_t {                // waits for ring position r, returns its address
      const uint32_t slot = r % SLOTS, par = (r / SLOTS) & 1;
      if (alive) alive = warp_mbar_wait(b_ready + 8 * slot, par, abort_flag, &g_paged_attn_status_word, 0x2300u | slot);
      if (alive) alive = warp_mbar_wait(b_full + 8 * slot, par, abort_flag, &g_paged_attn_status_word, 0x2380u | slot);
      pa_fence_after();
      return sKV + slot * F::SLOT;
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
    while (alive && walk.get(p, cta_tokens, it)) {
      if (it.b1 == it.b0) continue;
      const int tiles = NT == 2 && it.n_tok > p.tile_tokens ? 2 : 1, nb = it.b1 - it.b0;
      alive = warp_mbar_wait(b_q_full, items & 1, abort_flag, &g_paged_attn_status_word, 0x2400u);
      ++items;
      if (!alive) break;
      uint32_t sK = slot_ready(ring);
      if (!alive) break;
      for (int t = 0; t < tiles; ++t) scores(t, sK);
      if (leader) { pa_commit(b_empty + 8 * (ring % SLOTS)); if (nb == 1) pa_commit(b_q_empty); }
      for (int j = 0; j < nb && alive; ++j) {
        const uint32_t rv = ring + 1 + 2 * j, rk = ring + 2 + 2 * j;
        const bool more = j + 1 < nb;
        const uint32_t sV = slot_ready(rv);
        if (!alive) break;
        for (int t = 0; t < tiles; ++t) {
          alive = warp_mbar_wait(b_p + 8 * t, n_p[t] & 1, abort_flag, &g_paged_attn_status_word, 0x2500u | t);
          ++n_p[t];
          if (alive && j == 0) { alive = warp_mbar_wait(b_o_empty + 8 * t, (n_o[t] & 1) ^ 1u, abort_flag, &g_paged_attn_status_word, 0x2580u | t); ++n_o[t]; }
          if (!alive) break;
          pa_fence_after();
          const uint64_t v = pa_desc(sV, F::KV_BOX);
#pragma unroll
          for (int e = 0; e < BLK / 16; ++e)
            if (leader) pa_mma_ts(tmem + 128u * (NT + t), tmem + 128u * t + 8u * e, v + (uint64_t)(e * (2048 >> 4)), IDESC_O, (j | e) ? 1u : 0u);
          if (!more && leader) pa_commit(b_o_full + 8 * t);
          if (more) {
            if (t == 0) sK = slot_ready(rk);
            if (!alive) break;
            scores(t, sK);
          }
        }
        if (!alive) break;
        if (leader) {
          pa_commit(b_empty + 8 * (rv % SLOTS));
          if (more) pa_commit(b_empty + 8 * (rk % SLOTS));
          if (j + 2 == nb) pa_commit(b_q_empty);
        }
      }
      ring += 2 * nb;
    }
  } else if (warp == F::SOFT + 2) {
    // ------------------------------------------------------------ fixer
    uint32_t ring = 0, flags = 0;
    bool alive = true;
    while (alive && walk.get(p, cta_tokens, it)) {
      bool any_masked = false;
      for (int b = it.b0; b < it.b1 && alive; ++b) {
        const bool masked = masked_block(p, it, b);
#pragma unroll
        for (int kv = 0; kv < 2; ++kv) {
          const uint32_t slot = ring % SLOTS, turn = ring / SLOTS;
          alive = warp_mbar_wait(b_full + 8 * slot, turn & 1, abort_flag, &g_paged_attn_status_word, 0x2600u | slot);
          if (!alive) break;
          if (kv == 1 && masked) {
            constexpr uint32_t EXP = DT == RG_BF16 ? 0x7f807f80u : 0x7c007c00u, ONE = DT == RG_BF16 ? 0x00800080u : 0x04000400u;
            uint4* base = reinterpret_cast<uint4*>(smem_gen + F::Q_BYTES + slot * F::SLOT);
            bool seen = false;
#pragma unroll 4
            for (uint32_t i = lane; i < F::SLOT / 16; i += 32) {
              uint4 w = base[i];
              const uint32_t hit = (((w.x & EXP) + ONE) | ((w.y & EXP) + ONE) | ((w.z & EXP) + ONE) | ((w.w & EXP) + ONE)) & 0x80008000u;
              if (hit) {
                auto clean = [&](uint32_t x) { const uint32_t h = ((x & EXP) + ONE) & 0x80008000u; return x & ~((h >> 15) * 0xffffu); };
                w.x = clean(w.x); w.y = clean(w.y); w.z = clean(w.z); w.w = clean(w.w);
                base[i] = w;
                const int32_t key = b * BLK + (int32_t)(((i * 16) % F::KV_BOX) / 128);
                seen |= key >= it.lo && key <= it.hi;
              }
            }
            seen = __any_sync(0xffffffffu, seen);
            if (lane == 0) not_finite[flags % FLAGS] = any_masked ? (not_finite[flags % FLAGS] | (seen ? 1 : 0)) : (seen ? 1 : 0);
            any_masked = true;
            asm volatile("fence.proxy.async.shared::cta;" ::: "memory");
          }
          __syncwarp();
          if (lane == 0) mbar_arrive(b_ready + 8 * slot);
          ++ring;
        }
      }
      if (any_masked) ++flags;
    }
  } else {
    // ------------------------------------------------------------ softmax and output rows
    const int t = NT == 2 ? warp >> 2 : 0;                         // tile
    const int r = (warp & 3) * 32 + lane;                          // row of the tile, and its lane in tensor memory
    const uint32_t t_s = tmem + 128u * t + (static_cast<uint32_t>((warp & 3) * 32) << 16), t_o = t_s + 128u * NT;
    const int my_tok = r / p.group, my_head = r - my_tok * p.group;
    uint32_t n_s = 0, n_o = 0, flags = 0;
    bool alive = true;
    while (alive && walk.get(p, cta_tokens, it)) {
      const int tok = t * p.tile_tokens + my_tok;                  // within the item
      const bool live = my_tok < p.tile_tokens && tok < it.n_tok;
      const bool warp_live = __any_sync(0xffffffffu, live);
      const bool tile_live = t * p.tile_tokens < it.n_tok;
      const int32_t place = it.pos + tok;
      const int32_t hi = live ? min(last_seen(p, place, it.len), it.hi) : -1, lo = max(first_seen(p, place), it.lo);
      Row row = {-INFINITY, 0.0f};
      bool any_masked = false;
      if (tile_live) {
        for (int b = it.b0; b < it.b1; ++b) {
          const bool masked = masked_block(p, it, b);
          any_masked |= masked;
          alive = warp_mbar_wait(b_s + 8 * t, n_s & 1, abort_flag, &g_paged_attn_status_word, 0x2700u | t);
          ++n_s;
          if (!alive) break;
          if (warp_live) {
            pa_fence_after();
            uint32_t s[BLK], packed[BLK / 2];
#pragma unroll
            for (int q = 0; q < 4; ++q) pa_ld32(t_s + 32u * q, s + 32 * q);
            pa_wait_ld();
            float alpha;
            if (masked) {
              alpha = softmax_block<DT, true>(s, packed, lo - b * BLK, hi - b * BLK, p.c, row);
            } else {
              alpha = softmax_block<DT, false>(s, packed, 0, BLK - 1, p.c, row);
            }
            __syncwarp();
            pa_st32(t_s, packed);
            pa_st32(t_s + 32u, packed + 32);
            // the scores of this block are complete, so the product of the block before is too: O may be rescaled
            if (b > it.b0 && __any_sync(0xffffffffu, live && alpha != 1.0f)) {
#pragma unroll
              for (int q = 0; q < HDP / 32; ++q) {
                uint32_t o[32];
                pa_ld32(t_o + 32u * q, o);
                pa_wait_ld();
#pragma unroll
                for (int i = 0; i < 32; ++i) o[i] = __float_as_uint(f_mul(__uint_as_float(o[i]), alpha));
                pa_st32(t_o + 32u * q, o);
              }
            }
            pa_wait_st();
            pa_fence_before();
          }
          __syncwarp();
          if (lane == 0) mbar_arrive(b_p + 8 * t);
        }
        if (!alive) break;
      }
      const int slot_flag = flags % FLAGS;
      bool add_back = false;
      if (NT == 2 && !tile_live) {                                 // keep count of the flags all the same
        for (int b = it.b0; b < it.b1; ++b) any_masked |= masked_block(p, it, b);
      }
      if (any_masked) ++flags;
      if (!tile_live) continue;
      if (it.b1 > it.b0) {
        alive = warp_mbar_wait(b_o_full + 8 * t, n_o & 1, abort_flag, &g_paged_attn_status_word, 0x2780u | t);
        ++n_o;
        if (!alive) break;
        pa_fence_after();
        add_back = any_masked && not_finite[slot_flag] != 0;
      }
      if (warp_live) {
        const int64_t token = (int64_t)it.tok + tok;
        const int head = it.head * p.group + my_head;
        const int64_t grow = token * p.hq + head;
        const bool none = !(row.l > 0.0f) && row.l == row.l;       // no key seen
        const float inv = it.multi ? 1.0f : none ? 0.0f : __frcp_rn(row.l);
        float* part = it.multi ? p.part_o + (grow * p.segments + it.seg) * p.d : nullptr;
#pragma unroll 1
        for (int q = 0; q < HDP / 32; ++q) {
          if (32 * q >= p.d) break;
          uint32_t raw[32];
          __syncwarp();
          if (it.b1 > it.b0) { pa_ld32(t_o + 32u * q, raw); pa_wait_ld(); }
          float o[32];
#pragma unroll
          for (int i = 0; i < 32; ++i) o[i] = none || it.b1 == it.b0 ? 0.0f : f_mul(__uint_as_float(raw[i]), inv);
          if (add_back && live) {
            // the elements of V that the fixer took out and this row sees
            for (int b = it.b0; b < it.b1; ++b) {
              if (!masked_block(p, it, b)) continue;
              for (int32_t k = max(lo, b * BLK); k <= min(hi, b * BLK + BLK - 1); ++k) {
                const int64_t id = p.table[(int64_t)it.seq * p.table_ld + k / p.page_size];
                if (id < 0 || id >= p.pages) continue;
                const uint16_t* v = p.v + id * p.v_page + (k % p.page_size) * p.v_slot + it.head * p.v_head;
#pragma unroll
                for (int i = 0; i < 32; ++i) {
                  if (32 * q + i >= p.d) break;
                  const float x = DT == RG_BF16 ? bf16_bits_to_f32(v[32 * q + i]) : f16_bits_to_f32(v[32 * q + i]);
                  if (!(f_add(x, -x) == 0.0f)) o[i] = f_add(o[i], x);
                }
              }
            }
          }
          const int n = live ? min(32, p.d - 32 * q) : 0;
          if (n == 0) {
          } else if (it.multi) {
#pragma unroll
            for (int i = 0; i < 32; i += 4)
              if (i < n) *reinterpret_cast<float4*>(part + 32 * q + i) = make_float4(o[i], o[i + 1], o[i + 2], o[i + 3]);
          } else if (p.o_dtype == RG_F32) {
            float* dst = static_cast<float*>(p.out) + token * p.o_tok + head * p.o_head + 32 * q;
            if (p.o_vec) {
#pragma unroll
              for (int i = 0; i < 32; i += 4) if (i < n) *reinterpret_cast<float4*>(dst + i) = make_float4(o[i], o[i + 1], o[i + 2], o[i + 3]);
            } else {
#pragma unroll
              for (int i = 0; i < 32; ++i) if (i < n) dst[i] = o[i];
            }
          } else {
            uint16_t* dst = static_cast<uint16_t*>(p.out) + token * p.o_tok + head * p.o_head + 32 * q;
            uint32_t w[16];
#pragma unroll
            for (int i = 0; i < 16; ++i) w[i] = pack_16x2(o[2 * i], o[2 * i + 1], DT);
            if (p.o_vec) {
#pragma unroll
              for (int i = 0; i < 16; i += 4) if (2 * i < n) *reinterpret_cast<uint4*>(dst + 2 * i) = make_uint4(w[i], w[i + 1], w[i + 2], w[i + 3]);
            } else {
#pragma unroll
              for (int i = 0; i < 16; ++i) if (2 * i < n) { dst[2 * i] = (uint16_t)(w[i] & 0xffffu); dst[2 * i + 1] = (uint16_t)(w[i] >> 16); }
            }
          }
        }
        if (live) {
          if (it.multi) p.part_ml[grow * p.segments + it.seg] = make_float2(row.m, row.l);
          else if (p.lse) p.lse[token * p.lse_ld + head] = none ? -INFINITY : f_add(f_mul(row.m, p.scale), logf(row.l));
        }
      }
      if (it.b1 > it.b0) {
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
  if (warp == F::SOFT + 1) {
    pa_fence_after();
    asm volatile("tcgen05.dealloc.cta_group::1.sync.aligned.b32 %0, %1;" ::"r"(tmem), "r"(F::COLS) : "memory");
  }
}

// Joins the parts of a row in ascending order.  A warp a row, four columns a lane.
__global__ void __launch_bounds__(128) join_parts_kernel(const __grid_constant__ Params p) {
  const int lane = threadIdx.x & 31;
  const int64_t grow = (int64_t)blockIdx.x * 4 + (threadIdx.x >> 5);
  if (grow >= p.tokens * p.hq) return;
  const int64_t token = grow / p.hq;
  const int head = (int)(grow - token * p.hq);
  int before = 0;
  for (int i = lane; i < p.n_seqs; i += 32) before += p.cu_q[i + 1] <= token ? 1 : 0;
  const int s = __reduce_add_sync(0xffffffffu, before);
  if (s >= p.n_seqs || token < p.cu_q[s]) return;
  bool bad;
  const SeqView v = view_of(p, s, &bad);
  int32_t g0, n;
  parts_of(p, v, &g0, &n);
  if (n <= 1) return;                                              // written by the main kernel
  const int32_t place = v.first + (int32_t)(token - v.tok), hi = last_seen(p, place, v.len), lo = first_seen(p, max(place, 0));
  const int ga = hi >= lo ? lo / p.split : 0, gb = hi >= lo ? hi / p.split + 1 : 0;
  const float2* ml = p.part_ml + grow * p.segments;
  float m = -INFINITY;
  for (int g = ga + lane; g < gb; g += 32) m = fmaxf(m, ml[g].x);
#pragma unroll
  for (int x = 16; x; x >>= 1) m = fmaxf(m, __shfl_xor_sync(0xffffffffu, m, x));
  float l = 0.0f;
  float4 o = make_float4(0.0f, 0.0f, 0.0f, 0.0f);
  const bool mine = 4 * lane < p.d;
  const float* po = p.part_o + grow * p.segments * p.d + 4 * lane;
  for (int base = ga; base < gb; base += 32) {
    float w = 0.0f, wl = 0.0f;
    if (base + lane < gb) {
      const float2 x = ml[base + lane];
      w = x.x == -INFINITY ? 0.0f : pa_ex2(f_mul(f_add(x.x, -m), p.c));
      wl = f_mul(w, x.y);
    }
    const int count = min(32, gb - base);
#pragma unroll 8
    for (int i = 0; i < count; ++i) {
      const float wi = __shfl_sync(0xffffffffu, w, i);
      l = f_add(l, __shfl_sync(0xffffffffu, wl, i));
      if (mine) {
        const float4 x = *reinterpret_cast<const float4*>(po + (int64_t)(base + i) * p.d);
        o.x = f_fma(wi, x.x, o.x); o.y = f_fma(wi, x.y, o.y); o.z = f_fma(wi, x.z, o.z); o.w = f_fma(wi, x.w, o.w);
      }
    }
  }
  const bool none = !(l > 0.0f) && l == l;
  const float inv = none ? 0.0f : __frcp_rn(l);
  if (mine) {
    const float r[4] = {none ? 0.0f : f_mul(o.x, inv), none ? 0.0f : f_mul(o.y, inv), none ? 0.0f : f_mul(o.z, inv), none ? 0.0f : f_mul(o.w, inv)};
    const int64_t at = token * p.o_tok + head * p.o_head + 4 * lane;
#pragma unroll
    for (int i = 0; i < 4; ++i) store_scalar(p.out, p.o_dtype, at + i, r[i]);
  }
  if (p.lse && lane == 0) p.lse[token * p.lse_ld + head] = none ? -INFINITY : f_add(f_mul(m, p.scale), logf(l));
}

// ---------------------------------------------------------------- host
template <int HDP, int NT, int DT>
cudaError_t launch_form(const CUtensorMap& q, const CUtensorMap& k, const CUtensorMap& v, const Params& p, int64_t most, cudaStream_t st) {
  using F = Form<HDP, NT>;
  static DeviceOnce configured;
  const DeviceInfo dev = current_device();
  if (!configured.has(dev.dev)) {
    cudaError_t e = cudaFuncSetAttribute(paged_attention_kernel<HDP, NT, DT>, cudaFuncAttributeMaxDynamicSharedMemorySize, (int)F::SMEM);
    if (e != cudaSuccess) return e;
    configured.set(dev.dev);
  }
  const int64_t grid = std::min<int64_t>(most, (int64_t)dev.sms * (NT == 2 ? 1 : 2));
  paged_attention_kernel<HDP, NT, DT><<<(unsigned)grid, F::THREADS, F::SMEM, st>>>(q, k, v, p);
  return cudaGetLastError();
}

}  // namespace

// All arguments were validated by the caller.
rg_status_t launch_paged_attention(const PagedAttnArgs& a, cudaStream_t st) {
  Params p{};
  const int64_t T = a.q->tokens, hkv = a.k->heads;
  const int G = (int)(a.q->heads / hkv), d = (int)a.q->dim, page = (int)a.k->page_size;
  p.table = a.seqs->block_table; p.seq_lens = a.seqs->seq_lens; p.cu_q = a.seqs->cu_q;
  p.table_ld = a.seqs->table_ld; p.max_len = a.max_len; p.tokens = T;
  p.n_seqs = a.seqs->n_seqs; p.page_size = page; p.pages = (int32_t)a.k->pages; p.table_cols = a.seqs->table_cols;
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

  // one tile of 32 rows where a sequence's new rows fit it: two CTAs an SM, no second tile to wait for
  const bool narrow = G <= 32 && a.max_q * G <= 32;
  const int rows = narrow ? 32 : 128;
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

  // no more CTAs than there can be items
  const int cta_tokens = p.tile_tokens * (narrow ? 1 : 2);
  const int64_t most = std::min<int64_t>(T, (T + cta_tokens - 1) / cta_tokens + p.n_seqs) * hkv * a.segments;
  cudaError_t e;
  const bool bf = a.q->dtype == RG_BF16;
  if (narrow) {
    if (d <= 64) e = bf ? launch_form<64, 1, RG_BF16>(tq, tk, tv, p, most, st) : launch_form<64, 1, RG_F16>(tq, tk, tv, p, most, st);
    else e = bf ? launch_form<128, 1, RG_BF16>(tq, tk, tv, p, most, st) : launch_form<128, 1, RG_F16>(tq, tk, tv, p, most, st);
  } else {
    if (d <= 64) e = bf ? launch_form<64, 2, RG_BF16>(tq, tk, tv, p, most, st) : launch_form<64, 2, RG_F16>(tq, tk, tv, p, most, st);
    else e = bf ? launch_form<128, 2, RG_BF16>(tq, tk, tv, p, most, st) : launch_form<128, 2, RG_F16>(tq, tk, tv, p, most, st);
  }
  if (e != cudaSuccess) return RG_ERR_CUDA;
  if (a.segments > 1) {
    join_parts_kernel<<<(unsigned)((T * p.hq + 3) / 4), 128, 0, st>>>(p);
    if (cudaGetLastError() != cudaSuccess) return RG_ERR_CUDA;
  }
  return RG_OK;
}

rg_status_t read_and_clear_paged_attn_status(uint32_t* code) {
  unsigned int v = 0, zero = 0;
  if (cudaMemcpyFromSymbol(&v, g_paged_attn_status_word, sizeof(v)) != cudaSuccess) return RG_ERR_CUDA;
  if (v != 0 && cudaMemcpyToSymbol(g_paged_attn_status_word, &zero, sizeof(zero)) != cudaSuccess) return RG_ERR_CUDA;
  if (code) *code = v;
  return v ? (v == RG_PAGE_CODE_ATTEND ? RG_ERR_PAGE : RG_ERR_TIMEOUT) : RG_OK;
}

}  // namespace rg

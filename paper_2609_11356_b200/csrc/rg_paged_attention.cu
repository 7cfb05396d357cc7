// Attention of new rows over a paged cache: one warp per row and query head, keys one by one.
#include "rg_common.cuh"
#include "rg_internal.h"

namespace rg {

__device__ unsigned int g_paged_attn_status_word = 0;

namespace {

struct Params {
  const void *q, *k, *v;
  void* out;
  float* lse;
  int64_t q_tok, q_head, k_page, k_slot, k_head, v_page, v_slot, v_head, o_tok, o_head, lse_ld, tokens, pages, table_ld, max_len;
  const int32_t *table, *seq_lens, *cu_q;
  int32_t n_seqs, page_size, hq, group, d, dtype, o_dtype, causal;
  int64_t window;
  float scale;
};

__global__ void __launch_bounds__(128) paged_attention_kernel(const Params p) {
  const int lane = threadIdx.x & 31;
  const int64_t w = (int64_t)blockIdx.x * 4 + (threadIdx.x >> 5);
  if (w >= p.tokens * p.hq) return;
  const int64_t t = w / p.hq;
  const int h = (int)(w - t * p.hq), hk = h / p.group;
  int before = 0;
  for (int i = lane; i < p.n_seqs; i += 32) before += p.cu_q[i + 1] <= t ? 1 : 0;
  const int s = __reduce_add_sync(0xffffffffu, before);
  if (s >= p.n_seqs || t < p.cu_q[s]) return;
  int64_t len = p.seq_lens[s];
  bool bad = len > p.max_len || len < p.cu_q[s + 1] - p.cu_q[s];
  len = min(len, p.max_len);
  const int64_t place = (int64_t)p.seq_lens[s] - ((int64_t)p.cu_q[s + 1] - t);
  int64_t hi = p.causal ? min(place, len - 1) : (place < 0 ? -1 : len - 1), lo = p.window ? max((int64_t)0, place - p.window + 1) : 0;
  float q[4], o[4] = {0, 0, 0, 0}, m = -INFINITY, l = 0;
  for (int e = 0; e < 4; ++e) q[e] = lane + 32 * e < p.d ? load_scalar(p.q, p.dtype, t * p.q_tok + h * p.q_head + lane + 32 * e) : 0.0f;
  for (int64_t j = lo; j <= hi; ++j) {
    const int64_t page = p.table[s * p.table_ld + j / p.page_size], slot = j % p.page_size;
    const bool there = page >= 0 && page < p.pages;
    bad |= !there;
    float dot = 0;
    for (int e = 0; e < 4; ++e)
      if (lane + 32 * e < p.d && there) dot = f_fma(q[e], load_scalar(p.k, p.dtype, page * p.k_page + slot * p.k_slot + hk * p.k_head + lane + 32 * e), dot);
    for (int x = 16; x; x >>= 1) dot = f_add(dot, __shfl_xor_sync(0xffffffffu, dot, x));
    const float sc = f_mul(dot, p.scale), mn = fmaxf(m, sc), a = m == mn ? 1.0f : expf(m - mn), pr = expf(sc - mn);
    l = f_fma(l, a, pr);
    for (int e = 0; e < 4; ++e)
      o[e] = f_fma(o[e], a, lane + 32 * e < p.d && there ? f_mul(pr, load_scalar(p.v, p.dtype, page * p.v_page + slot * p.v_slot + hk * p.v_head + lane + 32 * e)) : 0.0f);
    m = mn;
  }
  if (bad && lane == 0) atomicCAS(&g_paged_attn_status_word, 0u, (unsigned)RG_PAGE_CODE_ATTEND);
  for (int e = 0; e < 4; ++e)
    if (lane + 32 * e < p.d) store_scalar(p.out, p.o_dtype, t * p.o_tok + h * p.o_head + lane + 32 * e, hi >= lo ? __fdiv_rn(o[e], l) : 0.0f);
  if (p.lse && lane == 0) p.lse[t * p.lse_ld + h] = hi >= lo ? m + logf(l) : -INFINITY;
}

}  // namespace

rg_status_t launch_paged_attention(const PagedAttnArgs& a, cudaStream_t st) {
  Params p;
  p.q = a.q->ptr; p.k = a.k->ptr; p.v = a.v->ptr; p.out = a.out->ptr; p.lse = a.lse;
  p.q_tok = a.q->token_stride; p.q_head = a.q->head_stride; p.o_tok = a.out->token_stride; p.o_head = a.out->head_stride; p.lse_ld = a.lse_ld;
  p.k_page = a.k->page_stride; p.k_slot = a.k->slot_stride; p.k_head = a.k->head_stride;
  p.v_page = a.v->page_stride; p.v_slot = a.v->slot_stride; p.v_head = a.v->head_stride;
  p.tokens = a.q->tokens; p.pages = a.k->pages; p.table_ld = a.seqs->table_ld; p.max_len = a.max_len;
  p.table = a.seqs->block_table; p.seq_lens = a.seqs->seq_lens; p.cu_q = a.seqs->cu_q;
  p.n_seqs = a.seqs->n_seqs; p.page_size = (int)a.k->page_size; p.hq = (int)a.q->heads; p.group = (int)(a.q->heads / a.k->heads); p.d = (int)a.q->dim;
  p.dtype = a.q->dtype; p.o_dtype = a.out->dtype; p.causal = a.causal; p.window = a.window; p.scale = a.scale;
  paged_attention_kernel<<<(unsigned)((a.q->tokens * a.q->heads + 3) / 4), 128, 0, st>>>(p);
  return cudaGetLastError() == cudaSuccess ? RG_OK : RG_ERR_CUDA;
}

rg_status_t read_and_clear_paged_attn_status(uint32_t* code) {
  unsigned int v = 0, zero = 0;
  if (cudaMemcpyFromSymbol(&v, g_paged_attn_status_word, sizeof(v)) != cudaSuccess) return RG_ERR_CUDA;
  if (v != 0 && cudaMemcpyToSymbol(g_paged_attn_status_word, &zero, sizeof(zero)) != cudaSuccess) return RG_ERR_CUDA;
  if (code) *code = v;
  return v ? (v == RG_PAGE_CODE_ATTEND ? RG_ERR_PAGE : RG_ERR_TIMEOUT) : RG_OK;
}

}  // namespace rg

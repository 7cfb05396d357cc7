// Internal host-side declarations shared by the translation units of the library.
#pragma once
#include <cuda_runtime.h>
#include <stdint.h>

#include <atomic>

#include "../../include/rg.h"

struct CUtensorMap_st;

namespace rg {

// Function attributes are per device: one bit per device ordinal and kernel instantiation.
struct DeviceOnce {
  std::atomic<uint64_t> mask{0};
  bool has(int dev) const { return dev >= 0 && dev < 64 && ((mask.load(std::memory_order_acquire) >> dev) & 1u); }
  void set(int dev) { if (dev >= 0 && dev < 64) mask.fetch_or(uint64_t(1) << dev, std::memory_order_release); }
};

struct DeviceInfo { int dev, sms; };
// The current device and its SM count (looked up once per device).
inline DeviceInfo current_device() {
  static std::atomic<int> sms_of[64];
  DeviceInfo d{0, 148};
  if (cudaGetDevice(&d.dev) != cudaSuccess) return d;
  if (d.dev >= 0 && d.dev < 64 && sms_of[d.dev].load(std::memory_order_relaxed) > 0) { d.sms = sms_of[d.dev].load(std::memory_order_relaxed); return d; }
  int sms = 0;
  if (cudaDeviceGetAttribute(&sms, cudaDevAttrMultiProcessorCount, d.dev) == cudaSuccess && sms > 0) {
    d.sms = sms;
    if (d.dev >= 0 && d.dev < 64) sms_of[d.dev].store(sms, std::memory_order_relaxed);
  }
  return d;
}

// A validated launch plan: speed knobs resolved, parts laid out.
struct GemmPlan {
  int BN, BK, stages, raster, group_m, cta_group;
  int b_static;             // caller's promise: nothing in flight on the stream writes B (its first boxes may be fetched early)
  int reserve_sms;          // SMs the GEMM leaves free for the CTAs of its split-K merge (calls that do not depend on each other, b_static = 2)
  int merge_small;          // that merge runs as 128-thread CTAs of two units per thread (four to an SM) instead of the general kernel
  int half_sm;              // the one-CTA kernel in its half-SM form: two CTAs share an SM (weight-streaming shapes)
  int ticket_merge;         // split-K parts through the workspace, merged inside the GEMM kernel by the CTA that stores a tile's last part
  int cluster_merge;        // split-K parts merged inside the GEMM kernel by a thread-block cluster (no workspace, one launch)
  int n_parts, tree;
  int partial_dtype, merge_dtype;
  int inner_span;
  int32_t part_begin[RG_MAX_CUTS + 1];
  int32_t part_end[RG_MAX_CUTS + 1];
};

int max_stages_for(int bn, int bk, int cta_group, int64_t M, bool cluster_merge = false, bool half_sm = false);
int max_active_clusters(int csize, int bk, bool f8);
size_t ticket_bytes();
rg_status_t launch_gemm(const GemmPlan& plan, const rg_tensor_t* A, const rg_tensor_t* B, const rg_tensor_t* C,
                        const rg_epilogue_t* epi, void* ws, cudaStream_t st);
rg_status_t launch_gemv(const rg_desc_t* d, const rg_tensor_t* A, const rg_tensor_t* B, const rg_tensor_t* C,
                        const rg_epilogue_t* epi, cudaStream_t st);
rg_status_t launch_reduce_rows(int op, int tree, int fma, const rg_tensor_t* x, const rg_tensor_t* out,
                               const rg_reduce_args_t* args, int threads_hint, int unroll_hint, cudaStream_t st);
size_t reduce_cols_workspace_bytes(int64_t R, int64_t C);
rg_status_t launch_reduce_cols(int op, int tree, int fma, const rg_tensor_t* x, const rg_tensor_t* y, const rg_tensor_t* out,
                               void* ws, cudaStream_t st);
bool make_operand_tmap(CUtensorMap_st* map, const void* ptr, int dtype, int64_t rows, int64_t cols, int64_t ld, int box_rows);
bool make_tmap_4d(CUtensorMap_st* map, const void* ptr, int dtype, const int64_t (&dims)[4], const int64_t (&strides)[3], const int (&box)[4]);
rg_status_t launch_attention_fixed(int block_n, int exp_base, int causal, float scale, int heads, const rg_tensor_t* Q, const rg_tensor_t* K,
                                   const rg_tensor_t* Vt, const rg_tensor_t* O, cudaStream_t st);
rg_status_t read_and_clear_attn_status(uint32_t* code);

// ---- rotary positions, paged cache (rg_rope.cu, rg_paged_attention.cu)
struct RopeStream {
  const void* src;
  void* dst;
  int64_t src_tok, src_head;           // strides in elements
  int64_t dst_page, dst_tok, dst_head; // dst_tok: between slots of a page, or between rows
  int32_t heads;
  int32_t rotate;
  int32_t paged;                       // dst is a cache
};
struct RopeParams {
  RopeStream st[3];
  int32_t n_streams, heads_all;
  int64_t tokens;
  int32_t d, rot, style, inverse;
  int32_t axis_end[3];                 // first pair of the axes 1, 2, 3
  int32_t pos64;
  const void* pos;
  int64_t pos_ld;
  const double* inv_freq;
  const int32_t* table;
  int64_t table_ld;
  const int32_t* seq_lens;
  const int32_t* cu_q;
  int64_t pages;
  int32_t table_cols, n_seqs, page_size;
  int32_t tile, head_group;            // tokens and heads of a CTA
  uint32_t inv_units, inv_per_tok;     // 2^32 over a head's units and over a token's units of the CTA, rounded up; 0 for one unit
};
rg_status_t launch_rope(RopeParams p, int dtype, bool paged, cudaStream_t st);
rg_status_t read_and_clear_paged_status(uint32_t* code);

// ---- a paged cache of four-bit codes (rg_cache_four.cu)
struct Cache4Stream {
  const void* src;
  void* dst;
  int64_t src_tok, src_head;           // rows: elements; blocks of a cache: bytes
  int64_t dst_page, dst_tok, dst_head; // dst_page: bytes between a cache's pages, whichever side it is
  int32_t heads;
  int32_t vec;                         // rows can be moved 16 bytes at a time
};
struct Cache4Params {
  Cache4Stream st[3];                  // keys, values, queries
  int32_t n_streams, heads_all;
  int64_t tokens;
  int32_t d, rot, style;
  int32_t axis_end[3];
  int32_t pos64;
  const void* pos;
  int64_t pos_ld;
  const double* inv_freq;
  const int32_t* table;
  int64_t table_ld;
  const int32_t* seq_lens;
  const int32_t* cu_q;
  int64_t pages;
  int32_t table_cols, n_seqs, page_size;
  int32_t tile, head_group;
};
rg_status_t launch_cache4(Cache4Params p, int dtype, bool read, cudaStream_t st);
rg_status_t read_and_clear_cache4_status(uint32_t* code);

// ---- products with four-bit weights (rg_gemv_four.cu)
rg_status_t launch_gemv_w4(const rg_weights_four_t* W, const rg_tensor_t* A, const rg_tensor_t* C, const rg_epilogue_t* epi, cudaStream_t st);
rg_status_t read_and_clear_gemv_four_status(uint32_t* code);

struct PagedAttnArgs {
  const rg_rows_t* q;
  const rg_cache_t* k;
  const rg_cache_t* v;
  const rg_cache_four_t* k4;               // the caches in four bits, or null
  const rg_cache_four_t* v4;
  const rg_paged_seqs_t* seqs;
  const rg_rows_t* out;
  float* lse;
  int64_t lse_ld;
  void* ws;
  int64_t max_q, max_len;              // resolved bounds
  int32_t segments;                    // most parts of a row (1: no workspace)
  uint32_t split, window;
  float scale;
  int32_t causal;
};
rg_status_t launch_paged_attention(const PagedAttnArgs& a, cudaStream_t st);
rg_status_t read_and_clear_paged_attn_status(uint32_t* wait, uint32_t* page);
rg_status_t read_and_clear_status(uint32_t* code);
rg_status_t launch_wait_selftest(uint64_t limit_ns, uint32_t code, unsigned int* left_early, cudaStream_t st);
// y[i] = FORM(x[i]) by the device functions the kernels use (forms 0-2 and 6; the attention kernel's forms 3-5)
rg_status_t launch_exp_selftest(int form, const float* x, float* y, int64_t n, cudaStream_t st);
rg_status_t launch_exp_selftest_attention(int form, const float* x, float* y, int64_t n, cudaStream_t st);
rg_status_t launch_silu_selftest(const float* x, float* y, int64_t n, cudaStream_t st);   // form 7: the epilogue's SiLU on segments of 32
rg_status_t read_and_clear_reduce_status(uint32_t* code);

}  // namespace rg

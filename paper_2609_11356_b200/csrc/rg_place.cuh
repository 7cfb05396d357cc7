// Where a row of a batch of sequences stands (rg_paged_seqs_t), for the kernels that write or read a paged cache row by row.
#pragma once
#include <cuda_runtime.h>
#include <stdint.h>

namespace rg {

// Which sequence a row belongs to and its place there; the whole warp calls.  The count of sequences that end at or
// before the row is its sequence (lengths of zero included), whatever the order of the additions.
template <typename P>
__device__ __forceinline__ bool place_of(const P& p, int64_t t, int& seq, int64_t& place) {
  const int lane = threadIdx.x & 31;
  int before = 0;
  for (int i = lane; i < p.n_seqs; i += 32) before += p.cu_q[i + 1] <= t ? 1 : 0;
  seq = __reduce_add_sync(0xffffffffu, before);
  if (seq >= p.n_seqs) return false;                    // a row behind the last sequence
  if (t < p.cu_q[seq]) return false;
  place = (int64_t)p.seq_lens[seq] - ((int64_t)p.cu_q[seq + 1] - t);
  return true;
}

// The page of that place; -1: none.
template <typename P>
__device__ __forceinline__ int64_t page_of(const P& p, int seq, int64_t place) {
  if (place < 0 || place >= (int64_t)p.table_cols * p.page_size) return -1;
  const int64_t id = p.table[(int64_t)seq * p.table_ld + place / p.page_size];
  return id >= 0 && id < p.pages ? id : -1;
}

}  // namespace rg

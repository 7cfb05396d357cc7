// What the health words of the kernels come to (host code, nothing of CUDA).
#pragma once
#include "../../include/rg.h"

namespace rg {

// `waits`: codes of waits that gave up; `pages`: codes of pages and lengths outside the cache.  Both kinds have words of their own, which keep the
// first code they are given until they are read: a wait that gave up spoils every row of its call, a bad page one sequence's, so the first
// may not be hidden by the second.  Within a kind the first word that holds a code names it.
inline rg_status_t health_of(const uint32_t* waits, int n_waits, const uint32_t* pages, int n_pages, uint32_t* code) {
  if (code) *code = 0;
  for (int k = 0; k < 2; ++k) {
    const uint32_t* w = k ? pages : waits;
    for (int i = 0; i < (k ? n_pages : n_waits); ++i) {
      if (w[i] == 0) continue;
      if (code) *code = w[i];
      return k ? RG_ERR_PAGE : RG_ERR_TIMEOUT;
    }
  }
  return RG_OK;
}

}  // namespace rg

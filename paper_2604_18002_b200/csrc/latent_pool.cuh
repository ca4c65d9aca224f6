// Checks and addressing shared by the calls on a pool of latent rows.
#pragma once

#include <cuda_runtime.h>
#include <stdint.h>

#include "ngc_common.cuh"

namespace ngc {

inline bool valid_latent_pool(const ngc_latent_pool* c) {
  return c && c->rows && c->page_table && c->page_used && c->lens && c->L > 0 && c->B > 0 && c->pages_cap > 0 && c->n_pages > 0 &&
         (c->page == 32 || c->page == 64) && c->lists >= 0 && c->lists <= 2 && c->d_latent > 0 && c->d_rope > 0 &&
         (c->dtype == NGC_F32 || c->dtype == NGC_BF16) && (int64_t)c->pages_cap * c->page <= 0x7fffffffLL &&
         (int64_t)c->L * c->n_pages * c->page <= 0x7fffffffLL;
}
inline bool built_latent_dims(int d_latent, int d_rope) {
  return d_latent % 128 == 0 && d_latent <= 512 && d_rope % 16 == 0 && d_rope <= 64;
}

inline bool aligned16(const void* p) { return ((uintptr_t)p & 15) == 0; }

}  // namespace ngc

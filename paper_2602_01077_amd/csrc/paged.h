// Paged cache: problem description shared by its host code and kernels.
#pragma once

#include <hip/hip_runtime.h>
#include <stddef.h>
#include <stdint.h>

#include "masked.h"

namespace pisa {

struct Paged {
  const unsigned char* q;
  unsigned char *k, *v;    // pages
  const int32_t *table, *lengths;
  const float* slopes;     // may be null
  unsigned char* out;
  float* lse;              // may be null
  Strides sk, sv;          // batch: from page to page
  int seqs, heads, kv_heads, group, d, dtype, page_size, num_pages, max_pages;
  float scale, cap;
  void* workspace;
};

size_t paged_workspace_bytes(const Paged& p);
hipError_t launch_paged_attention(const Paged& p, hipStream_t stream);
hipError_t launch_paged_append(const Paged& p, const void* k, const void* v, int tokens, const int32_t* offsets, hipStream_t stream);

}  // namespace pisa

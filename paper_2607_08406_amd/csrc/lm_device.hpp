// What the operators over requests read of a request.
#pragma once

#include <hip/hip_runtime.h>
#include <stdint.h>

#include "mca_lm.h"

namespace mca {

// Cached tokens of request r that count.
__device__ __forceinline__ int cached_of(const mca_tree_attention_args& a, int r) {
  const int most = (int)min((int64_t)a.max_len, (int64_t)a.max_blocks * a.block_size);
  return max(0, min(a.lengths[r], most));
}
// Request r's rows; false if there are none or they are out of range.
__device__ __forceinline__ bool rows_of(const mca_tree_attention_args& a, int r, int* first, int* n) {
  const int64_t f = a.offsets[r], e = a.offsets[r + 1];
  *first = (int)f;
  *n = (int)(e - f);
  return f >= 0 && e > f && e <= a.n_rows && e - f <= a.max_nodes;
}

}  // namespace mca

// Host-side launchers of the language-model operators (mca_lm.h): the paged
// cache's tables and rows (lm_cache.hip), the attention of drafted tokens
// (lm_attention.hip) and token log probabilities (lm_logprobs.hip).  Arguments
// have been validated (lm_api.hip).
#pragma once

#include <hip/hip_runtime.h>
#include <stdint.h>

#include "mca_lm.h"

namespace mca {

struct TablesArgs {
  const int32_t *old_len, *new_len;
  int32_t n_req, block_size;
  int32_t* table;
  int64_t table_stride;
  int32_t max_blocks, n_blocks;
  int32_t *free_list, *offsets;
  int64_t* slots;
  int64_t max_tokens;
  int32_t* status;
};
hipError_t lm_launch_tables(const TablesArgs& a, hipStream_t s);

hipError_t lm_launch_append(const mca_cache_append_args& a, hipStream_t s);

// How the attention call is split: chunks of `chunk` cached tokens, at most
// `splits` of them for a request, or evenly over `sharers` workgroups where that
// is not 0; partial results take `bytes` of workspace.
struct AttnPlan {
  int32_t chunk, splits, sharers;
  size_t bytes;
};
AttnPlan lm_attention_plan(const mca_tree_attention_args& a);
hipError_t lm_launch_attention(const mca_tree_attention_args& a, const AttnPlan& p, hipStream_t s);

// How a row of logits is split over workgroups.
struct LogprobsPlan {
  int32_t splits;
  size_t bytes;
};
LogprobsPlan lm_logprobs_plan(const mca_token_logprobs_args& a);
hipError_t lm_launch_logprobs(const mca_token_logprobs_args& a, const LogprobsPlan& p, hipStream_t s);
hipError_t lm_launch_logprobs_grad(const mca_token_logprobs_grad_args& a, hipStream_t s);

// Failure without a context: the message for mca_last_error(NULL) (mca_api.hip).
int lm_fail(int code, const char* msg);
int lm_device_fail(hipError_t e, const char* what);
// The checks of mca_tree_attention's sizes that need no pointers (lm_api.hip);
// null if they hold, else the message, with the status in *code.
const char* lm_check_attention(const mca_tree_attention_args& a, int* code);

}  // namespace mca

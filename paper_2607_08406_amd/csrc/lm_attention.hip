// mca_tree_attention: the attention of drafted tokens over a cache in the queries' type.
#include "lm_attention.hpp"

namespace mca {

AttnPlan lm_attention_plan(const mca_tree_attention_args& a) { return attention_plan<false>(a); }

hipError_t lm_launch_attention(const mca_tree_attention_args& a, const AttnPlan& plan, hipStream_t s) {
  return launch_attention<false>(a, plan, nullptr, nullptr, s);
}

}  // namespace mca

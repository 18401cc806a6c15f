// mca_tree_attention8: the attention of drafted tokens over a cache of 8-bit values.
#include "lm_attention.hpp"

namespace mca {

AttnPlan lm_attention8_plan(const mca_tree_attention8_args& a) { return attention_plan<true>(a.of); }

hipError_t lm_launch_attention8(const mca_tree_attention8_args& a, const AttnPlan& plan, hipStream_t s) {
  return launch_attention<true>(a.of, plan, a.k_scale, a.v_scale, s);
}

}  // namespace mca

// mca_tree_attention: the attention of drafted tokens over a cache in the queries' type.
#include "lm_attention.hpp"

namespace mca {

AttnPlan lm_attention_plan(const mca_tree_attention_args& a) {
  AttnPlan p{};
  if (a.n_req == 0) return p;
  const int64_t wgs = (int64_t)row_tiles(a) * a.n_kv_head * a.n_req;
  if (is_wide(a)) {
    // Shared, if that saves more than the joining costs.  A workgroup for each tile of
    // rows takes as many rounds of `tiles` as the chip needs for them all; shared, a
    // part of a round counts as such.  An fp32 tile counts twice, as its products do.
    // The joining costs about the time of 12 tiles and of the parts, two a workgroup.
    // (128 rows, 4 key heads, bf16, head_dim 128, shared and not: one request of 512
    // tokens 33 and 28 us, of 1024 33 and 41; 16 of 1024 52 and 43, of 2048 58 and 71;
    // 64 of 4096 147 and 133, of 16384 380 and 464.)
    const bool one = wide_waves(a) == 8 || (a.dtype == MCA_TYPE_F32 && a.head_dim > 128);  // LDS or registers of a CU
    const int tokens = tile_tokens(a), resident = kCUs * (one ? 1 : 2);
    const int64_t tiles = (a.max_len + tokens - 1) / tokens;
    p.chunk = a.max_len;
    p.splits = 1;
    const int64_t idle = (wgs + resident - 1) / resident * resident - wgs;
    const bool saves = (a.dtype == MCA_TYPE_F32 ? 2 : 1) * tiles * idle / resident > 12 + std::min<int64_t>(wgs, resident) / 8;
    if (saves && wgs * (tiles + MCA_MAX_NODES / 32) < (1 << 30)) {
      p.sharers = (int32_t)std::min<int64_t>(resident, (wgs * (tiles + MCA_MAX_NODES / 32) / kLeastUnits + 8) / 8 * 8);
      p.bytes = ((size_t)a.n_req + 1 + 63) / 64 * 256 + (size_t)2 * p.sharers * tile_rows(a) * (a.head_dim + 1) * sizeof(float);
    }
    return p;
  }
  // Chunks of at least two tiles a wave while there are fewer than two workgroups a
  // CU; behind that of 1536 tokens, up to 16 workgroups a CU, which evens out requests
  // of different lengths.  (Workgroups in all of 512, 1024, 2048 and 4096, bf16,
  // head_dim 128, 8 key heads: one request of 200000 162, 170, 185 and 185 us; 32 of
  // 8192 to 32768 526, 500, 478 and 470.)
  const int64_t step = kAttnWaves * kTilePos;
  const int64_t first = std::min<int64_t>((512 + wgs - 1) / wgs, (a.max_len + 2 * step - 1) / (2 * step));
  const int64_t more = std::min<int64_t>((4096 + wgs - 1) / wgs, (a.max_len + 1535) / 1536);
  const int64_t want = std::clamp<int64_t>(std::max(first, more), 1, 256);
  const int64_t chunk = (a.max_len + want - 1) / want;
  p.chunk = (int32_t)std::max<int64_t>(step, (chunk + step - 1) / step * step);
  p.splits = (int32_t)std::max<int64_t>(1, ((int64_t)a.max_len + p.chunk - 1) / p.chunk);
  p.bytes = p.splits > 1 ? (size_t)a.n_rows * a.n_head * p.splits * (a.head_dim + 1) * sizeof(float) : 0;
  return p;
}

hipError_t lm_launch_attention(const mca_tree_attention_args& a, const AttnPlan& plan, hipStream_t s) {
  return launch_attention<false>(a, plan, nullptr, nullptr, s);
}

}  // namespace mca

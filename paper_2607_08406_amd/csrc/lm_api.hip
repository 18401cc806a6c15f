// C entry points of the language-model operators (mca_lm.h): validation, then
// the launchers.  mca_extend, which needs a context, is in mca_api.hip.
#include <cmath>

#include "lm_kernels.hpp"

namespace {

constexpr int64_t kMaxInt = 0x7ffffffe;    // counts that a kernel holds in 32 bits
constexpr int64_t kMaxGrid = (1 << 24) - 1;  // workgroups of 256 threads in a grid

int invalid(const char* msg) { return mca::lm_fail(MCA_EINVAL, msg); }
int unsupported(const char* msg) { return mca::lm_fail(MCA_EUNSUPPORTED, msg); }
bool known_type(int32_t t) { return t == MCA_TYPE_F32 || t == MCA_TYPE_BF16 || t == MCA_TYPE_F16; }
int64_t type_bytes(int32_t t) { return t == MCA_TYPE_F32 ? 4 : 2; }
bool aligned(const void* p, uintptr_t n) { return ((uintptr_t)p & (n - 1)) == 0; }
bool strides_ok(std::initializer_list<int64_t> s, int64_t most) {
  for (int64_t x : s)
    if (x < 0 || x > most) return false;
  return true;
}
constexpr int64_t kMaxStride = (int64_t)1 << 40;

const char* check_logprobs(const mca_token_logprobs_args& a, int* code) {
  *code = MCA_EINVAL;
  if (!known_type(a.dtype)) return "unknown dtype";
  if (a.n_rows < 0) return "n_rows must not be negative";
  if (a.n_vocab < 1) return "n_vocab must be positive";
  if (a.n_top < 0 || a.n_top > MCA_MAX_TOP) return "n_top out of range [0, 32]";
  if (a.n_top > a.n_vocab) return "n_top must be at most n_vocab";
  *code = MCA_EUNSUPPORTED;
  if (a.n_rows > kMaxGrid) return "at most 2^24 - 1 rows";
  if (a.n_vocab > ((int64_t)1 << 30)) return "n_vocab must be at most 2^30";
  *code = MCA_OK;
  return nullptr;
}

}  // namespace

namespace mca {

const char* lm_check_attention(const mca_tree_attention_args& a, int* code) {
  *code = MCA_EINVAL;
  if (!known_type(a.dtype)) return "unknown dtype";
  if (a.n_req < 0 || a.n_req > MCA_MAX_REQ) return "n_req out of range [0, 65535]";
  if (a.n_rows < 0 || a.n_rows > kMaxInt) return "n_rows out of range";
  if (a.n_kv_head < 1 || a.n_head < 1 || a.n_head % a.n_kv_head != 0) return "n_head must be a positive multiple of n_kv_head";
  if (a.head_dim < 1) return "head_dim must be positive";
  if (a.block_size < 1 || a.n_blocks < 1 || a.max_blocks < 0) return "block_size and n_blocks must be positive, max_blocks not negative";
  if (a.max_nodes < 1 || a.max_nodes > MCA_MAX_NODES) return "max_nodes out of range [1, 128]";
  if (a.max_len < 0) return "max_len must not be negative";
  *code = MCA_EUNSUPPORTED;
  if (a.head_dim > 256) return "head_dim must be at most 256";
  if (a.head_dim * type_bytes(a.dtype) % 16 != 0) return "head_dim must be a multiple of 16 bytes";
  if ((int64_t)a.max_blocks * a.block_size > kMaxInt) return "max_blocks * block_size must stay below 2^31 - 1";
  if (a.max_len > (1 << 30)) return "max_len must be at most 2^30";  // positions behind the last fit 32 bits
  if ((int64_t)a.n_blocks * a.n_kv_head > kMaxInt || (int64_t)a.n_blocks * a.n_kv_head * a.block_size > kMaxInt)
    return "n_blocks * n_kv_head * block_size must stay below 2^31 - 1";
  // workgroups: at least 16 rows each, and a few thousand more when split
  const int64_t tiles = ((int64_t)a.max_nodes * (a.n_head / a.n_kv_head) + 15) / 16;
  if (tiles > kMaxGrid / 16 || tiles * a.n_kv_head > kMaxGrid / 2 || tiles * a.n_kv_head * a.n_req > kMaxGrid / 2 ||
      (int64_t)a.n_head * a.max_nodes > kMaxGrid)
    return "too many requests times heads for one call";
  *code = MCA_OK;
  return nullptr;
}

}  // namespace mca

extern "C" {

int mca_block_tables(const int32_t* old_len, const int32_t* new_len, int32_t n_req, int32_t block_size, int32_t* table,
                     int64_t table_stride, int32_t max_blocks, int32_t* free_list, int32_t n_blocks, int32_t* offsets,
                     int64_t* slots, int64_t max_tokens, int32_t* status, void* hip_stream) {
  if (n_req < 1 || n_req > MCA_MAX_REQ) return invalid("n_req out of range [1, 65535]");
  if (block_size < 1 || max_blocks < 1 || n_blocks < 1) return invalid("block_size, max_blocks and n_blocks must be positive");
  if ((int64_t)max_blocks * block_size > kMaxInt || n_blocks > kMaxInt) return unsupported("max_blocks * block_size and n_blocks must stay below 2^31 - 1");
  if (table_stride < max_blocks || table_stride > kMaxStride) return invalid("table_stride must be at least max_blocks");
  if (max_tokens < 0 || max_tokens > kMaxInt) return invalid("max_tokens out of range");
  if (!old_len || !new_len || !table || !free_list || !offsets || (!slots && max_tokens > 0) || !status)
    return invalid("an array is NULL");
  if (!aligned(old_len, 4) || !aligned(new_len, 4) || !aligned(table, 4) || !aligned(free_list, 4) || !aligned(offsets, 4) ||
      !aligned(slots, 8) || !aligned(status, 4))
    return invalid("an array is not aligned to its elements");
  mca::TablesArgs a{old_len,    new_len,  n_req,     block_size, table, table_stride, max_blocks,
                    n_blocks, free_list, offsets,    slots, max_tokens,   status};
  const hipError_t e = mca::lm_launch_tables(a, (hipStream_t)hip_stream);
  return e == hipSuccess ? MCA_OK : mca::lm_device_fail(e, "mca_block_tables");
}

int mca_cache_append(const mca_cache_append_args* args, void* hip_stream) {
  if (args == nullptr) return invalid("args is NULL");
  const mca_cache_append_args& a = *args;
  if (!known_type(a.dtype)) return invalid("unknown dtype");
  if (a.n < 0 || a.n_src < 0) return invalid("n and n_src must not be negative");
  if (a.n_kv_head < 1 || a.head_dim < 1 || a.block_size < 1 || a.n_blocks < 1)
    return invalid("n_kv_head, head_dim, block_size and n_blocks must be positive");
  const int64_t el = type_bytes(a.dtype);
  if ((int64_t)a.n_kv_head * a.head_dim > (1 << 24)) return unsupported("a row has at most 2^24 values");
  if (a.n > kMaxGrid || a.n_src > kMaxInt) return unsupported("at most 2^24 - 1 rows");
  if (!strides_ok({a.k_row, a.k_head, a.v_row, a.v_head}, kMaxStride)) return invalid("strides must not be negative");
  if (a.n == 0 || a.n_src == 0) return MCA_OK;  // every source row is outside an empty source
  if (!a.k || !a.v || !a.k_cache || !a.v_cache || !a.slots) return invalid("an array is NULL");
  if (!aligned(a.k, el) || !aligned(a.v, el) || !aligned(a.k_cache, el) || !aligned(a.v_cache, el) || !aligned(a.slots, 8) ||
      !aligned(a.rows, 4))
    return invalid("an array is not aligned to its elements");
  const hipError_t e = mca::lm_launch_append(a, (hipStream_t)hip_stream);
  return e == hipSuccess ? MCA_OK : mca::lm_device_fail(e, "mca_cache_append");
}

int mca_tree_attention_plan(const mca_tree_attention_args* args, size_t* workspace_bytes) {
  if (args == nullptr || workspace_bytes == nullptr) return invalid("args or workspace_bytes is NULL");
  int code;
  const char* msg = mca::lm_check_attention(*args, &code);
  if (msg != nullptr) return mca::lm_fail(code, msg);
  *workspace_bytes = mca::lm_attention_plan(*args).bytes;
  return MCA_OK;
}

int mca_tree_attention(const mca_tree_attention_args* args, void* hip_stream) {
  if (args == nullptr) return invalid("args is NULL");
  const mca_tree_attention_args& a = *args;
  int code;
  const char* msg = mca::lm_check_attention(a, &code);
  if (msg != nullptr) return mca::lm_fail(code, msg);
  if (!std::isfinite(a.scale)) return invalid("scale must be finite");
  const int64_t el = type_bytes(a.dtype);
  if (!strides_ok({a.q_row, a.q_head, a.k_row, a.k_head, a.v_row, a.v_head, a.out_row, a.out_head, a.table_stride}, kMaxStride) ||
      a.table_stride < a.max_blocks)
    return invalid("strides must not be negative, table_stride at least max_blocks");
  if (a.k_row * el > 0x7fffffff || a.v_row * el > 0x7fffffff) return unsupported("rows of k and v must be less than 2^31 bytes apart");
  if (a.n_req == 0 || a.n_rows == 0) return MCA_OK;
  if (!a.q || !a.k || !a.v || !a.out || !a.k_cache || !a.v_cache || !a.lengths || !a.offsets || !a.parents ||
      (!a.table && a.max_blocks > 0))
    return invalid("an array is NULL");
  if (!aligned(a.q, 16) || !aligned(a.k, 16) || !aligned(a.v, 16) || !aligned(a.out, 16) || !aligned(a.k_cache, 16) ||
      !aligned(a.v_cache, 16))
    return invalid("q, k, v, out and the caches must be 16-byte aligned");
  for (int64_t s : {a.q_row, a.q_head, a.k_row, a.k_head, a.v_row, a.v_head, a.out_row, a.out_head})
    if (s * el % 16 != 0) return invalid("strides must be multiples of 16 bytes");
  if (!aligned(a.table, 4) || !aligned(a.lengths, 4) || !aligned(a.offsets, 4) || !aligned(a.parents, 4) || !aligned(a.lse, 4))
    return invalid("an array is not aligned to its elements");
  const mca::AttnPlan plan = mca::lm_attention_plan(a);
  if (plan.bytes > 0) {
    if (a.workspace == nullptr || !aligned(a.workspace, 256)) return invalid("workspace must be a 256-byte aligned array");
    if (a.workspace_bytes < plan.bytes) return mca::lm_fail(MCA_ENOSPACE, "workspace smaller than mca_tree_attention_plan()");
  }
  const hipError_t e = mca::lm_launch_attention(a, plan, (hipStream_t)hip_stream);
  return e == hipSuccess ? MCA_OK : mca::lm_device_fail(e, "mca_tree_attention");
}

int mca_token_logprobs_plan(const mca_token_logprobs_args* args, size_t* workspace_bytes) {
  if (args == nullptr || workspace_bytes == nullptr) return invalid("args or workspace_bytes is NULL");
  int code;
  const char* msg = check_logprobs(*args, &code);
  if (msg != nullptr) return mca::lm_fail(code, msg);
  *workspace_bytes = mca::lm_logprobs_plan(*args).bytes;
  return MCA_OK;
}

int mca_token_logprobs(const mca_token_logprobs_args* args, void* hip_stream) {
  if (args == nullptr) return invalid("args is NULL");
  const mca_token_logprobs_args& a = *args;
  int code;
  const char* msg = check_logprobs(a, &code);
  if (msg != nullptr) return mca::lm_fail(code, msg);
  if (a.token_bytes != 4 && a.token_bytes != 8) return invalid("token_bytes must be 4 or 8");
  if (a.logits_row < a.n_vocab || a.logits_row > kMaxStride) return invalid("logits_row must be at least n_vocab");
  if (a.n_rows == 0) return MCA_OK;
  if (!a.logits || !a.tokens || !a.logprob || !a.entropy || !a.lse || (a.n_top > 0 && (!a.top_logprob || !a.top_id)))
    return invalid("an array is NULL");
  if (!aligned(a.logits, type_bytes(a.dtype)) || !aligned(a.tokens, a.token_bytes) || !aligned(a.logprob, 4) || !aligned(a.entropy, 4) ||
      !aligned(a.lse, 4) || !aligned(a.top_logprob, 4) || !aligned(a.top_id, 4))
    return invalid("an array is not aligned to its elements");
  const mca::LogprobsPlan plan = mca::lm_logprobs_plan(a);
  if (plan.bytes > 0) {
    if (a.workspace == nullptr || !aligned(a.workspace, 256)) return invalid("workspace must be a 256-byte aligned array");
    if (a.workspace_bytes < plan.bytes) return mca::lm_fail(MCA_ENOSPACE, "workspace smaller than mca_token_logprobs_plan()");
  }
  const hipError_t e = mca::lm_launch_logprobs(a, plan, (hipStream_t)hip_stream);
  return e == hipSuccess ? MCA_OK : mca::lm_device_fail(e, "mca_token_logprobs");
}

int mca_token_logprobs_grad(const mca_token_logprobs_grad_args* args, void* hip_stream) {
  if (args == nullptr) return invalid("args is NULL");
  const mca_token_logprobs_grad_args& a = *args;
  if (!known_type(a.dtype)) return invalid("unknown dtype");
  if (a.n_rows < 0 || a.n_vocab < 1) return invalid("n_rows must not be negative, n_vocab positive");
  if (a.n_rows > kMaxGrid) return unsupported("at most 2^24 - 1 rows");
  if (a.n_vocab > ((int64_t)1 << 30)) return unsupported("n_vocab must be at most 2^30");
  if (a.token_bytes != 4 && a.token_bytes != 8) return invalid("token_bytes must be 4 or 8");
  if (a.logits_row < a.n_vocab || a.grad_row < a.n_vocab || a.logits_row > kMaxStride || a.grad_row > kMaxStride)
    return invalid("logits_row and grad_row must be at least n_vocab");
  if (a.n_rows == 0) return MCA_OK;
  if (!a.logits || !a.tokens || !a.lse || !a.grad || (a.grad_entropy != nullptr && !a.entropy)) return invalid("an array is NULL");
  if (a.logits == a.grad && a.logits_row != a.grad_row) return invalid("a gradient in place of the logits takes their stride");
  const int64_t el = type_bytes(a.dtype);
  if (!aligned(a.logits, el) || !aligned(a.grad, el) || !aligned(a.tokens, a.token_bytes) || !aligned(a.lse, 4) || !aligned(a.entropy, 4) ||
      !aligned(a.grad_logprob, 4) || !aligned(a.grad_entropy, 4))
    return invalid("an array is not aligned to its elements");
  const hipError_t e = mca::lm_launch_logprobs_grad(a, (hipStream_t)hip_stream);
  return e == hipSuccess ? MCA_OK : mca::lm_device_fail(e, "mca_token_logprobs_grad");
}

}  // extern "C"

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

// The checks of mca_tree_attention's arguments behind those of its sizes; *empty if
// there is nothing to do.  The message, with the status in *code.
const char* check_attention_arrays(const mca_tree_attention_args& a, int* code, bool* empty) {
  auto fail = [&](int c, const char* msg) {
    *code = c;
    return msg;
  };
  if (!std::isfinite(a.scale)) return fail(MCA_EINVAL, "scale must be finite");
  const int64_t el = type_bytes(a.dtype);
  if (!strides_ok({a.q_row, a.q_head, a.k_row, a.k_head, a.v_row, a.v_head, a.out_row, a.out_head, a.table_stride}, kMaxStride) ||
      a.table_stride < a.max_blocks)
    return fail(MCA_EINVAL, "strides must not be negative, table_stride at least max_blocks");
  if (a.k_row * el > 0x7fffffff || a.v_row * el > 0x7fffffff) return fail(MCA_EUNSUPPORTED, "rows of k and v must be less than 2^31 bytes apart");
  if (a.n_req == 0 || a.n_rows == 0) {
    *empty = true;
    return nullptr;
  }
  if (!a.q || !a.k || !a.v || !a.out || !a.k_cache || !a.v_cache || !a.lengths || !a.offsets || !a.parents ||
      (!a.table && a.max_blocks > 0))
    return fail(MCA_EINVAL, "an array is NULL");
  if (!aligned(a.q, 16) || !aligned(a.k, 16) || !aligned(a.v, 16) || !aligned(a.out, 16) || !aligned(a.k_cache, 16) ||
      !aligned(a.v_cache, 16))
    return fail(MCA_EINVAL, "q, k, v, out and the caches must be 16-byte aligned");
  for (int64_t s : {a.q_row, a.q_head, a.k_row, a.k_head, a.v_row, a.v_head, a.out_row, a.out_head})
    if (s * el % 16 != 0) return fail(MCA_EINVAL, "strides must be multiples of 16 bytes");
  if (!aligned(a.table, 4) || !aligned(a.lengths, 4) || !aligned(a.offsets, 4) || !aligned(a.parents, 4) || !aligned(a.lse, 4))
    return fail(MCA_EINVAL, "an array is not aligned to its elements");
  return nullptr;
}

const char* check_cache8(int32_t n_req, int32_t n_kv_head, int32_t head_dim, int32_t block_size, int32_t n_blocks, int32_t max_blocks,
                         int64_t n, int* code) {
  *code = MCA_EINVAL;
  if (n_req < 0 || n_req > MCA_MAX_REQ) return "n_req out of range [0, 65535]";
  if (n < 0) return "n must not be negative";
  if (n_kv_head < 1 || head_dim < 1 || block_size < 1 || n_blocks < 1 || max_blocks < 0)
    return "n_kv_head, head_dim, block_size and n_blocks must be positive, max_blocks not negative";
  *code = MCA_EUNSUPPORTED;
  if (head_dim % 16 != 0) return "head_dim of a cache of 8-bit values must be a multiple of 16";
  if ((int64_t)n_kv_head * head_dim > (1 << 24)) return "a row has at most 2^24 values";
  if ((int64_t)block_size * head_dim > (1 << 30)) return "a block has at most 2^30 values of a head";
  if ((int64_t)max_blocks * block_size > kMaxInt) return "max_blocks * block_size must stay below 2^31 - 1";
  if (n > kMaxInt || (n / block_size + 2 * (int64_t)n_req) * n_kv_head > kMaxGrid) return "too many blocks times heads for one call";
  *code = MCA_OK;
  return nullptr;
}

// Temperatures that multiply logits in 32 bits: neither they nor their product with log2 e
// overflow or vanish, which would make NaN of 0 or -inf.
bool scale_ok(double x) { return x >= 0x1p-100 && x <= 0x1p100; }

const char* check_verify(const mca_verify_drafts_args& a, int* code) {
  *code = MCA_EINVAL;
  if (!known_type(a.dtype)) return "unknown dtype";
  if (a.n_req < 0 || a.n_req > MCA_MAX_REQ) return "n_req out of range [0, 65535]";
  if (a.n_rows < 0) return "n_rows must not be negative";
  if (a.max_nodes < 1 || a.max_nodes > MCA_MAX_NODES) return "max_nodes out of range [1, 128]";
  if (a.n_vocab < 1) return "n_vocab must be positive";
  *code = MCA_EUNSUPPORTED;
  if (a.n_rows > kMaxGrid) return "at most 2^24 - 1 rows";
  if (a.n_vocab > ((int64_t)1 << 30)) return "n_vocab must be at most 2^30";
  *code = MCA_OK;
  return nullptr;
}

const char* check_distill(int32_t dtype, int32_t n_top, int32_t rest, float scale, int64_t n_rows, int64_t n_vocab, int* code) {
  *code = MCA_EINVAL;
  if (!known_type(dtype)) return "unknown dtype";
  if (n_rows < 0) return "n_rows must not be negative";
  if (n_vocab < 1) return "n_vocab must be positive";
  if (n_top < 1 || n_top > MCA_MAX_TOP) return "n_top out of range [1, 32]";
  if (!scale_ok(scale)) return "scale must be positive, from 2^-100 to 2^100";
  if (rest != 0 && rest != 1) return "rest must be 0 or 1";
  if (rest == 1 && scale != 1.0f) return "the other symbols as one outcome (rest) take a scale of 1";
  *code = MCA_EUNSUPPORTED;
  if (n_rows > kMaxGrid) return "at most 2^24 - 1 rows";
  if (n_vocab > ((int64_t)1 << 30)) return "n_vocab must be at most 2^30";
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
  bool empty = false;
  const char* msg = mca::lm_check_attention(a, &code);
  if (msg == nullptr) msg = check_attention_arrays(a, &code, &empty);
  if (msg != nullptr) return mca::lm_fail(code, msg);
  if (empty) return MCA_OK;
  const mca::AttnPlan plan = mca::lm_attention_plan(a);
  if (plan.bytes > 0) {
    if (a.workspace == nullptr || !aligned(a.workspace, 256)) return invalid("workspace must be a 256-byte aligned array");
    if (a.workspace_bytes < plan.bytes) return mca::lm_fail(MCA_ENOSPACE, "workspace smaller than mca_tree_attention_plan()");
  }
  const hipError_t e = mca::lm_launch_attention(a, plan, (hipStream_t)hip_stream);
  return e == hipSuccess ? MCA_OK : mca::lm_device_fail(e, "mca_tree_attention");
}

int mca_cache8_append(const mca_cache8_append_args* args, void* hip_stream) {
  if (args == nullptr) return invalid("args is NULL");
  const mca_cache8_append_args& a = *args;
  if (!known_type(a.dtype)) return invalid("unknown dtype");
  int code;
  const char* msg = check_cache8(a.n_req, a.n_kv_head, a.head_dim, a.block_size, a.n_blocks, a.max_blocks, a.n, &code);
  if (msg != nullptr) return mca::lm_fail(code, msg);
  if (a.n_src < 0) return invalid("n_src must not be negative");
  const int64_t el = type_bytes(a.dtype);
  if (!strides_ok({a.k_row, a.k_head, a.v_row, a.v_head, a.table_stride}, kMaxStride) || a.table_stride < a.max_blocks)
    return invalid("strides must not be negative, table_stride at least max_blocks");
  if (a.n_req == 0 || a.n == 0 || a.max_blocks == 0) return MCA_OK;
  if ((a.n_src > 0 && (!a.k || !a.v)) || !a.k_cache || !a.v_cache || !a.k_scale || !a.v_scale || !a.table || !a.lengths || !a.offsets)
    return invalid("an array is NULL");
  if (!aligned(a.k, 16) || !aligned(a.v, 16) || !aligned(a.k_cache, 16) || !aligned(a.v_cache, 16))
    return invalid("k, v and the caches must be 16-byte aligned");
  for (int64_t x : {a.k_row, a.k_head, a.v_row, a.v_head})
    if (x * el % 16 != 0) return invalid("strides must be multiples of 16 bytes");
  if (!aligned(a.table, 4) || !aligned(a.lengths, 4) || !aligned(a.offsets, 4) || !aligned(a.rows, 4))
    return invalid("an array is not aligned to its elements");
  const hipError_t e = mca::lm_launch_append8(a, (hipStream_t)hip_stream);
  return e == hipSuccess ? MCA_OK : mca::lm_device_fail(e, "mca_cache8_append");
}

int mca_cache8_read(const mca_cache8_read_args* args, void* hip_stream) {
  if (args == nullptr) return invalid("args is NULL");
  const mca_cache8_read_args& a = *args;
  if (!known_type(a.dtype)) return invalid("unknown dtype");
  int code;
  const char* msg = check_cache8(a.n_req, a.n_kv_head, a.head_dim, a.block_size, a.n_blocks, a.max_blocks, a.n, &code);
  if (msg != nullptr) return mca::lm_fail(code, msg);
  const int64_t el = type_bytes(a.dtype);
  if (!strides_ok({a.k_row, a.k_head, a.v_row, a.v_head, a.table_stride}, kMaxStride) || a.table_stride < a.max_blocks)
    return invalid("strides must not be negative, table_stride at least max_blocks");
  if (a.n_req == 0 || a.n == 0) return MCA_OK;
  if (!a.k || !a.v || !a.k_cache || !a.v_cache || !a.k_scale || !a.v_scale || (!a.table && a.max_blocks > 0) || !a.start || !a.offsets)
    return invalid("an array is NULL");
  if (!aligned(a.k, 16) || !aligned(a.v, 16) || !aligned(a.k_cache, 16) || !aligned(a.v_cache, 16))
    return invalid("k, v and the caches must be 16-byte aligned");
  for (int64_t x : {a.k_row, a.k_head, a.v_row, a.v_head})
    if (x * el % 16 != 0) return invalid("strides must be multiples of 16 bytes");
  if (!aligned(a.table, 4) || !aligned(a.start, 4) || !aligned(a.offsets, 4)) return invalid("an array is not aligned to its elements");
  const hipError_t e = mca::lm_launch_read8(a, (hipStream_t)hip_stream);
  return e == hipSuccess ? MCA_OK : mca::lm_device_fail(e, "mca_cache8_read");
}

int mca_tree_attention8_plan(const mca_tree_attention8_args* args, size_t* workspace_bytes) {
  if (args == nullptr || workspace_bytes == nullptr) return invalid("args or workspace_bytes is NULL");
  int code;
  const char* msg = mca::lm_check_attention(args->of, &code);
  if (msg != nullptr) return mca::lm_fail(code, msg);
  if (args->of.head_dim % 16 != 0) return unsupported("head_dim of a cache of 8-bit values must be a multiple of 16");
  *workspace_bytes = mca::lm_attention8_plan(*args).bytes;
  return MCA_OK;
}

int mca_tree_attention8(const mca_tree_attention8_args* args, void* hip_stream) {
  if (args == nullptr) return invalid("args is NULL");
  const mca_tree_attention_args& a = args->of;
  int code;
  bool empty = false;
  const char* msg = mca::lm_check_attention(a, &code);
  if (msg == nullptr && a.head_dim % 16 != 0) {
    code = MCA_EUNSUPPORTED;
    msg = "head_dim of a cache of 8-bit values must be a multiple of 16";
  }
  if (msg == nullptr) msg = check_attention_arrays(a, &code, &empty);
  if (msg != nullptr) return mca::lm_fail(code, msg);
  if (empty) return MCA_OK;
  if (!args->k_scale || !args->v_scale) return invalid("an array is NULL");
  const mca::AttnPlan plan = mca::lm_attention8_plan(*args);
  if (plan.bytes > 0) {
    if (a.workspace == nullptr || !aligned(a.workspace, 256)) return invalid("workspace must be a 256-byte aligned array");
    if (a.workspace_bytes < plan.bytes) return mca::lm_fail(MCA_ENOSPACE, "workspace smaller than mca_tree_attention8_plan()");
  }
  const hipError_t e = mca::lm_launch_attention8(*args, plan, (hipStream_t)hip_stream);
  return e == hipSuccess ? MCA_OK : mca::lm_device_fail(e, "mca_tree_attention8");
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

int mca_verify_drafts_plan(const mca_verify_drafts_args* args, size_t* workspace_bytes) {
  if (args == nullptr || workspace_bytes == nullptr) return invalid("args or workspace_bytes is NULL");
  int code;
  const char* msg = check_verify(*args, &code);
  if (msg != nullptr) return mca::lm_fail(code, msg);
  *workspace_bytes = mca::lm_verify_plan(*args);
  return MCA_OK;
}

int mca_verify_drafts(const mca_verify_drafts_args* args, void* hip_stream) {
  if (args == nullptr) return invalid("args is NULL");
  const mca_verify_drafts_args& a = *args;
  int code;
  const char* msg = check_verify(a, &code);
  if (msg != nullptr) return mca::lm_fail(code, msg);
  if (a.greedy != 0 && a.greedy != 1) return invalid("greedy must be 0 or 1");
  const bool draft = a.draft != nullptr && !a.greedy;
  if (!a.greedy && !scale_ok(a.scale)) return invalid("scale must be positive, from 2^-100 to 2^100");
  if (draft && !scale_ok(a.draft_scale)) return invalid("draft_scale must be positive, from 2^-100 to 2^100");
  if (a.target_row < a.n_vocab || a.target_row > kMaxStride) return invalid("target_row must be at least n_vocab");
  if (draft && (a.draft_row < a.n_vocab || a.draft_row > kMaxStride)) return invalid("draft_row must be at least n_vocab");
  if (a.n_req == 0 && a.n_rows == 0) return MCA_OK;
  if (a.n_rows > 0 && (!a.target || !a.tokens || !a.parents || (!a.greedy && !a.accept) || !a.rows)) return invalid("an array is NULL");
  if (!a.offsets || (a.n_req > 0 && (!a.lengths || (!a.greedy && !a.sample) || !a.new_len || !a.token))) return invalid("an array is NULL");
  const int64_t el = type_bytes(a.dtype);
  if (!aligned(a.target, el) || (draft && !aligned(a.draft, el)) || !aligned(a.tokens, 4) || !aligned(a.parents, 4) || !aligned(a.offsets, 4) ||
      !aligned(a.lengths, 4) || !aligned(a.accept, 4) || !aligned(a.sample, 4) || !aligned(a.new_len, 4) || !aligned(a.rows, 4) ||
      !aligned(a.token, 4))
    return invalid("an array is not aligned to its elements");
  const size_t bytes = mca::lm_verify_plan(a);
  if (bytes > 0) {
    if (a.workspace == nullptr || !aligned(a.workspace, 256)) return invalid("workspace must be a 256-byte aligned array");
    if (a.workspace_bytes < bytes) return mca::lm_fail(MCA_ENOSPACE, "workspace smaller than mca_verify_drafts_plan()");
  }
  const hipError_t e = mca::lm_launch_verify(a, (hipStream_t)hip_stream);
  return e == hipSuccess ? MCA_OK : mca::lm_device_fail(e, "mca_verify_drafts");
}

int mca_distill_plan(const mca_distill_args* args, size_t* workspace_bytes) {
  if (args == nullptr || workspace_bytes == nullptr) return invalid("args or workspace_bytes is NULL");
  int code;
  const char* msg = check_distill(args->dtype, args->n_top, args->rest, args->scale, args->n_rows, args->n_vocab, &code);
  if (msg != nullptr) return mca::lm_fail(code, msg);
  *workspace_bytes = mca::lm_distill_plan(*args).bytes;
  return MCA_OK;
}

int mca_distill(const mca_distill_args* args, void* hip_stream) {
  if (args == nullptr) return invalid("args is NULL");
  const mca_distill_args& a = *args;
  int code;
  const char* msg = check_distill(a.dtype, a.n_top, a.rest, a.scale, a.n_rows, a.n_vocab, &code);
  if (msg != nullptr) return mca::lm_fail(code, msg);
  if (a.logits_row < a.n_vocab || a.logits_row > kMaxStride) return invalid("logits_row must be at least n_vocab");
  if (a.n_rows == 0) return MCA_OK;
  if (!a.logits || !a.logprob || !a.ids || !a.loss || !a.lse || (a.rest && !a.lse_rest)) return invalid("an array is NULL");
  if (!aligned(a.logits, type_bytes(a.dtype)) || !aligned(a.logprob, 4) || !aligned(a.ids, 4) || !aligned(a.loss, 4) || !aligned(a.lse, 4) ||
      !aligned(a.lse_rest, 4))
    return invalid("an array is not aligned to its elements");
  const mca::LogprobsPlan plan = mca::lm_distill_plan(a);
  if (plan.bytes > 0) {
    if (a.workspace == nullptr || !aligned(a.workspace, 256)) return invalid("workspace must be a 256-byte aligned array");
    if (a.workspace_bytes < plan.bytes) return mca::lm_fail(MCA_ENOSPACE, "workspace smaller than mca_distill_plan()");
  }
  const hipError_t e = mca::lm_launch_distill(a, plan, (hipStream_t)hip_stream);
  return e == hipSuccess ? MCA_OK : mca::lm_device_fail(e, "mca_distill");
}

int mca_distill_grad(const mca_distill_grad_args* args, void* hip_stream) {
  if (args == nullptr) return invalid("args is NULL");
  const mca_distill_grad_args& a = *args;
  int code;
  const char* msg = check_distill(a.dtype, a.n_top, a.rest, a.scale, a.n_rows, a.n_vocab, &code);
  if (msg != nullptr) return mca::lm_fail(code, msg);
  if (a.logits_row < a.n_vocab || a.grad_row < a.n_vocab || a.logits_row > kMaxStride || a.grad_row > kMaxStride)
    return invalid("logits_row and grad_row must be at least n_vocab");
  if (a.n_rows == 0) return MCA_OK;
  if (!a.logits || !a.logprob || !a.ids || !a.lse || !a.grad_loss || !a.grad || (a.rest && !a.lse_rest)) return invalid("an array is NULL");
  if (a.logits == a.grad && a.logits_row != a.grad_row) return invalid("a gradient in place of the logits takes their stride");
  const int64_t el = type_bytes(a.dtype);
  if (!aligned(a.logits, el) || !aligned(a.grad, el) || !aligned(a.logprob, 4) || !aligned(a.ids, 4) || !aligned(a.lse, 4) ||
      !aligned(a.lse_rest, 4) || !aligned(a.grad_loss, 4))
    return invalid("an array is not aligned to its elements");
  const hipError_t e = mca::lm_launch_distill_grad(a, (hipStream_t)hip_stream);
  return e == hipSuccess ? MCA_OK : mca::lm_device_fail(e, "mca_distill_grad");
}

}  // extern "C"

/*
 * mca_lm.h -- C ABI of libmca's operators that answer with a trained language
 * model: a paged cache of keys and values, the attention of drafted tokens over
 * it, and the log probabilities read off the logits; and mca_extend, which runs
 * a Transformer context's committed net on drafted tokens with them.
 *
 * Conventions of the operators (mca.h's hold for mca_extend):
 *   - Every array is device memory that the caller owns.  Nothing is kept
 *     between calls, no memory is allocated, nothing is synchronised: a call
 *     enqueues kernels on hip_stream (hipStream_t as void*; NULL = the null
 *     stream) and returns.  The calling thread's current device must be the
 *     stream's.  Calls may be captured into a graph.
 *   - A workspace (256-byte aligned, at least the bytes of the plan call) is
 *     scratch: its contents need no preparation and mean nothing afterwards.
 *     Calls that may run at the same time need a workspace each.
 *   - Arguments are validated before anything is enqueued: MCA_EINVAL,
 *     MCA_EUNSUPPORTED or MCA_ENOSPACE with the message in
 *     mca_last_error(NULL); MCA_EDEVICE if a launch fails.  What only the
 *     device can see (lengths, offsets, block numbers, parents, tokens) is
 *     checked there and never leads to an access outside the arrays; each call
 *     says what such a value does.
 *   - Inputs and outputs must not overlap, nor an output's rows each other,
 *     except where a call says so.
 *   - Strides are in elements.  Vectors over the head dimension and over the
 *     vocabulary are contiguous.
 */
#ifndef MCA_LM_H_
#define MCA_LM_H_

#include "mca.h"

#ifdef __cplusplus
extern "C" {
#endif

/* element types */
#define MCA_TYPE_F32 0
#define MCA_TYPE_BF16 1
#define MCA_TYPE_F16 2

#define MCA_MAX_NODES 128  /* drafted tokens of a request in one call */
#define MCA_MAX_TOP 32     /* alternatives of a row */
#define MCA_MAX_REQ 65535  /* requests of a call */

/* ------------------------------------------------------------------------
 * The cache.  Keys and values lie in blocks of block_size tokens,
 * [n_blocks][n_kv_head][block_size][head_dim]; slot s = block * block_size + i
 * is one token's place.  Request r's token t lies in slot
 * table[r][t / block_size] * block_size + t % block_size.  Requests share no
 * blocks.  free_list [n_blocks] is a stack: of n_free = n_blocks minus the
 * blocks that the requests hold, its first n_free entries are the free ones.
 * ------------------------------------------------------------------------ */

/* mca_block_tables status[0] */
#define MCA_TABLES_OK 0
#define MCA_TABLES_EXHAUSTED 1 /* fewer free blocks than the requests need */
#define MCA_TABLES_LENGTH 2    /* a length outside [0, max_blocks * block_size], or more blocks held than n_blocks */
#define MCA_TABLES_SLOTS 3     /* more new tokens than max_tokens */

/* Block tables and slot map for requests that go from old_len[r] to new_len[r]
 * tokens (r < n_req <= MCA_MAX_REQ; 0 to a length: it enters; to 0: it ends).
 * The blocks that shrinking requests give up are pushed onto the free list in
 * the order of requests, then pages; the blocks that growing ones need are then
 * popped in that order, and written into table (rows of table_stride >=
 * max_blocks entries; entries of given-up blocks stay as they were).
 * offsets [n_req + 1]: where each request's new tokens start among all of
 * them; slots [max_tokens]: their slots, -1 behind the last.  status [4]:
 * MCA_TABLES_*, free blocks afterwards, new tokens, blocks taken.  If status[0]
 * is not MCA_TABLES_OK, tables and free list stay as they were, offsets are 0
 * and slots -1.  The order is fixed: equal inputs give equal tables; and the
 * call with the same lengths again gives the same results once more. */
int mca_block_tables(const int32_t* old_len, const int32_t* new_len, int32_t n_req,
                     int32_t block_size, int32_t* table, int64_t table_stride, int32_t max_blocks,
                     int32_t* free_list, int32_t n_blocks, int32_t* offsets, int64_t* slots,
                     int64_t max_tokens, int32_t* status, void* hip_stream);

/* Rows of keys and values into their slots: row i < n takes k[row][h][:] and
 * v[row][h][:], row = rows[i] (i if rows is NULL), to slots[i].  A row whose
 * slot is outside [0, n_blocks * block_size), or whose source row is outside
 * [0, n_src), is skipped.  Slots must differ from each other.  Any head_dim;
 * widest where head_dim, strides and addresses are multiples of 16 bytes. */
typedef struct mca_cache_append_args {
  int32_t dtype, n_kv_head, head_dim, block_size, n_blocks, reserved;
  int64_t n, n_src;
  const void* k;
  const void* v;
  int64_t k_row, k_head, v_row, v_head; /* strides */
  void* k_cache;
  void* v_cache;
  const int64_t* slots;
  const int32_t* rows;
} mca_cache_append_args;
int mca_cache_append(const mca_cache_append_args* args, void* hip_stream);

/* Attention of drafted tokens over the cache.  Rows offsets[r] ..
 * offsets[r + 1] - 1 of q, k, v are request r's nodes 0, 1, ... (at most
 * max_nodes <= MCA_MAX_NODES; offsets must not fall and end within n_rows).
 * Node i follows node parents[row] of the same request, which must be before
 * it, or (-1, and any other value) the request's cached tokens directly.  It
 * sees the request's lengths[r] cached tokens, its ancestors and itself:
 *   out = softmax(scale * q K^T) V,  lse = log sum exp(scale * q K^T)
 * over those, head h with key head h / (n_head / n_kv_head).  One node is a
 * decoding step; a chain (parents i - 1) is a piece of a prompt.  A value that
 * a node does not see never reaches its result, not if it is infinite or NaN; a
 * row of which every score is -inf is NaN, its lse too.
 * Rows behind the last request, and requests of more than max_nodes or of
 * offsets out of range, are left as they were.  lengths outside [0, max_len]
 * count as the nearest of these; cached tokens behind max_blocks or in a block
 * outside [0, n_blocks) are not there.  lse may be NULL.
 * head_dim at most 256, and head_dim, strides and addresses multiples of 16
 * bytes; max_len at most 2^30, n_blocks * n_kv_head * block_size below 2^31.  Scores, softmax and
 * sums in 32 bits; the weights of 16-bit values are rounded to 16 bits, each by at most half a step
 * of its own or, of fp16, 2^-17 of the largest weight among the 64 tokens around it. */
typedef struct mca_tree_attention_args {
  int32_t dtype, n_req, n_head, n_kv_head, head_dim, block_size, n_blocks, max_blocks, max_nodes,
      max_len;
  float scale;
  int32_t reserved;
  int64_t n_rows, table_stride;
  const void* q;
  const void* k;
  const void* v;
  int64_t q_row, q_head, k_row, k_head, v_row, v_head, out_row, out_head; /* strides */
  const void* k_cache;
  const void* v_cache;
  const int32_t* table;   /* [n_req] rows of max_blocks */
  const int32_t* lengths; /* [n_req] */
  const int32_t* offsets; /* [n_req + 1] */
  const int32_t* parents; /* [n_rows] */
  void* out;
  float* lse; /* [n_rows][n_head] or NULL */
  void* workspace;
  size_t workspace_bytes;
} mca_tree_attention_args;
/* Bytes of workspace for these sizes (pointers and strides are not read). */
int mca_tree_attention_plan(const mca_tree_attention_args* args, size_t* workspace_bytes);
int mca_tree_attention(const mca_tree_attention_args* args, void* hip_stream);

/* Log probabilities.  Row t < n_rows of logits z (n_vocab values, rows
 * logits_row apart), token tokens[t]:
 *   lse = log sum_v exp z_v,  logprob = z_token - lse,
 *   entropy = lse - sum_v p_v z_v,  p_v = exp(z_v - lse),
 * and the n_top <= MCA_MAX_TOP (<= n_vocab) largest log probabilities with
 * their symbols, in falling order, equal ones by rising symbol.  Infinite
 * logits of -inf have probability 0 and no part in the entropy.  A token
 * outside [0, n_vocab) is none: logprob 0.  A row of nothing but -inf gives
 * lse = -inf, entropy 0, and -inf for logprob and alternatives; a NaN or +inf
 * makes the row's floating results NaN and its alternatives unspecified (symbols
 * of the vocabulary).  tokens are int32, or int64 with token_bytes 8. */
typedef struct mca_token_logprobs_args {
  int32_t dtype, n_top, token_bytes, reserved;
  int64_t n_rows, n_vocab, logits_row;
  const void* logits;
  const void* tokens;
  float* logprob;     /* [n_rows] */
  float* entropy;     /* [n_rows] */
  float* lse;         /* [n_rows] */
  float* top_logprob; /* [n_rows][n_top], unused if n_top is 0 */
  int32_t* top_id;    /* [n_rows][n_top], unused if n_top is 0 */
  void* workspace;
  size_t workspace_bytes;
} mca_token_logprobs_args;
/* Bytes of workspace for these sizes (may be 0; pointers are not read). */
int mca_token_logprobs_plan(const mca_token_logprobs_args* args, size_t* workspace_bytes);
int mca_token_logprobs(const mca_token_logprobs_args* args, void* hip_stream);

/* Gradient of sum_t grad_logprob[t] logprob[t] + grad_entropy[t] entropy[t]
 * with respect to the logits, lse and entropy as mca_token_logprobs gave them:
 *   grad_v = grad_logprob (1[v = token] - p_v) - grad_entropy p_v (log p_v + entropy).
 * Either gradient may be NULL (0).  A row without a token has no first part,
 * a row of lse -inf gradient 0.  grad has the logits' type, rows grad_row
 * apart, and may be the logits themselves (same address and stride). */
typedef struct mca_token_logprobs_grad_args {
  int32_t dtype, token_bytes;
  int64_t n_rows, n_vocab, logits_row, grad_row;
  const void* logits;
  const void* tokens;
  const float* lse;
  const float* entropy;
  const float* grad_logprob;
  const float* grad_entropy;
  void* grad;
} mca_token_logprobs_grad_args;
int mca_token_logprobs_grad(const mca_token_logprobs_grad_args* args, void* hip_stream);

/* ------------------------------------------------------------------------
 * mca_extend: the committed net of a Transformer context on the nodes of the
 * requests' drafts (rows, offsets, parents, lengths, table as for
 * mca_tree_attention; max_nodes nodes and max_len cached tokens at most).
 * tokens [n_rows]; node i stands at position lengths[r] + its depth.  Block
 * b's cache is k_cache + b * cache_layer (fp32, [n_blocks][n_head][block_size]
 * [32]); the call reads it and does not write it: qkv [n_block][n_rows][3]
 * [n_head][32] receives every node's query, key and value of every block, from
 * which mca_cache_append keeps the rows that are accepted.  logits [n_rows]
 * (rows logits_row apart) receives the nodes' logits; rows behind the last
 * request stay as they were there and are unspecified in qkv.  A node whose
 * token is outside the vocabulary or whose position is outside the context
 * gets NaN, and so do the nodes that see it, no others.  n_rows times the
 * widest of 3 d_model, d_mlp and vocabulary below 2^31.  On the context's
 * stream; not synchronised.  MLP contexts: MCA_EINVAL.
 * ------------------------------------------------------------------------ */
typedef struct mca_extend_args {
  int32_t n_req, n_rows, max_nodes, max_len, block_size, n_blocks, max_blocks, reserved;
  int64_t table_stride, cache_layer, logits_row;
  const int32_t* tokens;
  const int32_t* parents;
  const int32_t* offsets;
  const int32_t* lengths;
  const int32_t* table;
  const float* k_cache;
  const float* v_cache;
  float* qkv;
  float* logits;
  void* workspace;
  size_t workspace_bytes;
} mca_extend_args;
int mca_extend_plan(mca_ctx* ctx, const mca_extend_args* args, size_t* workspace_bytes);
int mca_extend(mca_ctx* ctx, const mca_extend_args* args);

#ifdef __cplusplus
}
#endif

#endif /* MCA_LM_H_ */

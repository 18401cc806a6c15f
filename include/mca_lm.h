/*
 * mca_lm.h -- C ABI of libmca's operators that answer with a trained language
 * model: a paged cache of keys and values, in their own type or in 8 bits, the
 * attention of drafted tokens over it, which of them are accepted, the log
 * probabilities read off the logits and the loss against a teacher's; and
 * mca_extend, which runs a Transformer context's committed net on drafted tokens
 * with them.
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

/* ------------------------------------------------------------------------
 * A cache of 8-bit values.  Caches as above, of codes: floats of 4 exponent and 3
 * mantissa bits without infinities (e4m3: up to 448, steps of 2^-9 below 2^-6, NaN
 * 0x7f and 0xff).  k_scale and v_scale [n_blocks][n_kv_head] have a byte for each
 * block and key head: a code's value is its e4m3 value times 2^(byte - 127) (bytes
 * 0 and 255 count as 1 and 254).  head_dim is a multiple of 16.
 * ------------------------------------------------------------------------ */

/* Rows of keys and values quantised into the cache, for requests that go from
 * lengths[r] to lengths[r] + offsets[r + 1] - offsets[r] tokens: row i of them
 * (offsets[r] <= i < offsets[r + 1] <= n) takes k[row][h][:] and v[row][h][:],
 * row = rows[i] (i if rows is NULL), to position lengths[r] + i - offsets[r].
 * (lengths and offsets are mca_block_tables' old_len and offsets.)
 * A block's scale is the smallest power of two under which its new values are at
 * most 448, not below 2^-100 (fp16: 2^-15) and, if tokens of the request already
 * lie in the block, not below the one it has; where it grows, their codes are
 * rounded to the new one, which changes only those that become less than 2^-6.
 * Values are rounded to nearest, ties to even; those whose code would stand for
 * more than the source type holds (from 248 times 2^120, of fp16 2^8) get the largest
 * code that does not: 240 at that scale, and at the larger ones that blocks with tokens kept may have less.
 * Infinities and NaN become the code 0x7f and do not count for the scale.  A row
 * outside [0, n_src) counts as zeros.  Blocks outside [0, n_blocks), positions
 * behind max_blocks, and requests of negative lengths or of offsets out of range are
 * left as they were, and places behind a request's last token are.  Requests share no
 * blocks, and offsets do not fall.  The call with the same arguments again gives the same results once more. */
typedef struct mca_cache8_append_args {
  int32_t dtype, n_req, n_kv_head, head_dim, block_size, n_blocks, max_blocks, reserved;
  int64_t n, n_src, table_stride;
  const void* k;
  const void* v;
  int64_t k_row, k_head, v_row, v_head; /* strides; 16-byte aligned, as k and v */
  uint8_t* k_cache;
  uint8_t* v_cache; /* 16-byte aligned */
  uint8_t* k_scale;
  uint8_t* v_scale;
  const int32_t* table;   /* [n_req] rows of max_blocks */
  const int32_t* lengths; /* [n_req] */
  const int32_t* offsets; /* [n_req + 1] */
  const int32_t* rows;    /* [n] or NULL */
} mca_cache8_append_args;
int mca_cache8_append(const mca_cache8_append_args* args, void* hip_stream);

/* The values of requests' tokens: rows offsets[r] .. offsets[r + 1] - 1 < n of k
 * and v [n][n_kv_head][head_dim] receive request r's tokens start[r], start[r] + 1,
 * ..., exactly, unless they pass the type's range.  Tokens behind max_blocks or in a
 * block outside [0, n_blocks) are 0; rows of no request, and of requests whose start
 * is negative or whose offsets are out of range, stay as they were. */
typedef struct mca_cache8_read_args {
  int32_t dtype, n_req, n_kv_head, head_dim, block_size, n_blocks, max_blocks, reserved;
  int64_t n, table_stride;
  void* k;
  void* v;
  int64_t k_row, k_head, v_row, v_head; /* strides; 16-byte aligned, as k and v */
  const uint8_t* k_cache;
  const uint8_t* v_cache; /* 16-byte aligned */
  const uint8_t* k_scale;
  const uint8_t* v_scale;
  const int32_t* table;
  const int32_t* start;   /* [n_req] */
  const int32_t* offsets; /* [n_req + 1] */
} mca_cache8_read_args;
int mca_cache8_read(const mca_cache8_read_args* args, void* hip_stream);

/* mca_tree_attention over a cache of codes: its arguments with the caches' codes in
 * place of their values, and the scales.  q, k, v, out and the drafted tokens' part are
 * of dtype.  Keys and values are those that mca_cache8_read gives (of fp16 infinite
 * where they pass its range). */
typedef struct mca_tree_attention8_args {
  mca_tree_attention_args of;
  const uint8_t* k_scale;
  const uint8_t* v_scale;
} mca_tree_attention8_args;
int mca_tree_attention8_plan(const mca_tree_attention8_args* args, size_t* workspace_bytes);
int mca_tree_attention8(const mca_tree_attention8_args* args, void* hip_stream);

/* Verification of drafted tokens.  Request r has nodes offsets[r] .. offsets[r + 1]
 * - 1 (at most max_nodes <= MCA_MAX_NODES) as for mca_tree_attention; its node 0 is
 * the token before the draft, which is certain, and node i > 0 follows node
 * parents[row] < i (nodes without one are not reached).  Row t of target has the
 * logits of what follows node t, row t of draft the logits that the children of node t
 * were drawn from, independently of each other.  With p = softmax(scale target),
 * q = softmax(draft_scale draft), the children of the node reached last are tried in
 * their order, with c = 0 and S = 1 at first: child t of token x is accepted if
 *   accept[t] S q_x < p_x - c q_x;
 * otherwise c grows by S and S becomes sum_v max(p_v - c q_v, 0).  If none is accepted
 * the path ends, and the token that follows is drawn from w_v = max(p_v - c q_v, 0)
 * (from p if that is 0 everywhere): the first v with sum_{u <= v} w_u > sample[r]
 * sum w.  So path and token are distributed as if drawn from the target one by one.
 * Without draft (NULL) drafted tokens were given, not drawn: q is 1 at a child's token
 * and 0 elsewhere, w is p without the tokens rejected, S its sum.  greedy: a child is
 * accepted if its token has the node's largest target logit, the first of equal ones,
 * and that one's symbol follows; draft, accept, sample and the scales are not read.
 * accept [n_rows] and sample [n_req] lie in [0, 1) (sample outside it counts as
 * the nearest, NaN as 0).
 * new_len [n_req] is lengths[r] and the nodes accepted, node 0 among them; rows
 * [n_rows] the accepted nodes' rows, request after request, -1 behind the last
 * (mca_block_tables' new_len, mca_cache_append's and mca_cache8_append's rows); token
 * [n_req] the tokens that follow.  A child whose token is outside [0, n_vocab) is
 * not accepted and changes nothing.  At a node whose target row (or draft row, if it
 * has children) has no softmax (NaN, +inf, nothing but -inf),
 * the path ends and token is -1; so it is for requests without nodes, of more than
 * max_nodes or of offsets out of range, whose new_len is lengths[r].
 * Sums are held in 64 bits, of exponentials of 64 where a token is drawn (there c is a sum of
 * such ones, too), and where a child is tried of 32: each off by (1 + |exponent|) 2^-22 at
 * most, and up to 8 neighbours added before they go into a sum. */
typedef struct mca_verify_drafts_args {
  int32_t dtype, n_req, max_nodes, greedy;
  int64_t n_rows, n_vocab, target_row, draft_row;
  double scale, draft_scale; /* 2^-100 to 2^100 */
  const void* target;
  const void* draft;      /* or NULL */
  const int32_t* tokens;  /* [n_rows] */
  const int32_t* parents; /* [n_rows] */
  const int32_t* offsets; /* [n_req + 1] */
  const int32_t* lengths; /* [n_req] */
  const float* accept;    /* [n_rows] */
  const float* sample;    /* [n_req] */
  int32_t* new_len;       /* [n_req] */
  int32_t* rows;          /* [n_rows] */
  int32_t* token;         /* [n_req] */
  void* workspace;
  size_t workspace_bytes;
} mca_verify_drafts_args;
/* Bytes of workspace for these sizes (of the pointers only whether draft is NULL counts). */
int mca_verify_drafts_plan(const mca_verify_drafts_args* args, size_t* workspace_bytes);
int mca_verify_drafts(const mca_verify_drafts_args* args, void* hip_stream);

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

/* Distillation.  A row's teacher is n_top <= MCA_MAX_TOP symbols ids[t][j] with their log
 * probabilities (as mca_token_logprobs gives them); symbols outside [0, n_vocab) are
 * none, and a row of nothing else has loss and gradient 0.  With s = softmax(scale z)
 * of the student's logits z:
 *   rest 0: q = softmax over j of scale * logprob_j,
 *           loss = sum_j q_j (log q_j - log s_{id_j});
 *   rest 1: q_j = exp(logprob_j), and all other symbols are one more outcome, of
 *           probability q_r = max(0, 1 - sum_j q_j) under the teacher and s_r under the
 *           student: q_r (log q_r - log s_r) is added.  scale must be 1.
 * An outcome of teacher's probability 0 adds 0; one that only the student's is 0 for
 * makes the loss +inf.  lse = log sum_v exp(scale z_v), lse_rest the same over the
 * symbols that are none of the teacher's (rest 1).  NaN or +inf among the logits or a
 * valid entry's logprob makes the row's loss NaN.  A symbol may stand in several
 * entries, whose q add up (each with a term of its own). */
typedef struct mca_distill_args {
  int32_t dtype, n_top, rest;
  float scale; /* 2^-100 to 2^100 */
  int64_t n_rows, n_vocab, logits_row;
  const void* logits;
  const float* logprob; /* [n_rows][n_top] */
  const int32_t* ids;   /* [n_rows][n_top] */
  float* loss;          /* [n_rows] */
  float* lse;           /* [n_rows] */
  float* lse_rest;      /* [n_rows], unused if rest is 0 */
  void* workspace;
  size_t workspace_bytes;
} mca_distill_args;
/* Bytes of workspace for these sizes (may be 0; pointers are not read). */
int mca_distill_plan(const mca_distill_args* args, size_t* workspace_bytes);
int mca_distill(const mca_distill_args* args, void* hip_stream);

/* Gradient of sum_t grad_loss[t] loss[t] with respect to the logits, lse and lse_rest
 * as mca_distill gave them:
 *   grad_v = grad_loss scale (Q s_v - sum_{j: id_j = v} q_j),  Q = sum_j q_j + q_r,
 * and of symbols that are none of the teacher's with rest 1
 *   grad_v = grad_loss s_v (Q - q_r / s_r).
 * A row whose loss is NaN has a gradient of NaN, another one of lse -inf a gradient of 0.
 * (grad_loss 0 gives 0 for every finite loss.)  s_v is exp(scale z_v - lse) and off by
 * |lse| 2^-24 of itself, as lse is rounded to 32 bits.  grad has the logits' type, rows
 * grad_row apart, and may be the logits themselves (same address and stride). */
typedef struct mca_distill_grad_args {
  int32_t dtype, n_top, rest;
  float scale;
  int64_t n_rows, n_vocab, logits_row, grad_row;
  const void* logits;
  const float* logprob;
  const int32_t* ids;
  const float* lse;
  const float* lse_rest;
  const float* grad_loss; /* [n_rows] */
  void* grad;
} mca_distill_grad_args;
int mca_distill_grad(const mca_distill_grad_args* args, void* hip_stream);

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

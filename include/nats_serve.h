/* nats_serve.h -- generation from drafted tokens, and a cache with a budget, beside the decode steps of nats.h.
 *
 * Conventions as in nats.h: device pointers owned by the caller, dense row-major tensors, 16-byte aligned data pointers, one
 * HIP stream, no allocation, no synchronisation, arguments checked on the host before anything is launched, no floating-point
 * atomics, calls that overlap in time need different workspaces.  What a call writes, its workspace included, shares no memory with
 * anything else that it is given (NATS_ERR_SHAPE).  Routing per token.  nats_abi_version() counts nats.h; what is
 * declared here is found by name.
 *
 * A round of generation from drafts:
 *   nats_hybrid_attn_decode_tree   reads a tree of drafted tokens against the state and the cache; changes neither
 *   (the caller accepts a path of the tree)
 *   nats_hybrid_attn_tree_commit   writes the accepted path into the state, its softmax tokens into the cache (padded trees: .._ex)
 *   nats_cache_weights             adds the attention weight that the path's queries gave to every row of the cache
 *   nats_cache_evict_clear         cuts the cache down to a budget by those weights
 * The weights of rows that are not there have to be 0, for nats_cache_weights adds to what it finds and neither the commit nor the
 * decode steps touch them: an array of zeros at first, and nats_cache_evict_clear keeps it so.
 */
#ifndef NATS_SERVE_H_
#define NATS_SERVE_H_

#include "nats.h"

#ifdef __cplusplus
extern "C" {
#endif

#define NATS_TREE_MAX_NODES 64

typedef struct nats_tree_params {
    int32_t B, H;          /* sequences, linear heads                                                */
    int32_t T;             /* drafted tokens (nodes) per sequence, 1 .. NATS_TREE_MAX_NODES           */
    int32_t d;             /* 64 or 128                                                               */
    int32_t cap;           /* rows per (b, head) in the KV cache, at most 2^20 (in all the calls here)  */
    int32_t dtype;         /* nats_dtype of q, k, v, o and of the KV cache                            */
    float softmax_scale;   /* as in nats_dec_params                                                   */
    float la_scale;
    int32_t combine_mode;
    float rms_eps;
    int32_t linear_op;
    int32_t freeze_on_softmax;
    int32_t group;         /* head grouping as in nats_fwd_params: G = group (0 counts as 1, at most 8) output heads per linear
                              head.  q, k, alpha, beta, mask are [B,H,...]; state, caches, cache_len, v, q_nla, k_nla, w_nla,
                              w_la, o, lse, vis, err_flags are [B,H*G,...]                             */
    const void* q_nla;     /* [B,H*G,T,d] dtype or NULL: the softmax branch's own queries and keys;    */
    const void* k_nla;     /* both or neither (the commit reads k_nla alone)                           */
} nats_tree_params;

/* A tree of drafted tokens over the state and the cache.  parent [B,T] i32: the node that node i follows, one of 0 .. i - 1, or
 * -1: it follows the last committed token (any other number counts as -1).  With A(i) = node i and its ancestors, every node sees
 * what the decode step of nats.h would show it after the tokens of A(i) had been decoded one after the other:
 *   S_i = alpha_i S_parent(i), linear token: S_i += beta_i (v_i - S_i k_i) k_i^T    (S of the last committed token: state)
 *   o_i = merge(la_scale * S_i q_i, softmax attention over the cache's rows [0, cache_len) and the softmax tokens of A(i))
 * whatever room the cache has for those tokens.  What stands in nodes outside A(i) has no influence on o_i, not even an infinity or a NaN.
 *   state   : in  [B,H*G,d,d] f32           k_cache, v_cache : in  [B,H*G,cap,d]      cache_len : in  [B,H*G] i32
 *   q, k    : in  [B,H,T,d];  v : in [B,H*G,T,d];  alpha, beta : in [B,H,T] f32;  mask : in [B,H,T] u8, non-zero = softmax token
 *   n_nodes : in  [B] i32 or NULL (T): nodes i >= n_nodes[b] are not there: o_i = 0, lse_i = -inf
 *   w_nla, w_la : in [B,H*G,T] f32 or NULL, as in the decode step
 *   o       : out [B,H*G,T,d] dtype
 *   lse     : out [B,H*G,T] f32 or NULL: log-sum-exp of the logits that node i sees; -inf where it sees none
 *   workspace : nats_hybrid_attn_decode_tree_workspace_bytes(p) bytes or more, contents undefined afterwards */
size_t nats_hybrid_attn_decode_tree_workspace_bytes(const nats_tree_params* p);
nats_status nats_hybrid_attn_decode_tree(const nats_tree_params* p, const float* state, const void* k_cache, const void* v_cache,
                                         const int32_t* cache_len, const void* q, const void* k, const void* v, const float* alpha,
                                         const float* beta, const uint8_t* mask, const int32_t* parent, const int32_t* n_nodes,
                                         const float* w_nla, const float* w_la, void* o, float* lse, void* workspace,
                                         size_t workspace_bytes, void* hip_stream);

/* The path from the last committed token to node[b] (-1: nothing is accepted; [B] i32) is decoded for good: the state becomes
 * S_node, and the path's softmax tokens (rows of k_nla where that is given, of k otherwise, and of v) go behind the cache's rows.
 *   state, k_cache, v_cache, cache_len : in/out;  k, v, alpha, beta, mask, parent : as in the call that read the tree
 *   vis       : out [B,H*G,T] i32 or NULL: for a node of the path the rows of the cache, as it is now, that the node saw: those that
 *               were there and the path's softmax tokens up to the node itself; 0 for the other nodes
 *   err_flags : out [B,H*G] i32 or NULL: 1 where a softmax token found the cache full (it is not stored, and no later one is),
 *               2 where node[b] is no node, that is none of -1 .. T - 1 (nothing is done then), else 0
 * p->softmax_scale, la_scale, combine_mode, rms_eps and q_nla are not read. */
nats_status nats_hybrid_attn_tree_commit(const nats_tree_params* p, float* state, void* k_cache, void* v_cache, int32_t* cache_len,
                                         const void* k, const void* v, const float* alpha, const float* beta, const uint8_t* mask,
                                         const int32_t* parent, const int32_t* node, int32_t* vis, int32_t* err_flags,
                                         void* hip_stream);
/* The same for padded trees: nodes i >= n_nodes[b] are not there (as in the call that read the tree; [B] i32 or NULL: T), and a node[b]
 * that is not there is no node: flag 2, nothing is done. */
nats_status nats_hybrid_attn_tree_commit_ex(const nats_tree_params* p, float* state, void* k_cache, void* v_cache, int32_t* cache_len,
                                            const void* k, const void* v, const float* alpha, const float* beta, const uint8_t* mask,
                                            const int32_t* parent, const int32_t* n_nodes, const int32_t* node, int32_t* vis,
                                            int32_t* err_flags, void* hip_stream);

typedef struct nats_cache_weights_params {
    int32_t B, H;          /* sequences, heads of the cache (all output heads)                         */
    int32_t T;             /* queries per (b, head), at most 2^20                                      */
    int32_t d, cap, dtype; /* as above                                                                */
    int32_t q_group;       /* q is [B,H/q_group,T,d]: a query head serves q_group heads in a row (0 counts as 1) */
    int32_t vis_group;     /* vis is [B,H/vis_group,T]                                                */
    float softmax_scale;   /* as in nats_fwd_params                                                   */
    float decay;           /* what the weights so far are multiplied with                             */
} nats_cache_weights_params;

/* weights[c] <- decay * weights[c] + sum over the queries t that see row c (c < vis_t) of exp(scale * q_t . k_cache[c] - lse_t), for the
 * rows c < cache_len; the others are left as they are (0 for a row that is to be appended, see above).
 *   weights : in/out [B,H,cap] f32;  q : in, dtype;  k_cache : in [B,H,cap,d];  cache_len : in [B,H] i32
 *   vis     : in i32 or NULL (every query sees every row): rows of the cache that query t sees, counted from row 0 (the forward's cnt,
 *             the commit's vis); more than cache_len counts as cache_len
 *   lse     : in [B,H,T] f32 or NULL: the log-sum-exp that the weights are relative to (the forward's or the tree's lse, which
 *             may cover keys that are not in the cache); NULL: of the rows that the query sees.  A query with lse -inf adds nothing
 *   workspace : nats_cache_weights_workspace_bytes(p, lse != NULL) bytes or more (may be 0) */
size_t nats_cache_weights_workspace_bytes(const nats_cache_weights_params* p, int32_t lse_given);
nats_status nats_cache_weights(const nats_cache_weights_params* p, float* weights, const void* q, const void* k_cache,
                               const int32_t* cache_len, const int32_t* vis, const float* lse, void* workspace,
                               size_t workspace_bytes, void* hip_stream);

typedef struct nats_cache_evict_params {
    int32_t B, H, d, cap, dtype;   /* as above */
    int32_t keep;                  /* rows that a cache is cut down to, 1 .. cap */
    int32_t recent;                /* of these, the last ones of the cache, whatever their weight: 0 .. keep */
} nats_cache_evict_params;

/* Every cache of more than `keep` rows keeps its last `recent` rows and, of the others, the keep - recent rows of the largest weight
 * (of equal weights the lower row; a NaN counts as the lowest weight, -0 as 0), in their order: k_cache, v_cache and weights are
 * compacted in place, rows behind the first `keep` are left as they are, cache_len becomes `keep`.  Shorter caches stay as they are.
 * (Routing per chunk: between a commit and the next token, when no rows are provisional.)
 *   kept : out [B,H,keep] i32: the row that row r was before; -1 for rows that are not there
 * nats_cache_evict leaves the weights behind the first `keep` rows as they are, too: rows that are appended there later start with
 * them, unless the caller clears them (a caller that keeps the weights of the rows before, or that starts them anew, has no need to). */
nats_status nats_cache_evict(const nats_cache_evict_params* p, void* k_cache, void* v_cache, int32_t* cache_len, float* weights,
                             int32_t* kept, void* hip_stream);
/* The same, and the weights of the rows that a cache gives up, `keep` .. cache_len - 1, become 0: what is appended starts with nothing. */
nats_status nats_cache_evict_clear(const nats_cache_evict_params* p, void* k_cache, void* v_cache, int32_t* cache_len, float* weights,
                                   int32_t* kept, void* hip_stream);

#ifdef __cplusplus
}
#endif
#endif /* NATS_SERVE_H_ */

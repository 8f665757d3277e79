// Resolved calls of the operators of nats_serve.h, handed to the kernels (internal header).
#pragma once
#include <hip/hip_runtime.h>
#include <stdint.h>

#include "nats_serve.h"

namespace nats {

struct TreeCall {
    int B, H, G, T, d, cap, dtype;
    float scale, la_scale, eps;
    int combine_mode, linear_op, freeze;
    const float* state;
    const void *k_cache, *v_cache;
    const int32_t* cache_len;
    const void *q, *k, *v, *q_nla, *k_nla;
    const float *alpha, *beta;
    const uint8_t* mask;
    const int32_t *parent, *n_nodes;
    const float *w_nla, *w_la;
    void* o;
    float* lse;
    float* ws;
    // parts of the caches: `rows` rows each, n_split of a cache, or (even != 0) `even` blocks with the same number of rows each
    int rows, n_split, even;
    size_t off_anc, off_ola, off_part, off_ml, off_units;  // floats
    // Even parts go by units of TREE_UNIT rows: units()[h] of them lie before cache h (all of them: h = heads), units()[heads + 1] make a
    // block's share.  The part of cache h that block x has is part h + x of all.
    __host__ __device__ int32_t* units() const { return reinterpret_cast<int32_t*>(ws + off_units); }
    // [B][T] ancestor sets, from the linear branch's blocks to the merge
    __host__ __device__ uint64_t* anc() const { return reinterpret_cast<uint64_t*>(ws + off_anc); }
};
constexpr int TREE_UNIT = 32;
size_t tree_workspace(TreeCall& c);    // floats; fills rows, n_split, even and the offsets
nats_status launch_tree(const TreeCall& c, hipStream_t st);
void tree_cache_parts(TreeCall& c);
nats_status launch_tree_read(const TreeCall& c, hipStream_t st);   // both branches

struct TreeCommitCall {
    int B, H, G, T, d, cap, dtype;
    int linear_op, freeze;
    float* state;
    void *k_cache, *v_cache;
    int32_t* cache_len;
    const void *k, *v, *k_nla;
    const float *alpha, *beta;
    const uint8_t* mask;
    const int32_t *parent, *n_nodes, *node;
    int32_t *vis, *err_flags;
};
nats_status launch_tree_commit(const TreeCommitCall& c, hipStream_t st);

struct WeightsCall {
    int B, H, T, d, cap, dtype, q_group, vis_group;
    float scale, decay;
    float* weights;
    const void *q, *k_cache;
    const int32_t *cache_len, *vis;
    const float* lse;
    float* ws;
    int rows, parts;                                   // rows of a part, parts of a cache
    int row_waves, chunk, splits;                      // more than 64 queries: wavefronts of a block that take rows side by side, its
                                                       // queries, blocks that share a head's queries
    int t_lo, t_hi;                                    // the queries of a launch
    int pitch;                                         // of the logits that are kept
    size_t off_ml, off_logits, off_lse, off_sums;      // floats
};
size_t weights_workspace(WeightsCall& c, bool lse_given);   // floats; fills what follows ws
nats_status launch_cache_weights(const WeightsCall& c, hipStream_t st);

struct EvictCall {
    int B, H, d, cap, dtype, keep, recent;
    void *k_cache, *v_cache;
    int32_t* cache_len;
    float* weights;
    int32_t* kept;
    int clear;             // the weights behind the rows that stay become 0
};
nats_status launch_cache_evict(const EvictCall& c, hipStream_t st);

}  // namespace nats

// C ABI of nats_serve.h: host-side validation and the calls into the kernels.
#include <math.h>

#include <initializer_list>

#include "nats_common.h"
#include "serve.h"

namespace nats {

static bool aligned16(const void* p) { return (reinterpret_cast<uintptr_t>(p) & 15u) == 0; }

static nats_status check_pointers(std::initializer_list<const void*> needed, const char* names, std::initializer_list<const void*> optional) {
    for (const void* p : needed) {
        if (p == nullptr) { set_error("%s must all be non-NULL", names); return NATS_ERR_NULL; }
        if (!aligned16(p)) { set_error("pointer %p is not 16-byte aligned", p); return NATS_ERR_ALIGN; }
    }
    for (const void* p : optional)
        if (!aligned16(p)) { set_error("pointer %p is not 16-byte aligned", p); return NATS_ERR_ALIGN; }
    return NATS_OK;
}

// What a call writes, the first `written` arrays, must not share memory with anything else of the call.  (Arrays that are not given: NULL.)
struct Span {
    const char* name;
    const void* p;
    size_t n;   // bytes
};
static nats_status check_apart(std::initializer_list<Span> spans, int written) {
    for (const Span* a = spans.begin(); a != spans.begin() + written; ++a)
        for (const Span* b = a + 1; b != spans.end(); ++b) {
            const uintptr_t pa = (uintptr_t)a->p, pb = (uintptr_t)b->p;
            if (a->p != nullptr && b->p != nullptr && (pa < pb ? pb - pa < a->n : pa - pb < b->n)) {
                set_error("%s must not share memory with %s", a->name, b->name);
                return NATS_ERR_SHAPE;
            }
        }
    return NATS_OK;
}
static size_t element(int dtype) { return dtype == NATS_F32 ? 4 : 2; }

// sizes that all the operators share; the cache has H group heads
static nats_status check_cache(int dtype, int B, int H, int d, int cap, int group) {
    if (dtype != NATS_F32 && dtype != NATS_BF16) {
        set_error("dtype %d is neither NATS_F32 nor NATS_BF16", dtype);
        return NATS_ERR_DTYPE;
    }
    if (B <= 0 || H <= 0 || cap <= 0) {
        set_error("B, H, cap must be positive (got %d, %d, %d)", B, H, cap);
        return NATS_ERR_SHAPE;
    }
    if (d != 64 && d != 128) { set_error("d must be 64 or 128 (got %d)", d); return NATS_ERR_SHAPE; }
    if (B > 65535 || H > 65535 || (long long)B * H * group > 65535) {
        set_error("the number of (batch, head) pairs must not exceed 65535 (got B %d, H %d, group %d)", B, H, group);
        return NATS_ERR_SHAPE;
    }
    if (cap > 1 << 20) { set_error("cap must not exceed 2^20 (got %d)", cap); return NATS_ERR_SHAPE; }
    return NATS_OK;
}

static nats_status check_tree_params(const nats_tree_params* p) {
    if (p == nullptr) { set_error("params is NULL"); return NATS_ERR_NULL; }
    if (p->group < 0 || p->group > 8) { set_error("group must be between 1 and 8 (0 counts as 1; got %d)", p->group); return NATS_ERR_SHAPE; }
    const nats_status st = check_cache(p->dtype, p->B, p->H, p->d, p->cap, p->group ? p->group : 1);
    if (st != NATS_OK) return st;
    if (p->T < 1 || p->T > NATS_TREE_MAX_NODES) {
        set_error("T must be between 1 and %d (got %d)", NATS_TREE_MAX_NODES, p->T);
        return NATS_ERR_SHAPE;
    }
    if (p->combine_mode < 0 || p->combine_mode > 2) {
        set_error("combine_mode must be 0, 1 or 2 (got %d)", p->combine_mode);
        return NATS_ERR_SHAPE;
    }
    if ((p->linear_op != NATS_LINEAR_GDN && p->linear_op != NATS_LINEAR_GATED) ||
        (p->freeze_on_softmax != 0 && p->freeze_on_softmax != 1)) {
        set_error("linear_op must be a nats_linear_op and freeze_on_softmax 0 or 1 (got %d, %d)", p->linear_op,
                  p->freeze_on_softmax);
        return NATS_ERR_SHAPE;
    }
    return NATS_OK;
}

static void set_tree_sizes(const nats_tree_params& p, TreeCall& c) {
    c.B = p.B; c.H = p.H; c.G = p.group ? p.group : 1; c.T = p.T; c.d = p.d; c.cap = p.cap; c.dtype = p.dtype;
}

static nats_status check_weights_params(const nats_cache_weights_params* p) {
    if (p == nullptr) { set_error("params is NULL"); return NATS_ERR_NULL; }
    const nats_status st = check_cache(p->dtype, p->B, p->H, p->d, p->cap, 1);
    if (st != NATS_OK) return st;
    if (p->T <= 0 || p->T > 1 << 20 || (long long)p->B * p->H * p->T > (1ll << 31) - 1) {
        set_error("T must be between 1 and 2^20 and B*H*T fit in 31 bits (T %d)", p->T);
        return NATS_ERR_SHAPE;
    }
    if (p->q_group < 0 || p->vis_group < 0 || (p->q_group && p->H % p->q_group) || (p->vis_group && p->H % p->vis_group)) {
        set_error("q_group and vis_group must divide H (H %d, got %d, %d)", p->H, p->q_group, p->vis_group);
        return NATS_ERR_SHAPE;
    }
    return NATS_OK;
}

static void set_weights_sizes(const nats_cache_weights_params& p, WeightsCall& c) {
    c.B = p.B; c.H = p.H; c.T = p.T; c.d = p.d; c.cap = p.cap; c.dtype = p.dtype;
    c.q_group = p.q_group ? p.q_group : 1;
    c.vis_group = p.vis_group ? p.vis_group : 1;
    c.scale = p.softmax_scale > 0.f ? p.softmax_scale : 1.0f / sqrtf((float)p.d);
    c.decay = p.decay;
}

}  // namespace nats

using namespace nats;

extern "C" {

size_t nats_hybrid_attn_decode_tree_workspace_bytes(const nats_tree_params* p) {
    if (check_tree_params(p) != NATS_OK) return 0;
    TreeCall c{};
    set_tree_sizes(*p, c);
    return tree_workspace(c) * 4;
}

nats_status nats_hybrid_attn_decode_tree(const nats_tree_params* p, const float* state, const void* k_cache, const void* v_cache,
                                         const int32_t* cache_len, const void* q, const void* k, const void* v, const float* alpha,
                                         const float* beta, const uint8_t* mask, const int32_t* parent, const int32_t* n_nodes,
                                         const float* w_nla, const float* w_la, void* o, float* lse, void* workspace,
                                         size_t workspace_bytes, void* hip_stream) {
    nats_status st = check_tree_params(p);
    if (st != NATS_OK) return st;
    if ((p->q_nla == nullptr) != (p->k_nla == nullptr)) { set_error("q_nla and k_nla must be given together"); return NATS_ERR_NULL; }
    if (!cache_len || !alpha || !beta || !mask || !parent) {
        set_error("cache_len, alpha, beta, mask and parent must all be non-NULL");
        return NATS_ERR_NULL;
    }
    st = check_pointers({state, k_cache, v_cache, q, k, v, o}, "state, k_cache, v_cache, q, k, v and o", {p->q_nla, p->k_nla});
    if (st != NATS_OK) return st;
    for (const void* in : {(const void*)state, k_cache, v_cache, q, k, v, p->q_nla, p->k_nla})
        if (o == in || (lse != nullptr && (const void*)lse == in)) { set_error("o and lse must not alias an input"); return NATS_ERR_SHAPE; }
    if (o == (const void*)lse) { set_error("o and lse must be two arrays"); return NATS_ERR_SHAPE; }
    TreeCall c{};
    set_tree_sizes(*p, c);
    const size_t need = tree_workspace(c) * 4;
    if (workspace == nullptr || workspace_bytes < need) {
        set_error("workspace of %zu bytes given, %zu needed", workspace ? workspace_bytes : (size_t)0, need);
        return NATS_ERR_WORKSPACE;
    }
    if (!aligned16(workspace)) { set_error("the workspace is not 16-byte aligned"); return NATS_ERR_ALIGN; }
    const size_t es = element(c.dtype), nodes = (size_t)c.B * c.H * c.T, heads = (size_t)c.B * c.H * c.G, outs = nodes * c.G;
    const size_t cache = heads * c.cap * c.d * es;
    st = check_apart({{"o", o, outs * c.d * es}, {"lse", lse, 4 * outs}, {"the workspace", workspace, need},
                      {"state", state, 4 * heads * c.d * c.d}, {"k_cache", k_cache, cache}, {"v_cache", v_cache, cache},
                      {"cache_len", cache_len, 4 * heads}, {"q", q, nodes * c.d * es}, {"k", k, nodes * c.d * es}, {"v", v, outs * c.d * es},
                      {"alpha", alpha, 4 * nodes}, {"beta", beta, 4 * nodes}, {"mask", mask, nodes}, {"parent", parent, 4 * (size_t)c.B * c.T},
                      {"n_nodes", n_nodes, 4 * (size_t)c.B}, {"q_nla", p->q_nla, outs * c.d * es}, {"k_nla", p->k_nla, outs * c.d * es},
                      {"w_nla", w_nla, 4 * outs}, {"w_la", w_la, 4 * outs}}, 3);
    if (st != NATS_OK) return st;
    c.scale = p->softmax_scale > 0.f ? p->softmax_scale : 1.0f / sqrtf((float)p->d);
    c.la_scale = p->la_scale > 0.f ? p->la_scale : 1.0f;
    c.eps = p->rms_eps > 0.f ? p->rms_eps : 1e-6f;
    c.combine_mode = p->combine_mode; c.linear_op = p->linear_op; c.freeze = p->freeze_on_softmax;
    c.state = state; c.k_cache = k_cache; c.v_cache = v_cache; c.cache_len = cache_len;
    c.q = q; c.k = k; c.v = v; c.q_nla = p->q_nla; c.k_nla = p->k_nla;
    c.alpha = alpha; c.beta = beta; c.mask = mask; c.parent = parent; c.n_nodes = n_nodes;
    c.w_nla = w_nla; c.w_la = w_la; c.o = o; c.lse = lse;
    c.ws = static_cast<float*>(workspace);
    return launch_tree(c, reinterpret_cast<hipStream_t>(hip_stream));
}

nats_status nats_hybrid_attn_tree_commit_ex(const nats_tree_params* p, float* state, void* k_cache, void* v_cache, int32_t* cache_len,
                                            const void* k, const void* v, const float* alpha, const float* beta, const uint8_t* mask,
                                            const int32_t* parent, const int32_t* n_nodes, const int32_t* node, int32_t* vis,
                                            int32_t* err_flags, void* hip_stream) {
    nats_status st = check_tree_params(p);
    if (st != NATS_OK) return st;
    if (!cache_len || !alpha || !beta || !mask || !parent || !node) {
        set_error("cache_len, alpha, beta, mask, parent and node must all be non-NULL");
        return NATS_ERR_NULL;
    }
    st = check_pointers({state, k_cache, v_cache, k, v}, "state, k_cache, v_cache, k and v", {p->k_nla});
    if (st != NATS_OK) return st;
    if (k_cache == v_cache) { set_error("k_cache and v_cache must be two arrays"); return NATS_ERR_SHAPE; }
    for (const void* in : {k, v, p->k_nla})
        if ((const void*)state == in || k_cache == in || v_cache == in) {
            set_error("state, k_cache and v_cache must not alias an input");
            return NATS_ERR_SHAPE;
        }
    TreeCommitCall c{};
    c.B = p->B; c.H = p->H; c.G = p->group ? p->group : 1; c.T = p->T; c.d = p->d; c.cap = p->cap; c.dtype = p->dtype;
    c.linear_op = p->linear_op; c.freeze = p->freeze_on_softmax;
    c.state = state; c.k_cache = k_cache; c.v_cache = v_cache; c.cache_len = cache_len;
    c.k = k; c.v = v; c.k_nla = p->k_nla; c.alpha = alpha; c.beta = beta; c.mask = mask; c.parent = parent;
    c.n_nodes = n_nodes; c.node = node; c.vis = vis; c.err_flags = err_flags;
    const size_t es = element(c.dtype), nodes = (size_t)c.B * c.H * c.T, heads = (size_t)c.B * c.H * c.G, outs = nodes * c.G;
    const size_t cache = heads * c.cap * c.d * es;
    st = check_apart({{"state", state, 4 * heads * c.d * c.d}, {"k_cache", k_cache, cache}, {"v_cache", v_cache, cache},
                      {"cache_len", cache_len, 4 * heads}, {"vis", vis, 4 * outs}, {"err_flags", err_flags, 4 * heads},
                      {"k", k, nodes * c.d * es}, {"v", v, outs * c.d * es}, {"alpha", alpha, 4 * nodes}, {"beta", beta, 4 * nodes},
                      {"mask", mask, nodes}, {"parent", parent, 4 * (size_t)c.B * c.T}, {"n_nodes", n_nodes, 4 * (size_t)c.B},
                      {"node", node, 4 * (size_t)c.B}, {"k_nla", p->k_nla, outs * c.d * es}}, 6);
    if (st != NATS_OK) return st;
    return launch_tree_commit(c, reinterpret_cast<hipStream_t>(hip_stream));
}

nats_status nats_hybrid_attn_tree_commit(const nats_tree_params* p, float* state, void* k_cache, void* v_cache, int32_t* cache_len,
                                         const void* k, const void* v, const float* alpha, const float* beta, const uint8_t* mask,
                                         const int32_t* parent, const int32_t* node, int32_t* vis, int32_t* err_flags,
                                         void* hip_stream) {
    return nats_hybrid_attn_tree_commit_ex(p, state, k_cache, v_cache, cache_len, k, v, alpha, beta, mask, parent, nullptr, node, vis,
                                           err_flags, hip_stream);
}

size_t nats_cache_weights_workspace_bytes(const nats_cache_weights_params* p, int32_t lse_given) {
    if (check_weights_params(p) != NATS_OK) return 0;
    WeightsCall c{};
    set_weights_sizes(*p, c);
    return weights_workspace(c, lse_given != 0) * 4;
}

nats_status nats_cache_weights(const nats_cache_weights_params* p, float* weights, const void* q, const void* k_cache,
                               const int32_t* cache_len, const int32_t* vis, const float* lse, void* workspace,
                               size_t workspace_bytes, void* hip_stream) {
    nats_status st = check_weights_params(p);
    if (st != NATS_OK) return st;
    if (!cache_len) { set_error("cache_len is NULL"); return NATS_ERR_NULL; }
    st = check_pointers({weights, q, k_cache}, "weights, q and k_cache", {});
    if (st != NATS_OK) return st;
    if ((const void*)weights == q || (const void*)weights == k_cache || weights == lse) {
        set_error("weights must not alias an input");
        return NATS_ERR_SHAPE;
    }
    WeightsCall c{};
    set_weights_sizes(*p, c);
    const size_t need = weights_workspace(c, lse != nullptr) * 4;
    if (need > 0 && (workspace == nullptr || workspace_bytes < need)) {
        set_error("workspace of %zu bytes given, %zu needed", workspace ? workspace_bytes : (size_t)0, need);
        return NATS_ERR_WORKSPACE;
    }
    if (!aligned16(workspace)) { set_error("the workspace is not 16-byte aligned"); return NATS_ERR_ALIGN; }
    const size_t es = element(c.dtype), heads = (size_t)c.B * c.H;
    st = check_apart({{"weights", weights, 4 * heads * c.cap}, {"the workspace", need > 0 ? workspace : nullptr, need},
                      {"q", q, heads / c.q_group * c.T * c.d * es}, {"k_cache", k_cache, heads * c.cap * c.d * es},
                      {"cache_len", cache_len, 4 * heads}, {"vis", vis, 4 * heads / c.vis_group * c.T}, {"lse", lse, 4 * heads * c.T}}, 2);
    if (st != NATS_OK) return st;
    c.weights = weights; c.q = q; c.k_cache = k_cache; c.cache_len = cache_len; c.vis = vis; c.lse = lse;
    c.ws = static_cast<float*>(workspace);
    return launch_cache_weights(c, reinterpret_cast<hipStream_t>(hip_stream));
}

static nats_status evict(const nats_cache_evict_params* p, void* k_cache, void* v_cache, int32_t* cache_len, float* weights,
                         int32_t* kept, int clear, void* hip_stream) {
    if (p == nullptr) { set_error("params is NULL"); return NATS_ERR_NULL; }
    nats_status st = check_cache(p->dtype, p->B, p->H, p->d, p->cap, 1);
    if (st != NATS_OK) return st;
    if (p->keep < 1 || p->keep > p->cap || p->recent < 0 || p->recent > p->keep) {
        set_error("keep must be between 1 and cap, recent between 0 and keep (cap %d, got %d, %d)", p->cap, p->keep, p->recent);
        return NATS_ERR_SHAPE;
    }
    if (!cache_len || !kept) { set_error("cache_len and kept must be non-NULL"); return NATS_ERR_NULL; }
    st = check_pointers({k_cache, v_cache, weights}, "k_cache, v_cache and weights", {});
    if (st != NATS_OK) return st;
    if (k_cache == v_cache) { set_error("k_cache and v_cache must be two arrays"); return NATS_ERR_SHAPE; }
    const size_t heads = (size_t)p->B * p->H, cache = heads * p->cap * p->d * element(p->dtype);
    st = check_apart({{"k_cache", k_cache, cache}, {"v_cache", v_cache, cache}, {"cache_len", cache_len, 4 * heads},
                      {"weights", weights, 4 * heads * p->cap}, {"kept", kept, 4 * heads * p->keep}}, 5);
    if (st != NATS_OK) return st;
    EvictCall c{p->B, p->H, p->d, p->cap, p->dtype, p->keep, p->recent, k_cache, v_cache, cache_len, weights, kept, clear};
    return launch_cache_evict(c, reinterpret_cast<hipStream_t>(hip_stream));
}

nats_status nats_cache_evict(const nats_cache_evict_params* p, void* k_cache, void* v_cache, int32_t* cache_len, float* weights,
                             int32_t* kept, void* hip_stream) {
    return evict(p, k_cache, v_cache, cache_len, weights, kept, 0, hip_stream);
}

nats_status nats_cache_evict_clear(const nats_cache_evict_params* p, void* k_cache, void* v_cache, int32_t* cache_len, float* weights,
                                   int32_t* kept, void* hip_stream) {
    return evict(p, k_cache, v_cache, cache_len, weights, kept, 1, hip_stream);
}

}  // extern "C"

// A tree of drafted tokens read against the decode state and the cache (nats_hybrid_attn_decode_tree), and the commit of its accepted
// path (nats_hybrid_attn_tree_commit).
#include <math.h>

#include "nats_common.h"
#include "nats_serve.h"
#include "serve.h"
#include "tree_nodes.h"

namespace nats {

// ---- the parts, the node's softmax ancestors and the linear branch's row into the output: a wavefront per node and head ----
constexpr int MERGE_THREADS = 256;

template <typename T, int D>
__global__ __launch_bounds__(MERGE_THREADS) void tree_merge_kernel(TreeCall c) {
    constexpr int CPL = D / 64;   // columns per lane, side by side
    const int lane = threadIdx.x & 63, bhg = blockIdx.y, bh = bhg / c.G, b = bh / c.H, N = c.T;
    const int t = blockIdx.x * (MERGE_THREADS / 64) + __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    if (t >= N) return;
    const size_t at = (size_t)bhg * N + t;
    auto columns = [&](const T* row, float (&x)[CPL]) {
#pragma unroll
        for (int i = 0; i < CPL; ++i) x[i] = to_float(row[lane * CPL + i]);
    };
    auto store = [&](const float (&x)[CPL]) {
#pragma unroll
        for (int i = 0; i < CPL; ++i) ((T*)c.o)[at * D + lane * CPL + i] = from_float<T>(x[i]);
    };
    float res[CPL] = {};
    if (c.n_nodes != nullptr && t >= c.n_nodes[b]) {
        store(res);
        if (lane == 0 && c.lse != nullptr) c.lse[at] = -INFINITY;
        return;
    }
    const int n = min(max(c.cache_len[bhg], 0), c.cap), parts = (n + c.rows - 1) / c.rows;
    const uint64_t soft = __ballot(lane < N && c.mask[(size_t)bh * N + min(lane, N - 1)] != 0);
    const uint64_t sees = soft & c.anc()[(size_t)b * N + t];
    // the nodes' logits, lane j for node j, in the parts' units (powers of 2)
    constexpr float LOG2E = 1.44269504088896341f, LN2 = 0.693147180559945309f;
    const T* ks = c.k_nla != nullptr ? (const T*)c.k_nla + (size_t)bhg * N * D : (const T*)c.k + (size_t)bh * N * D;
    const T* v = (const T*)c.v + (size_t)bhg * N * D;
    float q[CPL], x = -INFINITY;
    columns(c.q_nla != nullptr ? (const T*)c.q_nla + at * D : (const T*)c.q + ((size_t)bh * N + t) * D, q);
    for (uint64_t left = sees; left; left &= left - 1) {
        const int j = __builtin_ctzll(left);
        float k[CPL], dot = 0.f;
        columns(ks + (size_t)j * D, k);
#pragma unroll
        for (int i = 0; i < CPL; ++i) dot += q[i] * k[i];
        dot = lane_group_sum<64>(dot);
        if (lane == j) x = dot * (c.scale * LOG2E);
    }
    auto top_of = [](float y) {
#pragma unroll
        for (int w = 1; w < 64; w *= 2) y = fmaxf(y, __shfl_xor(y, w));
        return y;
    };
    const bool mine = (sees >> lane) & 1;
    float m = top_of(x), ref = m == -INFINITY ? 0.f : m;
    float p = mine ? __builtin_amdgcn_exp2f(x - ref) : 0.f, l = lane_group_sum<64>(p), acc[CPL] = {};
    for (uint64_t left = sees; left; left &= left - 1) {
        const int j = __builtin_ctzll(left);
        float vj[CPL];
        columns(v + (size_t)j * D, vj);
        const float pj = __shfl(p, j);
#pragma unroll
        for (int i = 0; i < CPL; ++i) acc[i] += pj * vj[i];
    }
    for (int first = 0; first < parts; first += 64) {
        const size_t part = ((size_t)bhg * c.n_split + first) * N + t;
        float2 ml = make_float2(-INFINITY, 0.f);
        if (first + lane < parts) ml = *reinterpret_cast<const float2*>(c.ws + c.off_ml + (part + (size_t)lane * N) * 2);
        const float top = fmaxf(m, top_of(ml.x));
        ref = top == -INFINITY ? 0.f : top;
        const float was = __builtin_amdgcn_exp2f(m - ref), w = __builtin_amdgcn_exp2f(ml.x - ref);
        m = top;
        l = l * was + lane_group_sum<64>(first + lane < parts ? w * ml.y : 0.f);
#pragma unroll
        for (int i = 0; i < CPL; ++i) acc[i] *= was;
        const float* rows = c.ws + c.off_part + part * D + lane * CPL;
        const int here = min(parts - first, 64);
#pragma unroll 8
        for (int s = 0; s < here; ++s) {
            const float ws = __shfl(w, s);
#pragma unroll
            for (int i = 0; i < CPL; ++i) acc[i] += ws * rows[(size_t)s * N * D + i];
        }
    }
    const bool none = n == 0 && sees == 0;
    if (lane == 0 && c.lse != nullptr) c.lse[at] = none ? -INFINITY : (m + log2f(l)) * LN2;
    float o_nla[CPL], o_la[CPL];
#pragma unroll
    for (int i = 0; i < CPL; ++i) {
        o_nla[i] = none ? 0.f : acc[i] / l;
        o_la[i] = c.ws[c.off_ola + at * D + lane * CPL + i];
        res[i] = o_la[i] + o_nla[i];
    }
    if (c.combine_mode != 0) {
        const float def = c.combine_mode == 1 ? 0.5f : 1.f;
        const float wn = c.w_nla != nullptr ? c.w_nla[at] : def, wl = c.w_la != nullptr ? c.w_la[at] : def;
        float sn = 0.f, sl = 0.f;
#pragma unroll
        for (int i = 0; i < CPL; ++i) {
            res[i] = wn * o_nla[i] + wl * o_la[i];
            sn += c.combine_mode == 1 ? o_nla[i] * o_nla[i] : res[i] * res[i];
            sl += o_la[i] * o_la[i];
        }
        sn = sqrtf(lane_group_sum<64>(sn) / D + c.eps);
        sl = sqrtf(lane_group_sum<64>(sl) / D + c.eps);
#pragma unroll
        for (int i = 0; i < CPL; ++i) res[i] = c.combine_mode == 1 ? wn * o_nla[i] / sn + wl * o_la[i] / sl : res[i] / sn;
    }
    store(res);
}

// ---- commit: a block per output head; LPR = D / 4 lanes hold a row of S as a float4 each, the rows of S are independent of one
// another, so that the path's tokens follow each other without a barrier ----
constexpr int COMMIT_THREADS = 256;

template <typename T, int D>
__global__ __launch_bounds__(COMMIT_THREADS) void tree_commit_kernel(TreeCommitCall c) {
    constexpr int LPR = D / 4, PER_PASS = COMMIT_THREADS / LPR, PASSES = D / PER_PASS;
    __shared__ int s_path[64], s_row[64];
    __shared__ float s_a[64], s_b[64];
    __shared__ int s_n;
    const int bhg = blockIdx.x, bh = bhg / c.G, b = bh / c.H, tid = threadIdx.x, N = c.T;
    const int node = c.node[b];
    const bool refused = node < -1 || node >= N;
    if (tid < 64) {
        const bool none = refused || node < 0;
        const uint64_t anc = shfl_u64(ancestors(parent_of(c.parent, b, N, tid), tid), none ? 0 : node), path = none ? 0 : anc;
        const bool on = (path >> tid) & 1;
        const bool soft = on && c.mask[(size_t)bh * N + tid] != 0;
        const uint64_t softs = __ballot(soft);
        const uint64_t upto = (2ull << tid) - 1;        // lanes 0 .. tid (lane 63: all)
        const int len = c.cache_len[bhg], had = min(max(len, 0), c.cap), room = len < 0 ? 0 : c.cap - had;
        const int rank = __popcll(softs & upto), stored = min(__popcll(softs), room);
        if (on) {
            const int p = __popcll(path & (upto >> 1));
            s_path[p] = tid;
            s_a[p] = soft && c.freeze ? 1.f : c.alpha[(size_t)bh * N + tid];
            s_b[p] = soft ? 0.f : c.beta[(size_t)bh * N + tid];
            s_row[p] = soft && rank <= room ? had + rank - 1 : -1;
        }
        if (c.vis != nullptr && tid < N) c.vis[(size_t)bhg * N + tid] = on ? had + min(rank, room) : 0;
        if (tid == 0) {
            s_n = __popcll(path);
            if (stored > 0) c.cache_len[bhg] = had + stored;
            if (c.err_flags != nullptr) c.err_flags[bhg] = refused ? 2 : __popcll(softs) > room ? 1 : 0;
        }
    }
    __syncthreads();
    const int n = s_n;
    if (n == 0) return;
    const int lr = tid % LPR, r0 = tid / LPR;
    float* Sb = c.state + (size_t)bhg * D * D;
    const T* k = (const T*)c.k + (size_t)bh * N * D;
    const T* ks = c.k_nla != nullptr ? (const T*)c.k_nla + (size_t)bhg * N * D : k;
    const T* v = (const T*)c.v + (size_t)bhg * N * D;
    float4 S[PASSES];
#pragma unroll
    for (int p = 0; p < PASSES; ++p) S[p] = *reinterpret_cast<const float4*>(Sb + (size_t)(p * PER_PASS + r0) * D + lr * 4);
    for (int i = 0; i < n; ++i) {
        const int t = s_path[i], row = s_row[i];
        const float a = s_a[i], bt = s_b[i];
        float kk[4];
#pragma unroll
        for (int j = 0; j < 4; ++j) kk[j] = to_float(k[t * D + lr * 4 + j]);
#pragma unroll
        for (int p = 0; p < PASSES; ++p) {
            float4 s = S[p];
            s.x *= a; s.y *= a; s.z *= a; s.w *= a;
            if (bt != 0.f) {
                const float pred = lane_group_sum<LPR>(s.x * kk[0] + s.y * kk[1] + s.z * kk[2] + s.w * kk[3]);
                const float delta = bt * (to_float(v[t * D + p * PER_PASS + r0]) - (c.linear_op == 0 ? pred : 0.f));
                s.x += delta * kk[0]; s.y += delta * kk[1]; s.z += delta * kk[2]; s.w += delta * kk[3];
            }
            S[p] = s;
        }
        if (row >= 0 && tid < D) {
            ((T*)c.k_cache)[((size_t)bhg * c.cap + row) * D + tid] = ks[t * D + tid];
            ((T*)c.v_cache)[((size_t)bhg * c.cap + row) * D + tid] = v[t * D + tid];
        }
    }
#pragma unroll
    for (int p = 0; p < PASSES; ++p) *reinterpret_cast<float4*>(Sb + (size_t)(p * PER_PASS + r0) * D + lr * 4) = S[p];
}

// ---- host side ----
size_t tree_workspace(TreeCall& c) {
    const size_t heads = (size_t)c.B * c.H * c.G;
    c.rows = tree_cache_rows(c);
    c.n_split = (c.cap + c.rows - 1) / c.rows;
    c.off_anc = 0;
    c.off_ola = align_up((size_t)c.B * c.T * 2, 4);
    c.off_part = c.off_ola + heads * c.T * c.d;
    c.off_ml = c.off_part + heads * c.n_split * c.T * c.d;
    return c.off_ml + heads * c.n_split * c.T * 2;
}

template <typename T, int D>
static nats_status run_tree(const TreeCall& c, hipStream_t st) {
    const int heads = c.B * c.H * c.G;
    const nats_status r = launch_tree_read(c, st);
    if (r != NATS_OK) return r;
    constexpr int NODES = MERGE_THREADS / 64;
    ProfScope ps("tree_merge", st);
    hipLaunchKernelGGL((tree_merge_kernel<T, D>), dim3((c.T + NODES - 1) / NODES, heads), dim3(MERGE_THREADS), 0, st, c);
    return check_launch("tree");
}

nats_status launch_tree(const TreeCall& c, hipStream_t st) {
    if (c.dtype == NATS_F32) return c.d == 64 ? run_tree<float, 64>(c, st) : run_tree<float, 128>(c, st);
    return c.d == 64 ? run_tree<bf16_t, 64>(c, st) : run_tree<bf16_t, 128>(c, st);
}

template <typename T, int D>
static nats_status run_commit(const TreeCommitCall& c, hipStream_t st) {
    ProfScope ps("tree_commit", st);
    hipLaunchKernelGGL((tree_commit_kernel<T, D>), dim3(c.B * c.H * c.G), dim3(COMMIT_THREADS), 0, st, c);
    return check_launch("tree_commit");
}

nats_status launch_tree_commit(const TreeCommitCall& c, hipStream_t st) {
    if (c.dtype == NATS_F32) return c.d == 64 ? run_commit<float, 64>(c, st) : run_commit<float, 128>(c, st);
    return c.d == 64 ? run_commit<bf16_t, 64>(c, st) : run_commit<bf16_t, 128>(c, st);
}

}  // namespace nats

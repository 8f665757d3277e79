// A tree of drafted tokens read against the decode state and the cache (nats_hybrid_attn_decode_tree), and the commit of its accepted
// path (nats_hybrid_attn_tree_commit).
#include <math.h>

#include "mfma_util.h"
#include "nats_common.h"
#include "nats_serve.h"
#include "serve.h"
#include "tree_nodes.h"

namespace nats {

// ---- the parts, the node's softmax ancestors and the linear branch's row into the output: 32 lanes per node and head ----
// Bound by its chain of trips to memory (which parts there are, what is in them), so everything else is asked for at once; two nodes to
// a wavefront are half as many wavefronts (1024 heads with 16 nodes: 12.8 us against 13.9 with one).
constexpr int MERGE_THREADS = 256, MERGE_LANES = 32, MERGE_NODES = MERGE_THREADS / MERGE_LANES;

template <typename T, int D>
__global__ __launch_bounds__(MERGE_THREADS) void tree_merge_kernel(TreeCall c) {
    constexpr int CPL = D / MERGE_LANES;   // columns per lane, side by side
    constexpr int AHEAD = 4;               // parts that are asked for before it is known which there are (a part's place exists whatever
                                           // the length; what it holds enters only if the part does)
    constexpr float LOG2E = 1.44269504088896341f, LN2 = 0.693147180559945309f;
    typedef float cols __attribute__((ext_vector_type(CPL)));
    const int lane = threadIdx.x & 63, sl = lane % MERGE_LANES, bhg = blockIdx.y, bh = bhg / c.G, b = bh / c.H, N = c.T;
    const int node = blockIdx.x * MERGE_NODES + threadIdx.x / MERGE_LANES, t = min(node, N - 1);
    const size_t at = (size_t)bhg * N + t;
    auto columns = [&](const T* row) {
        cols x;
        if constexpr (sizeof(T) == 4) {
            x = *reinterpret_cast<const cols*>(row + sl * CPL);
        } else {
#pragma unroll
            for (int i = 0; i < CPL; i += 2) {
                const uint32_t w = *reinterpret_cast<const uint32_t*>(row + sl * CPL + i);
                x[i] = __uint_as_float(w << 16);
                x[i + 1] = __uint_as_float(w & 0xffff0000u);
            }
        }
        return x;
    };
    const int n = min(max(c.cache_len[bhg], 0), c.cap);
    int slot0 = bhg * c.n_split, parts = (n + c.rows - 1) / c.rows, last = c.n_split - 1;
    if (c.even) {
        const int32_t* units = c.units();
        const int from = units[bhg], to = units[bhg + 1], share = units[gridDim.y + 1];
        slot0 = bhg + from / share;
        parts = to > from ? (to - 1) / share - from / share + 1 : 0;
        last = max(parts - 1, 0);
    }
    const size_t part0 = (size_t)slot0 * N + t;
    const T* ks = c.k_nla != nullptr ? (const T*)c.k_nla + (size_t)bhg * N * D : (const T*)c.k + (size_t)bh * N * D;
    const T* v = (const T*)c.v + (size_t)bhg * N * D;
    const float* rows = c.ws + c.off_part + part0 * D + sl * CPL;
    const bool dead = c.n_nodes != nullptr && t >= c.n_nodes[b];
    const uint64_t anc = c.anc()[(size_t)b * N + t];
    const bool is_soft = c.mask[(size_t)bh * N + min(lane, N - 1)] != 0;
    const cols q = columns(c.q_nla != nullptr ? (const T*)c.q_nla + at * D : (const T*)c.q + ((size_t)bh * N + t) * D);
    float2 ml = *reinterpret_cast<const float2*>(c.ws + c.off_ml + (part0 + (size_t)min(sl, last) * N) * 2);
    cols ahead[AHEAD];
#pragma unroll
    for (int s = 0; s < AHEAD; ++s) ahead[s] = *reinterpret_cast<const cols*>(rows + (size_t)min(s, last) * N * D);
    const cols o_la = *reinterpret_cast<const cols*>(c.ws + c.off_ola + at * D + sl * CPL);
    const uint64_t sees = anc & __ballot(lane < N && is_soft);

    // the node's softmax ancestors, four at a time; logits in the parts' units (powers of 2), the same in every lane of the node
    float m = -INFINITY, l = 0.f;
    cols acc = {};
    for (uint64_t left = sees; __any(left != 0);) {
        cols k[4], x[4];
        float z[4], top = m;
        bool there[4];
#pragma unroll
        for (int e = 0; e < 4; ++e) {
            there[e] = left != 0;
            const int j = there[e] ? __builtin_ctzll(left) : 0;
            left &= left - 1;   // (0 stays 0)
            k[e] = columns(ks + (size_t)j * D);
            x[e] = columns(v + (size_t)j * D);
        }
#pragma unroll
        for (int e = 0; e < 4; ++e) {
            float dot = 0.f;
#pragma unroll
            for (int i = 0; i < CPL; ++i) dot += q[i] * k[e][i];
            dot = lane_group_sum<MERGE_LANES>(dot) * (c.scale * LOG2E);
            z[e] = there[e] ? dot : -INFINITY;
            top = fmaxf(top, z[e]);
        }
        const float ref = top == -INFINITY ? 0.f : top, was = __builtin_amdgcn_exp2f(m - ref);
        m = top;
        l *= was;
        acc *= was;
#pragma unroll
        for (int e = 0; e < 4; ++e)
            if (there[e]) {   // (a node that is not seen may hold anything)
                const float p = __builtin_amdgcn_exp2f(z[e] - ref);
                l += p;
                acc += p * x[e];
            }
    }
    for (int first = 0; first < parts; first += MERGE_LANES) {
        if (first > 0 && first + sl < parts)
            ml = *reinterpret_cast<const float2*>(c.ws + c.off_ml + (part0 + (size_t)(first + sl) * N) * 2);
        if (first + sl >= parts) ml = make_float2(-INFINITY, 0.f);
        float top = ml.x;
#pragma unroll
        for (int w = 1; w < MERGE_LANES; w *= 2) top = fmaxf(top, __shfl_xor(top, w));
        top = fmaxf(top, m);
        const float ref = top == -INFINITY ? 0.f : top;
        const float was = __builtin_amdgcn_exp2f(m - ref), w = __builtin_amdgcn_exp2f(ml.x - ref);
        m = top;
        l = l * was + lane_group_sum<MERGE_LANES>(w * ml.y);
        acc *= was;
        const int here = min(parts - first, MERGE_LANES), own = lane & ~(MERGE_LANES - 1);
        int s = 0;
        if (first == 0) {
#pragma unroll
            for (int e = 0; e < AHEAD; ++e)
                if (e < here) acc += __shfl(w, own + e) * ahead[e];
            s = AHEAD;
        }
#pragma unroll 8
        for (; s < here; ++s) acc += __shfl(w, own + s) * *reinterpret_cast<const cols*>(rows + (size_t)(first + s) * N * D);
    }
    const bool none = dead || (n == 0 && sees == 0);
    cols o_nla, res;
#pragma unroll
    for (int i = 0; i < CPL; ++i) o_nla[i] = none ? 0.f : acc[i] / l;
    res = o_la + o_nla;
    if (c.combine_mode != 0) {
        const float def = c.combine_mode == 1 ? 0.5f : 1.f;
        const float wn = c.w_nla != nullptr ? c.w_nla[at] : def, wl = c.w_la != nullptr ? c.w_la[at] : def;
        float sn = 0.f, sl2 = 0.f;
        res = wn * o_nla + wl * o_la;
#pragma unroll
        for (int i = 0; i < CPL; ++i) {
            sn += c.combine_mode == 1 ? o_nla[i] * o_nla[i] : res[i] * res[i];
            sl2 += o_la[i] * o_la[i];
        }
        sn = sqrtf(lane_group_sum<MERGE_LANES>(sn) / D + c.eps);
        sl2 = sqrtf(lane_group_sum<MERGE_LANES>(sl2) / D + c.eps);
#pragma unroll
        for (int i = 0; i < CPL; ++i) res[i] = c.combine_mode == 1 ? wn * o_nla[i] / sn + wl * o_la[i] / sl2 : res[i] / sn;
    }
    if (node >= N) return;
    if (sl == 0 && c.lse != nullptr) c.lse[at] = none ? -INFINITY : (m + log2f(l)) * LN2;
    T* o = (T*)c.o + at * D + sl * CPL;
    if constexpr (sizeof(T) == 4) {
#pragma unroll
        for (int i = 0; i < CPL; ++i) res[i] = dead ? 0.f : res[i];
        *reinterpret_cast<cols*>(o) = res;
    } else {
#pragma unroll
        for (int i = 0; i < CPL; i += 2) *reinterpret_cast<uint32_t*>(o + i) = dead ? 0u : pack_bf16x2(res[i], res[i + 1]);
    }
}

// ---- commit ----------------------------------------------------------------------------------------------------------------------
// A block per output head.  Eight lanes hold a row of S (D / 8 elements each), and the rows are independent of one another, so that the path's
// tokens follow each other without a barrier; eight tokens at a time come through LDS.  The state is kept as S / G with G the product
// of the decays so far: a softmax token then costs nothing and a linear one two operations per element, the product with k and
// the update (S would take a third).  G is taken back into S where it leaves 2^-40 .. 2.  S / G leaves fp32's range before S does, by as
// much as 2^40; a wavefront whose rows are not all finite at the end takes its tokens again, S by S.
constexpr int COMMIT_THREADS = 256, COMMIT_TOKENS = 8;

template <typename T, int D>
__global__ __launch_bounds__(COMMIT_THREADS) void tree_commit_kernel(TreeCommitCall c) {
    constexpr int LPR = 8, PER_PASS = COMMIT_THREADS / LPR, PASSES = D / PER_PASS, W = D / 32;   // W: 4 elements each of a lane's share
    __shared__ float s_k[COMMIT_TOKENS][D], s_v[COMMIT_TOKENS][D];
    __shared__ int s_path[64], s_row[64];
    __shared__ float s_a[64], s_b[64];
    __shared__ int s_n;
    const int bhg = blockIdx.x, bh = bhg / c.G, b = bh / c.H, tid = threadIdx.x, N = c.T;
    const int lr = tid % LPR, r0 = tid / LPR;
    float* Sb = c.state + (size_t)bhg * D * D;
    f32x4 S[PASSES][W];
#pragma unroll
    for (int p = 0; p < PASSES; ++p)
#pragma unroll
        for (int x = 0; x < W; ++x) S[p][x] = *reinterpret_cast<const f32x4*>(Sb + (size_t)(p * PER_PASS + r0) * D + 32 * x + 4 * lr);
    if (tid < 64) {
        const int node = c.node[b], there = c.n_nodes != nullptr ? min(max(c.n_nodes[b], 0), N) : N;
        const bool refused = node < -1 || node >= there, none = refused || node < 0;
        const bool softmax = c.mask[(size_t)bh * N + min(tid, N - 1)] != 0;
        const float alpha = c.alpha[(size_t)bh * N + min(tid, N - 1)], beta = c.beta[(size_t)bh * N + min(tid, N - 1)];
        const int len = c.cache_len[bhg], had = min(max(len, 0), c.cap), room = len < 0 ? 0 : c.cap - had;
        const uint64_t anc = shfl_u64(ancestors(parent_of(c.parent, b, N, tid), tid), none ? 0 : node), path = none ? 0 : anc;
        const bool on = (path >> tid) & 1, soft = on && softmax;
        const uint64_t softs = __ballot(soft);
        const uint64_t upto = (2ull << tid) - 1;        // lanes 0 .. tid (lane 63: all)
        const int rank = __popcll(softs & upto), stored = min(__popcll(softs), room);
        if (on) {
            const int p = __popcll(path & (upto >> 1));
            s_path[p] = tid;
            s_a[p] = soft && c.freeze ? 1.f : alpha;
            s_b[p] = soft ? 0.f : beta;
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
    const T* k = (const T*)c.k + (size_t)bh * N * D;
    const T* ks = c.k_nla != nullptr ? (const T*)c.k_nla + (size_t)bhg * N * D : k;
    const T* v = (const T*)c.v + (size_t)bhg * N * D;
    float G = 1.f;
    for (int first = 0; first < n; first += COMMIT_TOKENS) {
        const int here = min(n - first, COMMIT_TOKENS);
        if (first > 0) __syncthreads();   // the tokens before have been used
        for (int e = tid; e < here * D; e += COMMIT_THREADS) {
            const int i = e / D, x = e % D, t = s_path[first + i], row = s_row[first + i];
            const T vx = v[t * D + x];
            s_k[i][x] = to_float(k[t * D + x]);
            s_v[i][x] = to_float(vx);
            if (row >= 0) {
                ((T*)c.k_cache)[((size_t)bhg * c.cap + row) * D + x] = ks[t * D + x];
                ((T*)c.v_cache)[((size_t)bhg * c.cap + row) * D + x] = vx;
            }
        }
        __syncthreads();
        for (int i = 0; i < here; ++i) {
            const float bt = s_b[first + i];
            G *= s_a[first + i];
            if (!(fabsf(G) > 0x1p-40f && fabsf(G) < 2.f)) {
#pragma unroll
                for (int p = 0; p < PASSES; ++p)
#pragma unroll
                    for (int x = 0; x < W; ++x) S[p][x] *= G;
                G = 1.f;
            }
            if (bt == 0.f) continue;
            f32x4 kk[W];
#pragma unroll
            for (int x = 0; x < W; ++x) kk[x] = *reinterpret_cast<const f32x4*>(&s_k[i][32 * x + 4 * lr]);
            const float inv = 1.f / G;
#pragma unroll
            for (int p = 0; p < PASSES; ++p) {
                float u = s_v[i][p * PER_PASS + r0];
                if (c.linear_op == 0) {
                    float pred = 0.f;
#pragma unroll
                    for (int x = 0; x < W; ++x)
                        pred += S[p][x][0] * kk[x][0] + S[p][x][1] * kk[x][1] + S[p][x][2] * kk[x][2] + S[p][x][3] * kk[x][3];
                    u -= G * lane_group_sum<LPR>(pred);
                }
                u *= bt * inv;
#pragma unroll
                for (int x = 0; x < W; ++x) S[p][x] += u * kk[x];
            }
        }
    }
    bool fine = true;
#pragma unroll
    for (int p = 0; p < PASSES; ++p)
#pragma unroll
        for (int x = 0; x < W; ++x)
#pragma unroll
            for (int e = 0; e < 4; ++e) fine = fine && fabsf(S[p][x][e]) < INFINITY;
    if (!__all(fine)) {
        G = 1.f;
#pragma unroll
        for (int p = 0; p < PASSES; ++p)
#pragma unroll
            for (int x = 0; x < W; ++x) S[p][x] = *reinterpret_cast<const f32x4*>(Sb + (size_t)(p * PER_PASS + r0) * D + 32 * x + 4 * lr);
        for (int i = 0; i < n; ++i) {
            const int t = s_path[i];
            const float a = s_a[i], bt = s_b[i];
            f32x4 kk[W];
#pragma unroll
            for (int x = 0; x < W; ++x)
#pragma unroll
                for (int e = 0; e < 4; ++e) kk[x][e] = to_float(k[t * D + 32 * x + 4 * lr + e]);
#pragma unroll
            for (int p = 0; p < PASSES; ++p) {
#pragma unroll
                for (int x = 0; x < W; ++x) S[p][x] *= a;
                if (bt == 0.f) continue;
                float u = to_float(v[t * D + p * PER_PASS + r0]);
                if (c.linear_op == 0) {
                    float pred = 0.f;
#pragma unroll
                    for (int x = 0; x < W; ++x)
                        pred += S[p][x][0] * kk[x][0] + S[p][x][1] * kk[x][1] + S[p][x][2] * kk[x][2] + S[p][x][3] * kk[x][3];
                    u -= lane_group_sum<LPR>(pred);
                }
                u *= bt;
#pragma unroll
                for (int x = 0; x < W; ++x) S[p][x] += u * kk[x];
            }
        }
    }
#pragma unroll
    for (int p = 0; p < PASSES; ++p)
#pragma unroll
        for (int x = 0; x < W; ++x) *reinterpret_cast<f32x4*>(Sb + (size_t)(p * PER_PASS + r0) * D + 32 * x + 4 * lr) = G * S[p][x];
}

// ---- host side ----
size_t tree_workspace(TreeCall& c) {
    const size_t heads = (size_t)c.B * c.H * c.G;
    tree_cache_parts(c);
    const size_t parts = c.even ? heads + c.even : heads * c.n_split;
    c.off_anc = 0;
    c.off_ola = align_up((size_t)c.B * c.T * 2, 4);
    c.off_part = c.off_ola + heads * c.T * c.d;
    c.off_ml = c.off_part + parts * c.T * c.d;
    c.off_units = c.off_ml + parts * c.T * 2;
    return c.off_units + (c.even ? heads + 2 : 0);
}

template <typename T, int D>
static nats_status run_tree(const TreeCall& c, hipStream_t st) {
    const int heads = c.B * c.H * c.G;
    const nats_status r = launch_tree_read(c, st);
    if (r != NATS_OK) return r;
    ProfScope ps("tree_merge", st);
    hipLaunchKernelGGL((tree_merge_kernel<T, D>), dim3((c.T + MERGE_NODES - 1) / MERGE_NODES, heads), dim3(MERGE_THREADS), 0, st, c);
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

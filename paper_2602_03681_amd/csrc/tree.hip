// A tree of drafted tokens read against the decode state and the cache (nats_hybrid_attn_decode_tree), and the commit of its accepted
// path (nats_hybrid_attn_tree_commit).
#include <math.h>

#include "nats_common.h"
#include "nats_serve.h"
#include "serve.h"

namespace nats {

// The ancestor set of every node as a bit mask (itself among them), by one wavefront, lane i for node i: pointer jumping, six rounds
// whatever the tree.  parent in [-1, i - 1].
__device__ __forceinline__ uint64_t ancestors(int parent, int lane) {
    uint64_t m = 1ull << lane;
    int up = parent;
#pragma unroll
    for (int r = 0; r < 6; ++r) {
        const int at = up < 0 ? lane : up;
        const uint32_t lo = (uint32_t)__shfl((int)(uint32_t)m, at), hi = (uint32_t)__shfl((int)(uint32_t)(m >> 32), at);
        const int next = __shfl(up, at);
        if (up >= 0) {
            m |= ((uint64_t)hi << 32) | lo;
            up = next;
        }
    }
    return m;
}

// parent[b][i] as the kernels use it: what is no earlier node counts as the root
__device__ __forceinline__ int parent_of(const int32_t* parent, int b, int T, int i) {
    const int p = i < T ? parent[(size_t)b * T + i] : -1;
    return p >= 0 && p < i ? p : -1;
}

// ---- linear branch: a block per output head, thread r for state row r ----
//   u_i = b_i (v_i - g_i S k_i - sum_j r_ij (k_i . k_j) u_j),  o_i = la_scale (g_i S q_i + sum_j r_ij (q_i . k_j) u_j)
template <typename T, int D>
__global__ __launch_bounds__(D) void tree_linear_kernel(TreeCall c) {
    __shared__ float s_a[64], s_b[64], s_A[64][64], s_P[64][64];
    __shared__ uint64_t s_anc[64];
    __shared__ int s_par[64];
    const int bhg = blockIdx.x, bh = bhg / c.G, b = bh / c.H, tid = threadIdx.x, N = c.T;
    const T* q = (const T*)c.q + (size_t)bh * N * D;
    const T* k = (const T*)c.k + (size_t)bh * N * D;
    const T* v = (const T*)c.v + (size_t)bhg * N * D;
    if (tid < 64) {
        const int par = parent_of(c.parent, b, N, tid);
        s_par[tid] = par;
        s_anc[tid] = ancestors(par, tid);
        if (tid < N) {
            const bool soft = c.mask[(size_t)bh * N + tid] != 0;
            s_a[tid] = soft && c.freeze ? 1.f : c.alpha[(size_t)bh * N + tid];
            s_b[tid] = soft ? 0.f : c.beta[(size_t)bh * N + tid];
        }
    }
    __syncthreads();
    for (int e = tid; e < N * N; e += D) {
        const int i = e / N, j = e % N;
        if (!((s_anc[i] >> j) & 1)) continue;
        float r = 1.f;
        for (int n = i; n != j; n = s_par[n]) r *= s_a[n];
        float kk = 0.f, qk = 0.f;
        for (int x = 0; x < D; ++x) {
            const float kj = to_float(k[j * D + x]);
            kk += to_float(k[i * D + x]) * kj;
            qk += to_float(q[i * D + x]) * kj;
        }
        s_A[i][j] = r * kk;
        s_P[i][j] = r * qk;
    }
    __syncthreads();
    float S[D];
    for (int x = 0; x < D; ++x) S[x] = c.state[((size_t)bhg * D + tid) * D + x];
    float* U = c.ws + c.off_u + (size_t)bhg * N * D;
    float* O = c.ws + c.off_ola + (size_t)bhg * N * D;
    for (int i = 0; i < N; ++i) {
        float g = 1.f;
        for (int n = i; n >= 0; n = s_par[n]) g *= s_a[n];
        float sk = 0.f, sq = 0.f;
        for (int x = 0; x < D; ++x) {
            sk += S[x] * to_float(k[i * D + x]);
            sq += S[x] * to_float(q[i * D + x]);
        }
        sk *= g;
        sq *= g;
        for (uint64_t m = s_anc[i] & ~(1ull << i); m; m &= m - 1) {
            const int j = __builtin_ctzll(m);
            if (s_b[j] == 0.f) continue;
            sk += s_A[i][j] * U[j * D + tid];
            sq += s_P[i][j] * U[j * D + tid];
        }
        if (s_b[i] != 0.f) {
            const float u = s_b[i] * (to_float(v[i * D + tid]) - (c.linear_op == 0 ? sk : 0.f));
            U[i * D + tid] = u;
            sq += s_P[i][i] * u;
        }
        O[i * D + tid] = c.la_scale * sq;
    }
}

// ---- softmax branch: partial results (m, l, sum of weighted rows) of TREE_ROWS cache rows for one node ----
constexpr int TREE_ROWS = 256;

template <typename T, int D>
__global__ __launch_bounds__(TREE_ROWS) void tree_cache_kernel(TreeCall c) {
    __shared__ float s_p[TREE_ROWS], s_q[D], s_red[8], s_acc[TREE_ROWS / D][D];
    const int t = blockIdx.x, split = blockIdx.y, bhg = blockIdx.z, tid = threadIdx.x, N = c.T;
    const int n = min(max(c.cache_len[bhg], 0), c.cap), lo = split * TREE_ROWS, here = min(n - lo, TREE_ROWS);
    if (here <= 0) return;
    const T* q = c.q_nla != nullptr ? (const T*)c.q_nla + ((size_t)bhg * N + t) * D : (const T*)c.q + ((size_t)(bhg / c.G) * N + t) * D;
    if (tid < D) s_q[tid] = to_float(q[tid]) * c.scale;
    __syncthreads();
    const T* K = (const T*)c.k_cache + ((size_t)bhg * c.cap + lo) * D;
    const T* V = (const T*)c.v_cache + ((size_t)bhg * c.cap + lo) * D;
    float x = -INFINITY;
    if (tid < here) {
        x = 0.f;
        for (int e = 0; e < D; ++e) x += s_q[e] * to_float(K[(size_t)tid * D + e]);
    }
    float m = x;
    for (int w = 1; w < 64; w *= 2) m = fmaxf(m, __shfl_xor(m, w));
    if ((tid & 63) == 0) s_red[tid >> 6] = m;
    __syncthreads();
    m = fmaxf(fmaxf(s_red[0], s_red[1]), fmaxf(s_red[2], s_red[3]));
    const float ref = m == -INFINITY ? 0.f : m;
    const float p = tid < here ? expf(x - ref) : 0.f;
    s_p[tid] = p;
    const float l = lane_group_sum<64>(p);
    if ((tid & 63) == 0) s_red[4 + (tid >> 6)] = l;
    __syncthreads();
    const int col = tid % D, part = tid / D;
    float acc = 0.f;
    for (int r = part; r < here; r += TREE_ROWS / D) acc += s_p[r] * to_float(V[(size_t)r * D + col]);
    s_acc[part][col] = acc;
    __syncthreads();
    float* out = c.ws + c.off_part + (((size_t)bhg * c.n_split + split) * N + t) * (D + 2);
    if (tid < D) {
        acc = 0.f;
        for (int i = 0; i < TREE_ROWS / D; ++i) acc += s_acc[i][tid];
        out[2 + tid] = acc;
        if (tid == 0) {
            out[0] = m;
            out[1] = s_red[4] + s_red[5] + s_red[6] + s_red[7];
        }
    }
}

// ---- the parts, the node's softmax ancestors and the linear branch's row into the output: a block per node and head ----
template <typename T, int D>
__global__ __launch_bounds__(D) void tree_merge_kernel(TreeCall c) {
    __shared__ float s_red[4];
    __shared__ uint64_t s_sees;
    const int t = blockIdx.x, bhg = blockIdx.y, bh = bhg / c.G, b = bh / c.H, tid = threadIdx.x, N = c.T;
    auto block_sum = [&](float x) {
        x = lane_group_sum<64>(x);
        __syncthreads();
        if ((tid & 63) == 0) s_red[tid >> 6] = x;
        __syncthreads();
        return D > 64 ? s_red[0] + s_red[1] : s_red[0];
    };
    T* o = (T*)c.o + ((size_t)bhg * N + t) * D;
    if (c.n_nodes != nullptr && t >= c.n_nodes[b]) {
        o[tid] = from_float<T>(0.f);
        if (tid == 0 && c.lse != nullptr) c.lse[(size_t)bhg * N + t] = -INFINITY;
        return;
    }
    if (tid < 64) {
        uint64_t anc = ancestors(parent_of(c.parent, b, N, tid), tid);
        const uint64_t soft = __ballot(tid < N && c.mask[(size_t)bh * N + min(tid, N - 1)] != 0);
        if (tid == t) s_sees = anc & soft;
    }
    __syncthreads();
    const T* qs = c.q_nla != nullptr ? (const T*)c.q_nla + (size_t)bhg * N * D : (const T*)c.q + (size_t)bh * N * D;
    const T* ks = c.k_nla != nullptr ? (const T*)c.k_nla + (size_t)bhg * N * D : (const T*)c.k + (size_t)bh * N * D;
    const T* v = (const T*)c.v + (size_t)bhg * N * D;
    const int n = min(max(c.cache_len[bhg], 0), c.cap), parts = (n + TREE_ROWS - 1) / TREE_ROWS;
    float m = -INFINITY, l = 0.f, acc = 0.f;
    auto fold = [&](float m2, float l2, float acc2) {
        const float top = fmaxf(m, m2), ref = top == -INFINITY ? 0.f : top;
        const float w1 = expf(m - ref), w2 = expf(m2 - ref);
        l = w1 * l + w2 * l2;
        acc = w1 * acc + w2 * acc2;
        m = top;
    };
    for (int s = 0; s < parts; ++s) {
        const float* part = c.ws + c.off_part + (((size_t)bhg * c.n_split + s) * N + t) * (D + 2);
        fold(part[0], part[1], part[2 + tid]);
    }
    for (uint64_t x = s_sees; x; x &= x - 1) {
        const int j = __builtin_ctzll(x);
        const float dot = block_sum(to_float(qs[t * D + tid]) * c.scale * to_float(ks[j * D + tid]));
        fold(dot, 1.f, to_float(v[j * D + tid]));
    }
    const bool none = n == 0 && s_sees == 0;
    const float o_nla = none ? 0.f : acc / l;
    const float o_la = c.ws[c.off_ola + ((size_t)bhg * N + t) * D + tid];
    if (tid == 0 && c.lse != nullptr) c.lse[(size_t)bhg * N + t] = none ? -INFINITY : m + logf(l);
    float res = o_la + o_nla;
    if (c.combine_mode != 0) {
        const float def = c.combine_mode == 1 ? 0.5f : 1.f;
        const float wn = c.w_nla != nullptr ? c.w_nla[(size_t)bhg * N + t] : def;
        const float wl = c.w_la != nullptr ? c.w_la[(size_t)bhg * N + t] : def;
        if (c.combine_mode == 1) {
            const float sn = block_sum(o_nla * o_nla), sl = block_sum(o_la * o_la);
            res = wn * o_nla / sqrtf(sn / D + c.eps) + wl * o_la / sqrtf(sl / D + c.eps);
        } else {
            res = wn * o_nla + wl * o_la;
            res = res / sqrtf(block_sum(res * res) / D + c.eps);
        }
    }
    o[tid] = from_float<T>(res);
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
        const uint64_t anc = ancestors(parent_of(c.parent, b, N, tid), tid);
        const int at = refused || node < 0 ? 0 : node;
        const uint32_t lo = (uint32_t)__shfl((int)(uint32_t)anc, at), hi = (uint32_t)__shfl((int)(uint32_t)(anc >> 32), at);
        const uint64_t path = refused || node < 0 ? 0 : ((uint64_t)hi << 32) | lo;
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
size_t tree_workspace(TreeCall& c) {   // floats; fills the offsets
    const size_t heads = (size_t)c.B * c.H * c.G;
    c.n_split = (c.cap + TREE_ROWS - 1) / TREE_ROWS;
    c.off_ola = 0;
    c.off_u = heads * c.T * c.d;
    c.off_part = 2 * heads * c.T * c.d;
    return c.off_part + heads * c.n_split * c.T * (c.d + 2);
}

template <typename T, int D>
static nats_status run_tree(const TreeCall& c, hipStream_t st) {
    const int heads = c.B * c.H * c.G;
    {
        ProfScope ps("tree_linear", st);
        hipLaunchKernelGGL((tree_linear_kernel<T, D>), dim3(heads), dim3(D), 0, st, c);
    }
    {
        ProfScope ps("tree_cache", st);
        hipLaunchKernelGGL((tree_cache_kernel<T, D>), dim3(c.T, c.n_split, heads), dim3(TREE_ROWS), 0, st, c);
    }
    ProfScope ps("tree_merge", st);
    hipLaunchKernelGGL((tree_merge_kernel<T, D>), dim3(c.T, heads), dim3(D), 0, st, c);
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

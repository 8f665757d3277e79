// Attention weights that a cache's rows get (nats_cache_weights), and the eviction by them (nats_cache_evict).
#include <math.h>

#include <type_traits>

#include "nats_common.h"
#include "nats_serve.h"
#include "serve.h"
#include "softmax_terms.h"

namespace nats {

// ---- attention weights of a cache's rows ----------------------------------------------------------------------------------
//   w[c] <- decay w[c] + sum_t [c < vis_t] exp2(s q_t . k_c - L_t),   s = scale log2(e), L_t = lse_t log2(e)
// A product of queries and rows whose result is summed over the queries: with the rows as columns of a result tile a lane keeps one sum per
// row.  Few queries (a step's): the queries stay in registers and the rows of K stream, memory-bound.  Many (a prompt's): 16 or more rows
// stay and the queries stream; bound by the exponential, four cycles a piece per lane and pair, beside the same of matrix instructions.
//
// Without lse the sums over the cache are needed first.  Up to 16 queries the first pass then keeps its logits, 4 T bytes a row
// where K has 2 d or 4 d, and K is read once; beyond, writing and reading them would cost as much as K again.
constexpr float LOG2E = 1.44269504088896341f;
constexpr int CW_THREADS = 256, CW_WAVES = CW_THREADS / 64;
constexpr int CW_FEW = 64;       // queries that stay in registers
constexpr int CW_KEEP = 16;      // queries whose logits are kept
constexpr int CW_MOST_ROWS = 8192;   // of a part: a lane sums 512 of them one after the other

// 16 rows of D elements as an operand (lane l16: row, lane quarter lq: its share of every 32 or 16 columns), and the product of two
template <typename T, int D>
struct Rows16;
template <int D>
struct Rows16<bf16_t, D> {
    u32x4 x[D / 32];
    __device__ __forceinline__ void load(const bf16_t* p, int row, int last, int l16, int lq) {
        p += (size_t)min(row + l16, last) * D + 8 * lq;
#pragma unroll
        for (int i = 0; i < D / 32; ++i) x[i] = *reinterpret_cast<const u32x4*>(p + 32 * i);
    }
    __device__ __forceinline__ void load(const bf16_t* p, int l16, int lq, int pitch) {   // from LDS
#pragma unroll
        for (int i = 0; i < D / 32; ++i) x[i] = *reinterpret_cast<const u32x4*>(p + l16 * pitch + 32 * i + 8 * lq);
    }
    // with each of several (the sums side by side: an instruction does not wait for the one before)
    template <int N>
    __device__ __forceinline__ static void products(const Rows16& a, const Rows16 (&b)[N], f32x4 (&s)[N]) {
#pragma unroll
        for (int n = 0; n < N; ++n) s[n] = f32x4{0.f, 0.f, 0.f, 0.f};
#pragma unroll
        for (int i = 0; i < D / 32; ++i)
#pragma unroll
            for (int n = 0; n < N; ++n) s[n] = mfma_bf16(a.x[i], b[n].x[i], s[n]);
    }
};
template <int D>
struct Rows16<float, D> {
    float4 x[D / 16];
    __device__ __forceinline__ void load(const float* p, int row, int last, int l16, int lq) {
        p += (size_t)min(row + l16, last) * D + 4 * lq;
#pragma unroll
        for (int i = 0; i < D / 16; ++i) x[i] = ld4(p + 16 * i);
    }
    __device__ __forceinline__ void load(const float* p, int l16, int lq, int pitch) {   // from LDS
#pragma unroll
        for (int i = 0; i < D / 16; ++i) x[i] = ld4(p + l16 * pitch + 16 * i + 4 * lq);
    }
    template <int N>
    __device__ __forceinline__ static void products(const Rows16& a, const Rows16 (&b)[N], f32x4 (&s)[N]) {
#pragma unroll
        for (int n = 0; n < N; ++n) s[n] = f32x4{0.f, 0.f, 0.f, 0.f};
#pragma unroll
        for (int i = 0; i < D / 16; ++i) {
#pragma unroll
            for (int n = 0; n < N; ++n) s[n] = __builtin_amdgcn_mfma_f32_16x16x4f32(a.x[i].x, b[n].x[i].x, s[n], 0, 0, 0);
#pragma unroll
            for (int n = 0; n < N; ++n) s[n] = __builtin_amdgcn_mfma_f32_16x16x4f32(a.x[i].y, b[n].x[i].y, s[n], 0, 0, 0);
#pragma unroll
            for (int n = 0; n < N; ++n) s[n] = __builtin_amdgcn_mfma_f32_16x16x4f32(a.x[i].z, b[n].x[i].z, s[n], 0, 0, 0);
#pragma unroll
            for (int n = 0; n < N; ++n) s[n] = __builtin_amdgcn_mfma_f32_16x16x4f32(a.x[i].w, b[n].x[i].w, s[n], 0, 0, 0);
        }
    }
};

__device__ __forceinline__ int rows_of(const WeightsCall& c, int bh) { return min(max(c.cache_len[bh], 0), c.cap); }
// rows of the cache that query t of head bh sees
__device__ __forceinline__ int sees_rows(const WeightsCall& c, int bh, int t, int n) {
    if (c.vis == nullptr) return n;
    const int b = bh / c.H, h = bh % c.H;
    return min(max(c.vis[((size_t)b * (c.H / c.vis_group) + h / c.vis_group) * c.T + t], 0), n);
}
template <typename T>
__device__ __forceinline__ const T* queries(const WeightsCall& c, int bh) {
    const int b = bh / c.H, h = bh % c.H;
    return (const T*)c.q + ((size_t)b * (c.H / c.q_group) + h / c.q_group) * c.T * c.d;
}
// running maximum and sum of two parts into one
__device__ __forceinline__ void join(float& m, float& l, float m2, float l2) {
    const float top = fmaxf(m, m2), ref = top == -INFINITY ? 0.f : top;
    l = l * __builtin_amdgcn_exp2f(m - ref) + l2 * __builtin_amdgcn_exp2f(m2 - ref);
    m = top;
}

// ---- first pass without lse: maximum and sum of up to 16 NQ queries over a part of the rows; KEEP: the logits, too ----
// Result tiles have the rows of K as rows: a lane has 4 rows in a row of one query.
template <typename T, int D, int NQ, bool KEEP>
__global__ __launch_bounds__(CW_THREADS, 2) void weights_sums_kernel(WeightsCall c) {
    constexpr int KT = 2;   // tiles of rows in flight
    __shared__ float2 s_ml[CW_WAVES][NQ][16];
    const int bh = blockIdx.x, part = blockIdx.y, t0 = blockIdx.z * 16 * NQ, lane = threadIdx.x & 63, l16 = lane & 15, lq = lane >> 4;
    const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    const int n = rows_of(c, bh), lo = part * c.rows, last = min(n - lo, c.rows) - 1;
    if (last < 0) return;
    const T* K = (const T*)c.k_cache + ((size_t)bh * c.cap + lo) * D;
    Rows16<T, D> q[NQ], k[KT];
    int row = wave * 16 * KT;
#pragma unroll
    for (int i = 0; i < KT; ++i) k[i].load(K, row + 16 * i, last, l16, lq);
    int vis[NQ];
    float m[NQ], l[NQ];
#pragma unroll
    for (int x = 0; x < NQ; ++x) {
        const int t = min(t0 + 16 * x + l16, c.T - 1);
        q[x].load(queries<T>(c, bh), t0 + 16 * x, c.T - 1, l16, lq);
        vis[x] = sees_rows(c, bh, t, n) - lo;
        m[x] = -INFINITY;
        l[x] = 0.f;
    }
    const float scale2 = c.scale * LOG2E;
    for (; row <= last; row += CW_WAVES * 16 * KT) {
        f32x4 s[KT][NQ];
#pragma unroll
        for (int i = 0; i < KT; ++i) Rows16<T, D>::products(k[i], q, s[i]);
#pragma unroll
        for (int i = 0; i < KT; ++i) k[i].load(K, row + CW_WAVES * 16 * KT + 16 * i, last, l16, lq);
#pragma unroll
        for (int x = 0; x < NQ; ++x) {
            float top = m[x];
#pragma unroll
            for (int i = 0; i < KT; ++i)
#pragma unroll
                for (int j = 0; j < 4; ++j) {
                    const int r = row + 16 * i + 4 * lq + j;
                    s[i][x][j] = r <= last && r < vis[x] ? s[i][x][j] * scale2 : -INFINITY;
                    top = fmaxf(top, s[i][x][j]);
                }
            const float ref = top == -INFINITY ? 0.f : top;
            l[x] *= __builtin_amdgcn_exp2f(m[x] - ref);
            m[x] = top;
#pragma unroll
            for (int i = 0; i < KT; ++i)
#pragma unroll
                for (int j = 0; j < 4; ++j) l[x] += __builtin_amdgcn_exp2f(s[i][x][j] - ref);
            if (KEEP && l16 < c.T) {
#pragma unroll
                for (int i = 0; i < KT; ++i)   // (rows past the end within the part have their place, too)
                    if (row + 16 * i + 4 * lq <= last)
                        *reinterpret_cast<f32x4*>(c.ws + c.off_logits + ((size_t)bh * c.T + l16) * c.pitch + lo + row + 16 * i + 4 * lq) = s[i][x];
            }
        }
    }
#pragma unroll
    for (int x = 0; x < NQ; ++x) {
        join(m[x], l[x], lane_xor16(m[x], lane), lane_xor16(l[x], lane));
        join(m[x], l[x], lane_xor32(m[x], lane), lane_xor32(l[x], lane));
        if (lq == 0) s_ml[wave][x][l16] = make_float2(m[x], l[x]);
    }
    __syncthreads();
    const int t = t0 + (int)threadIdx.x;
    if (threadIdx.x >= 16 * NQ || t >= c.T) return;
    float2 r = s_ml[0][threadIdx.x / 16][threadIdx.x % 16];
#pragma unroll
    for (int w = 1; w < CW_WAVES; ++w) join(r.x, r.y, s_ml[w][threadIdx.x / 16][threadIdx.x % 16].x, s_ml[w][threadIdx.x / 16][threadIdx.x % 16].y);
    *reinterpret_cast<float2*>(c.ws + c.off_ml + (((size_t)bh * c.parts + part) * c.T + t) * 2) = r;
}

// the parts' maxima and sums into the log-sum-exp, a thread per query
__global__ __launch_bounds__(CW_THREADS) void weights_lse_kernel(WeightsCall c) {
    const int bh = blockIdx.x, t = blockIdx.y * CW_THREADS + threadIdx.x;
    if (t >= c.T) return;
    const int parts = (rows_of(c, bh) + c.rows - 1) / c.rows;
    float m = -INFINITY, l = 0.f;
    for (int p = 0; p < parts; ++p) {
        const float2 x = *reinterpret_cast<const float2*>(c.ws + c.off_ml + (((size_t)bh * c.parts + p) * c.T + t) * 2);
        join(m, l, x.x, x.y);
    }
    c.ws[c.off_lse + (size_t)bh * c.T + t] = l == 0.f ? -INFINITY : (m + log2f(l)) / LOG2E;
}

// ---- the weights from logits that were kept ----
constexpr int CW_KEPT_ROWS = 4;   // per thread
__global__ __launch_bounds__(CW_THREADS) void weights_kept_kernel(WeightsCall c) {
    const int bh = blockIdx.x, lane = threadIdx.x & 63, n = rows_of(c, bh), r0 = blockIdx.y * CW_THREADS * CW_KEPT_ROWS + threadIdx.x;
    if ((int)blockIdx.y * CW_THREADS * CW_KEPT_ROWS >= n) return;
    const float* z = c.ws + c.off_logits + (size_t)bh * c.T * c.pitch;
    float* weights = c.weights + (size_t)bh * c.cap;
    // the parts' sums of query lane % 16, a quarter of the parts per lane, by every wavefront for itself
    const int t = min(lane % CW_KEEP, c.T - 1), parts = (n + c.rows - 1) / c.rows;
    float m = -INFINITY, l = 0.f, w[CW_KEPT_ROWS], sum[CW_KEPT_ROWS];
    for (int p = lane / CW_KEEP; p < parts; p += 64 / CW_KEEP) {
        const float2 ml = *reinterpret_cast<const float2*>(c.ws + c.off_ml + (((size_t)bh * c.parts + p) * c.T + t) * 2);
        join(m, l, ml.x, ml.y);
    }
#pragma unroll
    for (int i = 0; i < CW_KEPT_ROWS; ++i) {
        w[i] = weights[min(r0 + i * CW_THREADS, n - 1)];
        sum[i] = 0.f;
    }
    join(m, l, lane_xor16(m, lane), lane_xor16(l, lane));
    join(m, l, lane_xor32(m, lane), lane_xor32(l, lane));
    const float lse = l == 0.f ? INFINITY : m + log2f(l);   // (a query that sees nothing: all its logits are -inf)
    const int vis = sees_rows(c, bh, t, n);
#pragma unroll 4
    for (int q = 0; q < c.T; ++q) {
        const float L = __shfl(lse, q);
        const int seen = __shfl(vis, q);
#pragma unroll
        for (int i = 0; i < CW_KEPT_ROWS; ++i) {
            const int r = min(r0 + i * CW_THREADS, n - 1);
            const float p = __builtin_amdgcn_exp2f(z[(size_t)q * c.pitch + r] - L);
            sum[i] += r < seen ? p : 0.f;   // (L may be NaN: in a row that the query does not see, p is then one, too)
        }
    }
#pragma unroll
    for (int i = 0; i < CW_KEPT_ROWS; ++i)
        if (r0 + i * CW_THREADS < n) weights[r0 + i * CW_THREADS] = c.decay * w[i] + sum[i];
}

// lse in powers of two and the number of visible rows of queries t .. t + 3 (those beyond T see nothing, nor do those with lse -inf)
__device__ __forceinline__ void query_bounds(const WeightsCall& c, const float* lse, int bh, int t, int n, f32x4& L, int (&vis)[4]) {
#pragma unroll
    for (int j = 0; j < 4; ++j) {
        const int at = min(t + j, c.T - 1);
        const float x = lse[at];
        L[j] = x * LOG2E;
        vis[j] = t + j < c.T && x != -INFINITY ? sees_rows(c, bh, at, n) : 0;
    }
}

// ---- few queries: they stay, the rows stream ----
template <typename T, int D, int NQ>
__global__ __launch_bounds__(CW_THREADS, 2) void weights_few_kernel(WeightsCall c) {
    constexpr int KT = sizeof(T) == 4 && D == 128 && NQ == 4 ? 1 : 2;   // (two would not fit into the registers)
    const int bh = blockIdx.x, part = blockIdx.y, lane = threadIdx.x & 63, l16 = lane & 15, lq = lane >> 4;
    const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    const int n = rows_of(c, bh), lo = part * c.rows, last = min(n - lo, c.rows) - 1;
    if (last < 0) return;
    const T* K = (const T*)c.k_cache + ((size_t)bh * c.cap + lo) * D;
    const float* lse = (c.lse != nullptr ? c.lse : c.ws + c.off_lse) + (size_t)bh * c.T;
    float* weights = c.weights + (size_t)bh * c.cap + lo;
    Rows16<T, D> q[NQ], k[KT];
    int row = wave * 16 * KT;
#pragma unroll
    for (int i = 0; i < KT; ++i) k[i].load(K, row + 16 * i, last, l16, lq);
    f32x4 L[NQ];
    int vis[NQ][4];
#pragma unroll
    for (int x = 0; x < NQ; ++x) {
        q[x].load(queries<T>(c, bh), 16 * x, c.T - 1, l16, lq);
        query_bounds(c, lse, bh, 16 * x + 4 * lq, n, L[x], vis[x]);
    }
    const float scale2 = c.scale * LOG2E;
    for (; row <= last; row += CW_WAVES * 16 * KT) {
        float sum[KT], w[KT];
        f32x4 s[NQ][KT];
#pragma unroll
        for (int i = 0; i < KT; ++i) {
            w[i] = weights[min(row + 16 * i + l16, last)];
        }
#pragma unroll
        for (int x = 0; x < NQ; ++x) Rows16<T, D>::products(q[x], k, s[x]);
#pragma unroll
        for (int i = 0; i < KT; ++i) k[i].load(K, row + CW_WAVES * 16 * KT + 16 * i, last, l16, lq);
#pragma unroll
        for (int i = 0; i < KT; ++i) {
            const int r = row + 16 * i + l16;
            sum[i] = 0.f;
#pragma unroll
            for (int x = 0; x < NQ; ++x)
#pragma unroll
                for (int j = 0; j < 4; ++j) {
                    const float p = __builtin_amdgcn_exp2f(s[x][i][j] * scale2 - L[x][j]);
                    sum[i] += lo + r < vis[x][j] ? p : 0.f;
                }
            sum[i] += lane_xor16(sum[i], lane);
            sum[i] += lane_xor32(sum[i], lane);
            if (lq == 0 && r <= last) weights[r] = c.decay * w[i] + sum[i];
        }
    }
}

// ---- many queries: 16 KT rows stay in every wavefront's registers, the queries stream ----
// WK of the block's wavefronts take rows side by side, the others other queries.  The queries come through LDS, 16 KB at a time and two steps
// deep: read from memory by the wavefronts as operands, 16 rows apart from lane to lane, every lane is an access of its own to the CU's
// cache, and their number (57 per instruction; 16 where four lanes read 64 bytes in a row) bound this kernel: 53 us against
// the 34 of this form (a prompt of 8192, 32 caches of 410 rows).  Bounds of the block's queries (at most CW_CHUNK) go through LDS, too; the steps
// before the first query that sees a row of the block's are left out.
constexpr int CW_CHUNK = 1024;
constexpr int CW_SPLITS = 64;   // blocks that share a row's queries in one launch (each writes a sum per row)
template <typename T, int D>
constexpr int many_tiles() { return sizeof(T) == 2 || D == 64 ? 4 : 2; }

template <typename T, int D, int WK>
__global__ __launch_bounds__(CW_THREADS, 2) void weights_many_kernel(WeightsCall c) {
    constexpr int KT = many_tiles<T, D>(), WQ = CW_WAVES / WK, ROWS = 16 * KT * WK;
    constexpr int QS = 16384 / (D * (int)sizeof(T));              // queries of a step: 32, 64 or 128
    constexpr int LANES = D * (int)sizeof(T) / 16;                // 16-byte words of a row
    constexpr int PITCH = D + LDS_PAD * 2 / (int)sizeof(T);       // elements
    constexpr int WORDS = 16384 / 16 / CW_THREADS;                // per thread and step
    __shared__ __attribute__((aligned(16))) T s_q[2][QS * PITCH];
    __shared__ float s_L[CW_CHUNK], s_sum[WQ][ROWS];
    __shared__ int s_vis[CW_CHUNK], s_first;
    const int bh = blockIdx.x, split = blockIdx.z, tid = threadIdx.x, lane = tid & 63, l16 = lane & 15, lq = lane >> 4;
    const int wave = __builtin_amdgcn_readfirstlane(tid >> 6), wk = wave % WK, wq = wave / WK;
    const int n = rows_of(c, bh), block0 = blockIdx.y * ROWS, r0 = block0 + wk * 16 * KT;
    if (block0 >= n) return;
    const int t0 = c.t_lo + split * c.chunk, here = min(c.chunk, c.t_hi - t0);
    const T* Q = queries<T>(c, bh) + (size_t)t0 * D;
    const float* lse = (c.lse != nullptr ? c.lse : c.ws + c.off_lse) + (size_t)bh * c.T + t0;
    float* sums = c.ws + c.off_sums + ((size_t)split * c.B * c.H + bh) * c.cap;
    if (tid == 0) s_first = here;
    __syncthreads();
    int first = here;
    for (int t = tid; t < (here + QS - 1) / QS * QS; t += CW_THREADS) {
        const int at = min(t, here - 1);
        const float x = lse[at];
        // queries that are not there, or whose lse is -inf, see nothing
        const int vis = t < here && x != -INFINITY ? sees_rows(c, bh, t0 + at, n) : 0;
        s_L[t] = x * LOG2E;
        s_vis[t] = vis;
        if (vis > block0) first = min(first, t);
    }
    first = wave_extreme_i32<false>(first);
    if (lane == 0) atomicMin(&s_first, first);
    __syncthreads();
    first = s_first / QS * QS;
    if (first >= here) {   // (uniform)
        if (tid < ROWS && block0 + tid < n) sums[block0 + tid] = 0.f;
        return;
    }
    float sum[KT];
#pragma unroll
    for (int i = 0; i < KT; ++i) sum[i] = 0.f;
    const float scale2 = c.scale * LOG2E;
    Rows16<T, D> k[KT];
    u32x4 word[WORDS];
    auto fetch = [&](int t) {
#pragma unroll
        for (int i = 0; i < WORDS; ++i) {
            const int row = min(t + (tid + i * CW_THREADS) / LANES, here - 1);
            word[i] = *reinterpret_cast<const u32x4*>(reinterpret_cast<const char*>(Q + (size_t)row * D) + (tid % LANES) * 16);
        }
    };
    auto put = [&](int at) {
#pragma unroll
        for (int i = 0; i < WORDS; ++i)
            *reinterpret_cast<u32x4*>(reinterpret_cast<char*>(&s_q[at][(tid + i * CW_THREADS) / LANES * PITCH]) + (tid % LANES) * 16) = word[i];
    };
    static_assert(CW_THREADS % LANES == 0 && QS % (16 * WQ) == 0, "a thread's words lie in one column, a step has a tile for every wavefront");
    fetch(first);
#pragma unroll
    for (int i = 0; i < KT; ++i) k[i].load((const T*)c.k_cache + (size_t)bh * c.cap * D, r0 + 16 * i, n - 1, l16, lq);
    put(0);
    __syncthreads();
    int at = 0;
    for (int t = first; t < here; t += QS, at ^= 1) {
        fetch(t + QS);   // (past the end: the last query)
        if (r0 < n) {
#pragma unroll
            for (int x = 0; x < QS / (16 * WQ); ++x) {
                const int u = 16 * (x * WQ + wq);
                const f32x4 L = *reinterpret_cast<const f32x4*>(&s_L[t + u + 4 * lq]);
                const int4 vis = *reinterpret_cast<const int4*>(&s_vis[t + u + 4 * lq]);
                const int least = min(min(vis.x, vis.y), min(vis.z, vis.w)), most = max(max(vis.x, vis.y), max(vis.z, vis.w));
                if (!__any(most > r0)) continue;
                Rows16<T, D> q;
                q.load(&s_q[at][u * PITCH], l16, lq, PITCH);
                f32x4 s[KT];
                Rows16<T, D>::products(q, k, s);
                if (__all(least >= r0 + 16 * KT)) {
#pragma unroll
                    for (int i = 0; i < KT; ++i)
#pragma unroll
                        for (int j = 0; j < 4; ++j) sum[i] += __builtin_amdgcn_exp2f(s[i][j] * scale2 - L[j]);
                } else {
                    const int v[4] = {vis.x, vis.y, vis.z, vis.w};
#pragma unroll
                    for (int i = 0; i < KT; ++i)
#pragma unroll
                        for (int j = 0; j < 4; ++j) {
                            const float p = __builtin_amdgcn_exp2f(s[i][j] * scale2 - L[j]);
                            sum[i] += r0 + 16 * i + l16 < v[j] ? p : 0.f;
                        }
                }
            }
        }
        put(at ^ 1);     // (its queries were used up before the barrier)
        __syncthreads();
    }
#pragma unroll
    for (int i = 0; i < KT; ++i) {
        sum[i] += lane_xor16(sum[i], lane);
        sum[i] += lane_xor32(sum[i], lane);
        if (lq == 0) s_sum[wq][wk * 16 * KT + 16 * i + l16] = sum[i];
    }
    __syncthreads();
    if (tid >= ROWS || block0 + tid >= n) return;
    float x = s_sum[0][tid];
#pragma unroll
    for (int w = 1; w < WQ; ++w) x += s_sum[w][tid];
    sums[block0 + tid] = x;
}

// the splits' sums onto the weights, in order; decay 1 for all but a call's first launch
__global__ __launch_bounds__(CW_THREADS) void weights_join_kernel(WeightsCall c, int splits, float decay) {
    const int bh = blockIdx.x, r = blockIdx.y * CW_THREADS + threadIdx.x;
    if (r >= rows_of(c, bh)) return;
    float x = 0.f;
#pragma unroll 8
    for (int s = 0; s < splits; ++s) x += c.ws[c.off_sums + ((size_t)s * c.B * c.H + bh) * c.cap + r];
    float* w = c.weights + (size_t)bh * c.cap + r;
    *w = decay * *w + x;
}

// Rows of a part: 256, or 128 where that leaves less than two parts per CU (us with parts of 128 / 256 / 512 / 1024 rows: 1024 caches of 64 ..
// 2048 rows, one query 74 / 69 / 69 / 72; 140 of up to 2778, 64 queries 34 / 25 / 24 / 25; 42 of up to 17187, 10 queries 21 / 20 / 24 / 27).
size_t weights_workspace(WeightsCall& c, bool lse_given) {
    const long long heads = (long long)c.B * c.H;
    c.rows = heads * ((c.cap + 255) / 256) < 512 ? 128 : 256;
    // Beyond 64 queries their groups of 64 are blocks, too, and load those queries, start a softmax and write a maximum and a sum per query
    // for every part: larger parts, as long as eight blocks per CU are left (us of a call without lse, parts of 256 rows / these: 64 caches of
    // 8192 rows, 8192 queries 4868 / 2882; 32 of 410, 8192 queries 234 / 140; 4 of 32768, 1024 queries 200 / 135, 156 with twice the
    // blocks; 1024 of 2048, 128 queries 399 / 326; 140 of 2778 in fp32, 100 queries 275 / 263).
    auto blocks_of_sums = [&] { return heads * ((c.cap + c.rows - 1) / c.rows) * ((c.T + 63) / 64); };
    while (c.T > CW_FEW && c.rows < min(c.cap, CW_MOST_ROWS) && blocks_of_sums() > 2048) c.rows *= 2;
    c.parts = (c.cap + c.rows - 1) / c.rows;
    size_t at = 0;
    if (!lse_given) {
        c.off_ml = at;
        at += (size_t)heads * c.parts * c.T * 2;
        at = align_up(at, 4);
        if (c.T <= CW_KEEP) {
            c.pitch = (c.cap + 31) / 32 * 32;
            c.off_logits = at;
            at += (size_t)heads * c.T * c.pitch;
        } else {
            c.off_lse = at;
            at += (size_t)heads * c.T;
        }
    }
    if (c.T > CW_FEW) {
        // rows of a block: those of up to four wavefronts, as the caches have them, for every row of the block's shares the reading of its
        // queries; queries of a block: as many as leave four blocks per CU.  Fewer rows, too, where that leaves the chip idle
        // (us of the kernel with 4 / 2 / 1 wavefronts on the rows: 32 caches of 410 rows, 8192 queries, 512 at a time 34 / 37 / 46;
        // 6 caches of 105 rows in fp32, 701 queries, 128 at a time 12 / 8 / 6).
        const int tiles = 16 * (c.dtype == NATS_BF16 || c.d == 64 ? 4 : 2), least = c.dtype == NATS_F32 && c.d == 128 ? 2 : 1;
        auto blocks = [&] { return heads * ((c.cap + c.row_waves * tiles - 1) / (c.row_waves * tiles)) * ((c.T + c.chunk - 1) / c.chunk); };
        c.row_waves = c.cap <= tiles ? least : c.cap <= 2 * tiles ? 2 : 4;
        c.chunk = CW_CHUNK;
        while (c.chunk > 128 && blocks() < 1024) c.chunk /= 2;
        while (c.row_waves > least && blocks() < 256) c.row_waves /= 2;
        if (blocks() < 256) c.chunk = 64;
        c.splits = min((c.T + c.chunk - 1) / c.chunk, CW_SPLITS);
        c.off_sums = at;
        at += (size_t)c.splits * heads * c.cap;
    }
    return at;
}

template <typename T, int D>
static void run_sums(const WeightsCall& c, hipStream_t st) {
    const int heads = c.B * c.H;
    const dim3 block(CW_THREADS);
    if (c.T <= CW_KEEP) {
        hipLaunchKernelGGL((weights_sums_kernel<T, D, 1, true>), dim3(heads, c.parts), block, 0, st, c);
    } else if (c.T <= 32) {
        hipLaunchKernelGGL((weights_sums_kernel<T, D, 2, false>), dim3(heads, c.parts), block, 0, st, c);
    } else {
        hipLaunchKernelGGL((weights_sums_kernel<T, D, 4, false>), dim3(heads, c.parts, (c.T + 63) / 64), block, 0, st, c);
    }
}

template <typename T, int D>
static nats_status run_weights(const WeightsCall& c, hipStream_t st) {
    const int heads = c.B * c.H;
    const dim3 block(CW_THREADS), rows(heads, (c.cap + CW_THREADS - 1) / CW_THREADS);
    if (c.lse == nullptr) {
        {
            ProfScope ps("weights_sums", st);
            run_sums<T, D>(c, st);
        }
        if (c.T <= CW_KEEP) {
            ProfScope ps("weights_kept", st);
            constexpr int ROWS = CW_THREADS * CW_KEPT_ROWS;
            hipLaunchKernelGGL(weights_kept_kernel, dim3(heads, (c.cap + ROWS - 1) / ROWS), block, 0, st, c);
            return check_launch("cache_weights");
        }
        ProfScope ps("weights_lse", st);
        hipLaunchKernelGGL(weights_lse_kernel, dim3(heads, (c.T + CW_THREADS - 1) / CW_THREADS), block, 0, st, c);
    }
    if (c.T <= CW_FEW) {
        ProfScope ps("weights_few", st);
        if (c.T <= 16) hipLaunchKernelGGL((weights_few_kernel<T, D, 1>), dim3(heads, c.parts), block, 0, st, c);
        else if (c.T <= 32) hipLaunchKernelGGL((weights_few_kernel<T, D, 2>), dim3(heads, c.parts), block, 0, st, c);
        else hipLaunchKernelGGL((weights_few_kernel<T, D, 4>), dim3(heads, c.parts), block, 0, st, c);
        return check_launch("cache_weights");
    }
    constexpr int ROWS = 16 * many_tiles<T, D>();
    for (int t = 0; t < c.T; t += c.splits * c.chunk) {
        WeightsCall x = c;
        x.t_lo = t;
        x.t_hi = min(c.T - t, c.splits * c.chunk) + t;
        const int splits = (x.t_hi - x.t_lo + c.chunk - 1) / c.chunk;
        {
            ProfScope ps("weights_many", st);
            const dim3 grid(heads, (c.cap + c.row_waves * ROWS - 1) / (c.row_waves * ROWS), splits);
            if constexpr (ROWS > 32)   // (16 KB of longer rows are too few queries for four wavefronts)
                if (c.row_waves == 1) hipLaunchKernelGGL((weights_many_kernel<T, D, 1>), grid, block, 0, st, x);
            if (c.row_waves == 2) hipLaunchKernelGGL((weights_many_kernel<T, D, 2>), grid, block, 0, st, x);
            if (c.row_waves == 4) hipLaunchKernelGGL((weights_many_kernel<T, D, 4>), grid, block, 0, st, x);
        }
        ProfScope ps("weights_join", st);
        hipLaunchKernelGGL(weights_join_kernel, rows, block, 0, st, x, splits, t == 0 ? c.decay : 1.f);
    }
    return check_launch("cache_weights");
}

nats_status launch_cache_weights(const WeightsCall& c, hipStream_t st) {
    if (c.dtype == NATS_F32) return c.d == 64 ? run_weights<float, 64>(c, st) : run_weights<float, 128>(c, st);
    return c.d == 64 ? run_weights<bf16_t, 64>(c, st) : run_weights<bf16_t, 128>(c, st);
}

// ---- eviction: which rows stay ---------------------------------------------------------------------------------------------
// A number that orders as the weights do (a NaN below all, -0 as 0); 0 is left for what is not to be chosen
__device__ __forceinline__ uint32_t weight_key(float w) {
    if (w != w) return 1;
    const uint32_t u = __float_as_uint(w + 0.f);
    return u & 0x80000000u ? ~u : u | 0x80000000u;
}

// One block per cache.  The weight of the last row that stays is found by halving the range of keys 10 bits at a time: counts of the rows in
// 1024 parts of the range that is left, which at first is that from the least key to the largest (with fixed digits most weights of an
// attention share a dozen values of the first one, and lanes that add to one address go one after the other; for equal weights the counts are kept
// in four copies, a lane's by its number).  As soon as a part stays as a whole its lower end is the border.  Then the rows above the
// border, and the lowest of those equal to it, are numbered in order and their weights moved, behind them the last `recent` ones.  A wavefront
// has up to PER x 64 rows in a row, as many as spread the cache over all wavefronts, so that ranks inside it are counts of ballot
// bits.  Up to THREADS x PER rows the keys stay in registers throughout; longer caches are gone through in such steps, once per 10 bits and
// once for the numbers (a step's rows are read before any of them is written, and no row's new place is behind its old one).  With few caches
// it is bound by its instructions, on the few CUs that have one.
constexpr int SELECT_BINS = 1024;
template <int THREADS>
struct SelectLds {
    int4 hist[SELECT_BINS];   // copy lane % 4 of every count
    uint32_t least[THREADS / 64], most[THREADS / 64];
    int sums[THREADS / 64], ties[THREADS / 64], stay[THREADS / 64], digit, rest, agree;
};

// false: the cache is within the budget, no row moves
template <int THREADS, int PER>
__device__ __forceinline__ bool evict_select(const EvictCall& c, int bh, SelectLds<THREADS>& s) {
    constexpr int WAVES = THREADS / 64, GROUP = 2, BINS = SELECT_BINS / THREADS;   // GROUP: rows of a lane behind one branch
    const int tid = threadIdx.x, lane = tid & 63, wave = __builtin_amdgcn_readfirstlane(tid >> 6);
    const int n = __builtin_amdgcn_readfirstlane(min(max(c.cache_len[bh], 0), c.cap));
    float* w = c.weights + (size_t)bh * c.cap;
    int32_t* kept = c.kept + (size_t)bh * c.keep;
    if (n <= c.keep) {
        for (int r = tid; r < c.keep; r += THREADS) kept[r] = r < n ? r : -1;
        return false;
    }
    const int m = n - c.recent;                       // the rows to choose from
    const int chosen = c.keep - c.recent;             // ... and how many of them stay
    const bool one = m <= THREADS * PER;
    const int per = one ? (m + THREADS * GROUP - 1) / (THREADS * GROUP) * GROUP : PER, step = THREADS * per;   // rows of a lane and of the block
    auto rows = [&](auto&& f) {   // f(i) for the lane's rows
#pragma unroll
        for (int g = 0; g < PER; g += GROUP)
            if (g < per) {
#pragma unroll
                for (int i = 0; i < GROUP; ++i) f(g + i);
            }
    };
    float x[PER];
    uint32_t key[PER];
    auto load = [&](int r0) {
        const int first = r0 + wave * 64 * per;       // uniform
        rows([&](int i) { x[i] = w[(uint32_t)min(first + lane + 64 * i, n - 1)]; });
        rows([&](int i) { key[i] = first + lane + 64 * i < m ? weight_key(x[i]) : 0; });
    };
    auto before = [&](uint64_t b) { return (int)__builtin_amdgcn_mbcnt_hi((uint32_t)(b >> 32), __builtin_amdgcn_mbcnt_lo((uint32_t)b, 0)); };
    // the keys of the rows that may be the last to stay are base .. base + width, and `rest` of these stay (a key of 0 less base is above
    // width: no key and no end of a range passes 32 bits)
    uint32_t base = 1, width = 0xff800000u - 1;
    int rest = chosen, agree = 0;
    if (chosen > 0) {
#pragma unroll
        for (int i = 0; i < BINS; ++i) s.hist[tid * BINS + i] = make_int4(0, 0, 0, 0);
        if (one) {
            load(0);
            uint32_t least = ~0u, most = 0;
            rows([&](int i) {
                least = min(least, key[i] - 1);       // (0 becomes the largest)
                most = max(most, key[i]);
            });
            least = (uint32_t)wave_extreme_i32<false>((int)(least ^ 0x80000000u)) ^ 0x80000000u;
            most = (uint32_t)wave_extreme_i32<true>((int)(most ^ 0x80000000u)) ^ 0x80000000u;
            if (lane == 0) {
                s.least[wave] = least;
                s.most[wave] = most;
            }
            __syncthreads();
            least = s.least[0];
            most = s.most[0];
#pragma unroll
            for (int v = 1; v < WAVES; ++v) {
                least = min(least, s.least[v]);
                most = max(most, s.most[v]);
            }
            base = least + 1;
            width = most - base;
        } else {
            __syncthreads();
        }
        for (int shift = max(22 - __clz((int)width), 0);; shift = max(shift - 10, 0)) {   // width >> shift < 1024
            for (int r0 = 0; r0 < m; r0 += step) {
                if (!one) load(r0);
                rows([&](int i) {
                    const uint32_t k = key[i] - base;
                    if (k <= width) atomicAdd(reinterpret_cast<int*>(&s.hist[k >> shift]) + (lane & 3), 1);
                });
            }
            __syncthreads();
            // a thread: BINS parts of the range, from the top
            int h[BINS], sum = 0;
#pragma unroll
            for (int i = 0; i < BINS; ++i) {
                int4& at = s.hist[SELECT_BINS - 1 - tid * BINS - i];
                sum += h[i] = at.x + at.y + at.z + at.w;
                at = make_int4(0, 0, 0, 0);
            }
            const int upto = wave_inclusive_scan_i32(sum);
            if (lane == 63) s.sums[wave] = upto;
            __syncthreads();
            int more = upto - sum;
#pragma unroll
            for (int v = 0; v < WAVES; ++v) more += v < wave ? s.sums[v] : 0;
            if (more < rest && rest <= more + sum) {
#pragma unroll
                for (int i = 0; i < BINS; ++i) {
                    if (more < rest && rest <= more + h[i]) {
                        s.digit = SELECT_BINS - 1 - tid * BINS - i;
                        s.rest = rest - more;
                        s.agree = h[i];
                    }
                    more += h[i];
                }
            }
            __syncthreads();
            base += (uint32_t)s.digit << shift;
            width = (1u << shift) - 1;
            rest = s.rest;
            agree = s.agree;
            if (shift == 0 || agree == rest) break;
        }
    }
    // rows with a key of `base` and more stay, and if these are too many, `rest` of those equal to it
    int done = 0, equal = 0;   // rows that stay, and rows equal to `base`, of the steps before
    for (int r0 = 0; chosen > 0 && r0 < m; r0 += step) {
        if (!one) load(r0);
        if (agree > rest) {
            int n_ties = 0;
            rows([&](int i) { n_ties += __popcll(__ballot(key[i] == base)); });
            if (lane == 0) s.ties[wave] = n_ties;
            __syncthreads();
            int rank = equal;
#pragma unroll
            for (int v = 0; v < WAVES; ++v) {
                if (v < wave) rank += s.ties[v];
                equal += s.ties[v];
            }
            rows([&](int i) {
                const uint64_t b = __ballot(key[i] == base);
                if (b != 0) {   // (uniform)
                    if (key[i] == base && rank + before(b) >= rest) key[i] = 0;
                    rank += __popcll(b);
                }
            });
        }
        int n_stay = 0;
        rows([&](int i) { n_stay += __popcll(__ballot(key[i] >= base)); });
        if (lane == 0) s.stay[wave] = n_stay;
        __syncthreads();   // the step's weights are in registers: a key was made of each
        int at = done;
#pragma unroll
        for (int v = 0; v < WAVES; ++v) {
            if (v < wave) at += s.stay[v];
            done += s.stay[v];
        }
        const int mine = r0 + wave * 64 * per + lane;
        rows([&](int i) {
            const bool stay = key[i] >= base;
            const uint64_t b = __ballot(stay);
            if (stay) {
                const uint32_t to = (uint32_t)(at + before(b));
                w[to] = x[i];
                kept[to] = mine + 64 * i;
            }
            at += __popcll(b);
        });
        if (!one) __syncthreads();   // s.ties and s.stay have been read
    }
    // the last rows, from m on to `chosen` on
    constexpr int TAIL = 4;   // per thread and step
    for (int i0 = 0; i0 < c.recent; i0 += THREADS * TAIL) {
        float y[TAIL];
#pragma unroll
        for (int j = 0; j < TAIL; ++j) y[j] = w[(uint32_t)min(m + i0 + j * THREADS + tid, n - 1)];
#pragma unroll
        for (int j = 0; j < TAIL; ++j) asm volatile("" : "+v"(y[j]));
        __syncthreads();   // (the chosen rows' weights were read before, and so were this step's)
#pragma unroll
        for (int j = 0; j < TAIL; ++j) {
            const int i = i0 + j * THREADS + tid;
            if (i < c.recent) {
                w[chosen + i] = y[j];
                kept[chosen + i] = m + i;
            }
        }
    }
    if (c.clear) {
        __syncthreads();   // the last rows' weights have been read
        for (int r = c.keep + tid; r < n; r += THREADS) w[r] = 0.f;
    }
    if (tid == 0) c.cache_len[bh] = c.keep;
    return true;
}

template <int THREADS, int PER>
__global__ __launch_bounds__(THREADS) void evict_select_kernel(EvictCall c) {
    __shared__ SelectLds<THREADS> s;
    evict_select<THREADS, PER>(c, blockIdx.x, s);
}

// ---- eviction: the rows move ---------------------------------------------------------------------------------------------------
// A block per cache, K or V, and slice of SLICE bytes of the rows, its rows in order.  Row r comes from kept[r] >= r, and kept rises: what a
// step reads lies at or behind the rows it writes, so a step's rows are all read before any of them is written (the barrier), and the next
// step's, which lie behind all that this one writes, are on their way meanwhile.
constexpr int MV_WORDS = 8;   // 16-byte words per thread and step
template <int SLICE, int THREADS>
__device__ __forceinline__ void evict_move_rows(const int32_t* kept, int keep, char* rows, int row_bytes) {
    constexpr int LANES = SLICE / 16, PER_WORD = THREADS / LANES, STEP = PER_WORD * MV_WORDS;   // rows
    const int tid = threadIdx.x, mine = tid / LANES;
    char* base = rows + (tid % LANES) * 16;
    u32x4 now[MV_WORDS], next[MV_WORDS];
    int src[MV_WORDS], src_next[MV_WORDS];
    auto sources = [&](int r0, int (&s)[MV_WORDS]) {
#pragma unroll
        for (int i = 0; i < MV_WORDS; ++i) {
            const int r = r0 + mine + i * PER_WORD;
            s[i] = kept[min(r, keep - 1)];
            s[i] = r < keep && s[i] > r ? s[i] : -1;   // (a row that stays where it is is not touched)
        }
    };
    auto fetch = [&](const int (&s)[MV_WORDS], u32x4 (&x)[MV_WORDS]) {   // (whole lines, read once and written once, go past the caches: 1024 caches 179 us against 191, 186 with the loads alone.  Parts of a
    // line do not: 16 caches in slices of 32 bytes 116 us against 41)
#pragma unroll
        for (int i = 0; i < MV_WORDS; ++i) {
            x[i] = u32x4{0, 0, 0, 0};
            const u32x4* const from = reinterpret_cast<const u32x4*>(base + (size_t)max(s[i], 0) * row_bytes);
            if (s[i] >= 0) {
                if constexpr (SLICE >= 128) x[i] = __builtin_nontemporal_load(from);
                else x[i] = *from;
            }
        }
    };
    sources(0, src);
    fetch(src, now);
    sources(STEP, src_next);
    for (int r0 = 0; r0 < keep; r0 += STEP) {
        fetch(src_next, next);
#pragma unroll
        for (int i = 0; i < MV_WORDS; ++i) asm volatile("" : "+v"(now[i]));   // they are here
        __syncthreads();
#pragma unroll
        for (int i = 0; i < MV_WORDS; ++i) {
            u32x4* const to = reinterpret_cast<u32x4*>(base + (size_t)(r0 + mine + i * PER_WORD) * row_bytes);
            if (src[i] >= 0) {
                if constexpr (SLICE >= 128) __builtin_nontemporal_store(now[i], to);
                else *to = now[i];
            }
            now[i] = next[i];
            src[i] = src_next[i];
        }
        sources(r0 + 2 * STEP, src_next);
    }
}

template <int SLICE, int THREADS>
__global__ __launch_bounds__(THREADS) void evict_move_kernel(EvictCall c, int row_bytes) {
    // blocks go to the eight XCDs in turn: the slices of an array to the same one, whose L2 then has the lines that they share
    const int slices = row_bytes / SLICE, turn = blockIdx.x / 8, slice = turn % slices, of = turn / slices * 8 + blockIdx.x % 8;
    const int bh = of / 2, array = of % 2;
    if (bh >= c.B * c.H) return;
    evict_move_rows<SLICE, THREADS>(c.kept + (size_t)bh * c.keep, c.keep,
                                    (char*)(array == 0 ? c.k_cache : c.v_cache) + (size_t)bh * c.cap * row_bytes + slice * SLICE, row_bytes);
}

// Both by one block per cache: with two caches per CU and more one's selection hides behind another's rows (us in one launch / in two: 2048
// caches of 2000 .. 4096 rows to 1000, d 128 414 / 421; 1024 of 700 .. 2048 to 1024 185 / 184; 512 of 1000 .. 4096 to 2048, d 64 88 / 91;
// but 256 of 700 .. 2048 to 1024 58 / 51: too few to hide anything), and where there is little to move a launch is most of the time.
template <int THREADS, int PER, int ROW>
__global__ __launch_bounds__(THREADS, 4) void evict_kernel(EvictCall c) {
    __shared__ SelectLds<THREADS> s;
    const int bh = blockIdx.x;
    if (!evict_select<THREADS, PER>(c, bh, s)) return;
    __syncthreads();   // `kept` is there
    const size_t at = (size_t)bh * c.cap * ROW;
    evict_move_rows<ROW, THREADS>(c.kept + (size_t)bh * c.keep, c.keep, (char*)c.k_cache + at, ROW);
    evict_move_rows<ROW, THREADS>(c.kept + (size_t)bh * c.keep, c.keep, (char*)c.v_cache + at, ROW);
}

nats_status launch_cache_evict(const EvictCall& c, hipStream_t st) {
    using std::integral_constant;
    const int heads = c.B * c.H, row_bytes = c.d * (c.dtype == NATS_F32 ? 4 : 2);
    if (c.cap <= 4096 && (heads >= 512 || (long long)c.keep * row_bytes <= 128 << 10)) {
        ProfScope ps("evict", st);
        auto run = [&](auto per, auto row) {
            hipLaunchKernelGGL((evict_kernel<256, decltype(per)::value, decltype(row)::value>), dim3(heads), dim3(256), 0, st, c);
        };
        auto rows = [&](auto per) {
            if (row_bytes == 128) run(per, integral_constant<int, 128>{});
            else if (row_bytes == 256) run(per, integral_constant<int, 256>{});
            else run(per, integral_constant<int, 512>{});
        };
        if (c.cap <= 1024) rows(integral_constant<int, 4>{});
        else rows(integral_constant<int, 16>{});
        return check_launch("cache_evict");
    }
    {
        ProfScope ps("evict_select", st);
        if (c.cap <= 4096) hipLaunchKernelGGL((evict_select_kernel<256, 16>), dim3(heads), dim3(256), 0, st, c);
        else hipLaunchKernelGGL((evict_select_kernel<1024, 32>), dim3(heads), dim3(1024), 0, st, c);
    }
    ProfScope ps("evict_move", st);
    // slices as wide as leave two blocks per CU; where even 64 bytes do not, blocks of 1024 threads, and 32 bytes below one (16 caches of
    // 32000 rows to 8192: 35 us, 41 with 64 bytes, 47 with 256 threads)
    auto move = [&](auto slice, auto threads) {
        constexpr int SLICE = decltype(slice)::value, THREADS = decltype(threads)::value;
        hipLaunchKernelGGL((evict_move_kernel<SLICE, THREADS>), dim3((2 * heads + 7) / 8 * 8 * (row_bytes / SLICE)), dim3(THREADS), 0, st, c, row_bytes);
    };
    const int bytes = heads * 2 * row_bytes;   // of a row of all caches, K and V
    if (row_bytes >= 256 && bytes >= 512 * 256) move(integral_constant<int, 256>{}, integral_constant<int, 256>{});
    else if (bytes >= 512 * 128) move(integral_constant<int, 128>{}, integral_constant<int, 256>{});
    else if (bytes >= 512 * 64) move(integral_constant<int, 64>{}, integral_constant<int, 256>{});
    else if (bytes >= 256 * 64) move(integral_constant<int, 64>{}, integral_constant<int, 1024>{});
    else move(integral_constant<int, 32>{}, integral_constant<int, 1024>{});
    return check_launch("cache_evict");
}

}  // namespace nats

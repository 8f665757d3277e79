// Attention weights that a cache's rows get (nats_cache_weights), and the eviction by them (nats_cache_evict).
#include <math.h>

#include "nats_common.h"
#include "nats_serve.h"
#include "serve.h"

namespace nats {

// rows of the cache that query t of head bh sees
__device__ __forceinline__ int sees_rows(const WeightsCall& c, int bh, int t, int n) {
    if (c.vis == nullptr) return n;
    const int b = bh / c.H, h = bh % c.H;
    return min(max(c.vis[((size_t)b * (c.H / c.vis_group) + h / c.vis_group) * c.T + t], 0), n);
}
template <typename T>
__device__ __forceinline__ const T* query(const WeightsCall& c, int bh, int t) {
    const int b = bh / c.H, h = bh % c.H;
    return (const T*)c.q + (((size_t)b * (c.H / c.q_group) + h / c.q_group) * c.T + t) * c.d;
}

// ---- log-sum-exp of the rows a query sees: a block per query ----
constexpr int CW_THREADS = 256;
template <typename T, int D>
__global__ __launch_bounds__(CW_THREADS) void weights_lse_kernel(WeightsCall c) {
    __shared__ float s_q[D], s_m[4], s_l[4];
    const int t = blockIdx.x, bh = blockIdx.y, tid = threadIdx.x;
    const int n = min(max(c.cache_len[bh], 0), c.cap), vis = sees_rows(c, bh, t, n);
    if (tid < D) s_q[tid] = to_float(query<T>(c, bh, t)[tid]) * c.scale;
    __syncthreads();
    const T* K = (const T*)c.k_cache + (size_t)bh * c.cap * D;
    float m = -INFINITY, l = 0.f;
    for (int r = tid; r < vis; r += CW_THREADS) {
        float x = 0.f;
        for (int e = 0; e < D; ++e) x += s_q[e] * to_float(K[(size_t)r * D + e]);
        const float top = fmaxf(m, x), ref = top == -INFINITY ? 0.f : top;
        l = l * expf(m - ref) + expf(x - ref);
        m = top;
    }
    float top = m;
    for (int w = 1; w < 64; w *= 2) top = fmaxf(top, __shfl_xor(top, w));
    l = lane_group_sum<64>(l * expf(m - (top == -INFINITY ? 0.f : top)));
    if ((tid & 63) == 0) { s_m[tid >> 6] = top; s_l[tid >> 6] = l; }
    __syncthreads();
    if (tid == 0) {
        float M = s_m[0], L = 0.f;
        for (int i = 1; i < 4; ++i) M = fmaxf(M, s_m[i]);
        for (int i = 0; i < 4; ++i) L += s_l[i] * expf(s_m[i] - (M == -INFINITY ? 0.f : M));
        c.ws[(size_t)bh * c.T + t] = vis > 0 ? M + logf(L) : -INFINITY;
    }
}

// ---- the weights: a thread per row ----
template <typename T, int D>
__global__ __launch_bounds__(CW_THREADS) void weights_add_kernel(WeightsCall c) {
    const int bh = blockIdx.y, r = blockIdx.x * CW_THREADS + threadIdx.x;
    const int n = min(max(c.cache_len[bh], 0), c.cap);
    if (r >= n) return;
    const T* K = (const T*)c.k_cache + ((size_t)bh * c.cap + r) * D;
    const float* lse = (c.lse != nullptr ? c.lse : c.ws) + (size_t)bh * c.T;
    float k[D];
    for (int e = 0; e < D; ++e) k[e] = to_float(K[e]) * c.scale;
    float sum = 0.f;
    for (int t = 0; t < c.T; ++t) {
        if (r >= sees_rows(c, bh, t, n) || lse[t] == -INFINITY) continue;
        const T* q = query<T>(c, bh, t);
        float x = 0.f;
        for (int e = 0; e < D; ++e) x += to_float(q[e]) * k[e];
        sum += expf(x - lse[t]);
    }
    float* w = c.weights + (size_t)bh * c.cap + r;
    *w = c.decay * *w + sum;
}

size_t weights_workspace(const WeightsCall& c, bool lse_given) { return lse_given ? 0 : (size_t)c.B * c.H * c.T; }

template <typename T, int D>
static nats_status run_weights(const WeightsCall& c, hipStream_t st) {
    const int heads = c.B * c.H;
    if (c.lse == nullptr) {
        ProfScope ps("cache_weights_lse", st);
        hipLaunchKernelGGL((weights_lse_kernel<T, D>), dim3(c.T, heads), dim3(CW_THREADS), 0, st, c);
    }
    ProfScope ps("cache_weights", st);
    hipLaunchKernelGGL((weights_add_kernel<T, D>), dim3((c.cap + CW_THREADS - 1) / CW_THREADS, heads), dim3(CW_THREADS), 0, st, c);
    return check_launch("cache_weights");
}

nats_status launch_cache_weights(const WeightsCall& c, hipStream_t st) {
    if (c.dtype == NATS_F32) return c.d == 64 ? run_weights<float, 64>(c, st) : run_weights<float, 128>(c, st);
    return c.d == 64 ? run_weights<bf16_t, 64>(c, st) : run_weights<bf16_t, 128>(c, st);
}

// ---- eviction: which rows stay ----
constexpr int EV_THREADS = 1024;

// A number that orders as the weights do (a NaN below all, -0 as 0)
__device__ __forceinline__ uint32_t weight_key(float w) {
    if (w != w) return 0;
    const uint32_t u = __float_as_uint(w + 0.f);
    return u & 0x80000000u ? ~u : u | 0x80000000u;
}

// exclusive prefix sum of an int over the block and its total
__device__ __forceinline__ int block_scan(int x, int* s_part, int& total) {
    const int tid = threadIdx.x, incl = wave_inclusive_scan_i32(x);
    __syncthreads();   // s_part of the scan before has been read
    if ((tid & 63) == 63) s_part[tid >> 6] = incl;
    __syncthreads();
    int before = 0;
    total = 0;
    for (int w = 0; w < EV_THREADS / 64; ++w) {
        if (w < (tid >> 6)) before += s_part[w];
        total += s_part[w];
    }
    return before + incl - x;
}

// One block per cache.  The weight of the last row that stays is found digit by digit (8 bits of its key at a time, from counts of the
// rows that agree in the digits so far); then the rows above it, the lowest of those equal to it and the last `recent` ones are
// numbered in order, and their weights moved.  A row's new place is never behind its old one, and a step's rows are read before
// any of them is written, so that the weights are compacted in place.
__global__ __launch_bounds__(EV_THREADS) void evict_select_kernel(EvictCall c) {
    __shared__ int s_hist[256], s_part[EV_THREADS / 64];
    __shared__ uint32_t s_digit;
    __shared__ int s_rest;
    const int bh = blockIdx.x, tid = threadIdx.x;
    const int n = min(max(c.cache_len[bh], 0), c.cap);
    float* w = c.weights + (size_t)bh * c.cap;
    int32_t* kept = c.kept + (size_t)bh * c.keep;
    if (n <= c.keep) {
        for (int r = tid; r < c.keep; r += EV_THREADS) kept[r] = r < n ? r : -1;
        return;
    }
    const int m = n - c.recent;   // the rows to choose from
    uint32_t prefix = 0;
    int rest = c.keep - c.recent;   // of the rows that agree with `prefix`, this many stay
    if (rest > 0) {
        for (int shift = 24; shift >= 0; shift -= 8) {
            for (int i = tid; i < 256; i += EV_THREADS) s_hist[i] = 0;
            __syncthreads();
            for (int r = tid; r < m; r += EV_THREADS) {
                const uint32_t key = weight_key(w[r]);
                if (shift == 24 || (key >> (shift + 8)) == (prefix >> (shift + 8))) atomicAdd(&s_hist[(key >> shift) & 255], 1);
            }
            __syncthreads();
            if (tid == 0) {
                int d = 255, left = rest;
                while (d > 0 && s_hist[d] < left) left -= s_hist[d--];
                s_digit = d;
                s_rest = left;
            }
            __syncthreads();
            prefix |= s_digit << shift;
            rest = s_rest;
            __syncthreads();
        }
    }
    int done = 0, equal = 0;   // rows that stay and rows equal to the threshold so far
    const bool any = c.keep > c.recent;
    for (int r0 = 0; r0 < n; r0 += EV_THREADS) {
        const int r = r0 + tid;
        const float x = r < n ? w[r] : 0.f;
        const uint32_t key = weight_key(x);
        const bool tie = r < m && any && key == prefix;
        int ties, all;
        const int rank = equal + block_scan(tie, s_part, ties);
        const bool stays = r < n && (r >= m || (any && (key > prefix || (tie && rank < rest))));
        const int at = done + block_scan(stays, s_part, all);   // (every thread has read its weight)
        if (stays) {
            w[at] = x;
            kept[at] = r;
        }
        done += all;
        equal += ties;
        __syncthreads();
    }
    if (tid == 0) c.cache_len[bh] = c.keep;
}

// ---- eviction: the rows move ----
// A block per cache, K or V, and slice of 64 bytes of the rows; rows in order, a step's rows read before any of them is written.
constexpr int MV_THREADS = 256, MV_ROWS = MV_THREADS / 4;
__global__ __launch_bounds__(MV_THREADS) void evict_move_kernel(EvictCall c, int row_bytes) {
    const int bh = blockIdx.y, slice = blockIdx.x, slices = row_bytes / 64, tid = threadIdx.x;
    char* base = (char*)(slice < slices ? c.k_cache : c.v_cache) + (size_t)bh * c.cap * row_bytes + (slice % slices) * 64 + (tid & 3) * 16;
    const int32_t* kept = c.kept + (size_t)bh * c.keep;
    for (int r0 = 0; r0 < c.keep; r0 += MV_ROWS) {
        const int r = r0 + (tid >> 2), src = r < c.keep ? kept[r] : -1;
        uint4 x = make_uint4(0, 0, 0, 0);
        if (src > r) x = *reinterpret_cast<const uint4*>(base + (size_t)src * row_bytes);
        asm volatile("" : "+v"(x.x), "+v"(x.y), "+v"(x.z), "+v"(x.w));   // the row has arrived before the barrier
        __syncthreads();
        if (src > r) *reinterpret_cast<uint4*>(base + (size_t)r * row_bytes) = x;
    }
}

nats_status launch_cache_evict(const EvictCall& c, hipStream_t st) {
    const int heads = c.B * c.H, row_bytes = c.d * (c.dtype == NATS_F32 ? 4 : 2);
    {
        ProfScope ps("evict_select", st);
        hipLaunchKernelGGL(evict_select_kernel, dim3(heads), dim3(EV_THREADS), 0, st, c);
    }
    ProfScope ps("evict_move", st);
    hipLaunchKernelGGL(evict_move_kernel, dim3(2 * row_bytes / 64, heads), dim3(MV_THREADS), 0, st, c, row_bytes);
    return check_launch("cache_evict");
}

}  // namespace nats

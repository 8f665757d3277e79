// Both branches of a tree of drafted tokens, read in one launch: the first blocks take the linear branch (tree_linear.h), the others the
// softmax branch over the cache: partial results (running maximum m, sum l, weighted sum of V rows) of up to 64 queries over a part of a
// cache's rows.  Side by side the linear branch's dependent steps cost nothing where there are rows to read.
//
// Memory-bound: a cache row of 4 d (bf16) or 8 d bytes (fp32) feeds 4 d T operations, at most T = 64 per byte, against the 240 (bf16)
// that a large product has per byte of a large copy on this card.  So all that matters is that every row is read once and that enough
// loads are in flight: a wavefront takes tiles of 32 rows (fp32: 16) by itself, holds a tile of K and one of V in registers, and asks
// for the next K as soon as the logits are there, for the next V as soon as it has been put in order, so that the softmax and
// the second product run while 16 KB per wavefront are on their way.  No LDS in the loop, no barrier.
//
//   S^T [key x query] = K Q^T      A = K rows as they lie in memory (16 bytes per lane), B = Q, in registers throughout
//   O^T [d_v x query] += V^T P^T   B = P^T as the first product's result tiles hold it (a lane has 4 consecutive keys of one query, two
//                                  tiles fill the 8 slots of a bf16 operand); A = V^T: a lane reads 8 (4) columns of the keys of
//                                  its slots, and column 8 l + e of all lanes l is row l of tile e: the keys' halves of a column are
//                                  joined by byte permutes (bf16) or stand as they came (fp32)
// bf16 tensors: logits are exact products summed in fp32; P enters as the sum of three bf16 terms, all of its 24 bits: with two (17 bits) ten
// times as many outputs were rounded to the wrong neighbour, and this kernel has matrix cycles to spare (us of a call with two / three: 1024
// caches of 64 .. 2048 rows, 16 nodes 148 / 148; 32 of 32000, 64 nodes 130 / 130, of 64 columns 82 / 87; 96 of 64 .. 1024, 33 nodes 27.5 / 28.2).
// Every term is cut off, so that the last one is exact, and the lower two are kept above 0, so that an infinity in V stays one.
#include <math.h>

#include "mfma_util.h"
#include "nats_common.h"
#include "serve.h"
#include "softmax_terms.h"
#include "tree_linear.h"

namespace nats {

// over the lanes l, l ^ 16, l ^ 32, l ^ 48, which share a query
__device__ __forceinline__ float over_quads_max(float x) {
    const int lane = threadIdx.x & 63;
    x = fmaxf(x, lane_xor32(x, lane));
    return fmaxf(x, lane_xor16(x, lane));
}
__device__ __forceinline__ float over_quads_sum(float x) {
    const int lane = threadIdx.x & 63;
    x += lane_xor32(x, lane);
    return x + lane_xor16(x, lane);
}

// A tile of 16 KT rows in a wavefront's registers, and the two products with it.
template <typename T, int D>
struct CacheTile;

template <int D>
struct CacheTile<bf16_t, D> {
    static constexpr int KT = 2, W = D / 32;   // W: 32-bit words of a V row per lane (D / 16 columns)
    using Query = u32x4[D / 32];               // column l16 of Q^T, elements 32 ks + 8 lq ..
    using Weights = u32x4[N_TERMS];            // the upper term first
    u32x4 k[KT][D / 32];
    uint32_t v[8][W];                          // slot s: key 16 (s / 4) + 4 lq + s % 4
    __device__ __forceinline__ static void load_query(const bf16_t* row, int lq, bool live, Query& q) {
#pragma unroll
        for (int i = 0; i < D / 32; ++i)
            q[i] = live ? *reinterpret_cast<const u32x4*>(row + 32 * i + 8 * lq) : u32x4{0, 0, 0, 0};
    }
    __device__ __forceinline__ void load_k(const bf16_t* K, int row, int last, int l16, int lq) {
#pragma unroll
        for (int t = 0; t < KT; ++t) {
            const bf16_t* p = K + (size_t)min(row + 16 * t + l16, last) * D + 8 * lq;
#pragma unroll
            for (int i = 0; i < D / 32; ++i) k[t][i] = *reinterpret_cast<const u32x4*>(p + 32 * i);
        }
    }
    template <bool ONCE>   // (read by one wavefront alone, in whole lines: past the caches)
    __device__ __forceinline__ void load_v(const bf16_t* V, int row, int last, int l16, int lq) {
#pragma unroll
        for (int s = 0; s < 8; ++s) {
            const bf16_t* p = V + (size_t)min(row + 16 * (s / 4) + 4 * lq + s % 4, last) * D + 2 * W * l16;
            if constexpr (W == 4) {
                const u32x4* w = reinterpret_cast<const u32x4*>(p);
                const u32x4 x = ONCE ? __builtin_nontemporal_load(w) : *w;
#pragma unroll
                for (int i = 0; i < 4; ++i) v[s][i] = x[i];
            } else {
                const uint2 x = *reinterpret_cast<const uint2*>(p);
                v[s][0] = x.x;
                v[s][1] = x.y;
            }
        }
    }
    __device__ __forceinline__ void clear_v(int row, int last, int lq) {   // rows past the last one may hold anything
#pragma unroll
        for (int s = 0; s < 8; ++s)
#pragma unroll
            for (int i = 0; i < W; ++i) v[s][i] = row + 16 * (s / 4) + 4 * lq + s % 4 > last ? 0u : v[s][i];
    }
    __device__ __forceinline__ void logits(const Query& q, f32x4 (&s)[KT]) const {
#pragma unroll
        for (int t = 0; t < KT; ++t) {
            s[t] = f32x4{0.f, 0.f, 0.f, 0.f};
#pragma unroll
            for (int i = 0; i < D / 32; ++i) s[t] = mfma_bf16(k[t][i], q[i], s[t]);
        }
    }
    __device__ __forceinline__ static void weights(const f32x4 (&p)[KT], Weights& w) {
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            float x = p[i / 2][2 * (i % 2)], y = p[i / 2][2 * (i % 2) + 1];
#pragma unroll
            for (int n = 0; n < N_TERMS; ++n) {
                w[n][i] = __builtin_amdgcn_perm(__float_as_uint(y), __float_as_uint(x), 0x07060302u);   // upper halves
                if (n == N_TERMS - 1) break;
                x = fmaxf(x - __uint_as_float(__float_as_uint(x) & 0xffff0000u), 0x1p-120f);
                y = fmaxf(y - __uint_as_float(__float_as_uint(y) & 0xffff0000u), 0x1p-120f);
            }
        }
    }
    // column `column(lq, j, e)` of the result is what element j of tile e holds
    __device__ __forceinline__ static int column(int lq, int j, int e) { return 2 * W * (4 * lq + j) + e; }
    template <int NQ>
    __device__ __forceinline__ void products(const f32x4 (&p)[NQ][KT], f32x4 (&o)[NQ][D / 16]) const {
        Weights w[NQ];
#pragma unroll
        for (int n = 0; n < NQ; ++n) weights(p[n], w[n]);
#pragma unroll
        for (int e = 0; e < D / 16; ++e) {
            u32x4 a;
#pragma unroll
            for (int i = 0; i < 4; ++i)
                a[i] = __builtin_amdgcn_perm(v[2 * i + 1][e / 2], v[2 * i][e / 2], e % 2 ? 0x07060302u : 0x05040100u);
#pragma unroll
            for (int i = N_TERMS - 1; i >= 0; --i)
#pragma unroll
                for (int n = 0; n < NQ; ++n) o[n][e] = mfma_bf16(a, w[n][i], o[n][e]);
        }
    }
};

template <int D>
struct CacheTile<float, D> {
    static constexpr int KT = 1;
    using Query = float4[D / 16];
    float4 k[D / 16];
    float4 v[4][D / 64];   // key 4 lq + j, columns 64 g + 4 l16 ..
    __device__ __forceinline__ static void load_query(const float* row, int lq, bool live, Query& q) {
#pragma unroll
        for (int i = 0; i < D / 16; ++i) q[i] = live ? ld4(row + 16 * i + 4 * lq) : make_float4(0.f, 0.f, 0.f, 0.f);
    }
    __device__ __forceinline__ void load_k(const float* K, int row, int last, int l16, int lq) {
        const float* p = K + (size_t)min(row + l16, last) * D + 4 * lq;
#pragma unroll
        for (int i = 0; i < D / 16; ++i) k[i] = ld4(p + 16 * i);
    }
    template <bool ONCE>
    __device__ __forceinline__ void load_v(const float* V, int row, int last, int l16, int lq) {
#pragma unroll
        for (int j = 0; j < 4; ++j)
#pragma unroll
            for (int g = 0; g < D / 64; ++g) v[j][g] = ld4(V + (size_t)min(row + 4 * lq + j, last) * D + 64 * g + 4 * l16);
    }
    __device__ __forceinline__ void clear_v(int row, int last, int lq) {
#pragma unroll
        for (int j = 0; j < 4; ++j)
#pragma unroll
            for (int g = 0; g < D / 64; ++g) {
                const bool out = row + 4 * lq + j > last;
                v[j][g].x = out ? 0.f : v[j][g].x;
                v[j][g].y = out ? 0.f : v[j][g].y;
                v[j][g].z = out ? 0.f : v[j][g].z;
                v[j][g].w = out ? 0.f : v[j][g].w;
            }
    }
    __device__ __forceinline__ void logits(const Query& q, f32x4 (&s)[KT]) const {
        s[0] = f32x4{0.f, 0.f, 0.f, 0.f};
#pragma unroll
        for (int i = 0; i < D / 16; ++i) s[0] = mac16(k[i], q[i], s[0]);
    }
    __device__ __forceinline__ static int column(int lq, int j, int e) { return 64 * (e / 4) + 16 * lq + 4 * j + e % 4; }
    template <int NQ>
    __device__ __forceinline__ void products(const f32x4 (&p)[NQ][KT], f32x4 (&o)[NQ][D / 16]) const {
#pragma unroll
        for (int g = 0; g < D / 64; ++g)
#pragma unroll
            for (int n = 0; n < NQ; ++n) {
#pragma unroll
                for (int j = 0; j < 4; ++j) {
                    o[n][4 * g] = __builtin_amdgcn_mfma_f32_16x16x4f32(v[j][g].x, p[n][0][j], o[n][4 * g], 0, 0, 0);
                    o[n][4 * g + 1] = __builtin_amdgcn_mfma_f32_16x16x4f32(v[j][g].y, p[n][0][j], o[n][4 * g + 1], 0, 0, 0);
                    o[n][4 * g + 2] = __builtin_amdgcn_mfma_f32_16x16x4f32(v[j][g].z, p[n][0][j], o[n][4 * g + 2], 0, 0, 0);
                    o[n][4 * g + 3] = __builtin_amdgcn_mfma_f32_16x16x4f32(v[j][g].w, p[n][0][j], o[n][4 * g + 3], 0, 0, 0);
                }
            }
    }
};

constexpr int TC_THREADS = 256, TC_WAVES = TC_THREADS / 64;
constexpr int TREE_LEAST_UNITS = 8;   // of a block's share

// `count` rows of cache bhg from `lo` on, into part `slot`.  NQ: tiles of 16 queries per wavefront; QG: groups of 16 NQ queries in a block, the block's other wavefronts share the rows
template <int D, int NQ>
struct CacheLds {
    f32x4 o[2][NQ * (D / 16)][64];
    float ml[2][NQ][2][64];
};

template <typename T, int D, int NQ, int QG>
__device__ __forceinline__ void tree_cache_block(const TreeCall& c, int bhg, int lo, int count, int slot, CacheLds<D, NQ>& lds) {
    using Tile = CacheTile<T, D>;
    constexpr int KT = Tile::KT, ROWS = 16 * KT, KG = TC_WAVES / QG, E = D / 16;
    constexpr float LOG2E = 1.44269504088896341f;
    auto& s_o = lds.o;
    auto& s_ml = lds.ml;
    const int lane = threadIdx.x & 63, l16 = lane & 15, lq = lane >> 4;
    const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), qg = wave / KG, kg = wave % KG;
    const int last = count - 1;
    const T* K = (const T*)c.k_cache + ((size_t)bhg * c.cap + lo) * D;
    const T* V = (const T*)c.v_cache + ((size_t)bhg * c.cap + lo) * D;
    const T* Q = c.q_nla != nullptr ? (const T*)c.q_nla + (size_t)bhg * c.T * D : (const T*)c.q + (size_t)(bhg / c.G) * c.T * D;
    const float scale2 = c.scale * LOG2E;

    // (A tile past the end is asked for too, all its rows the last one: with the loads behind a condition the compiler gave registers of
    // the V tile to temporaries.)
    Tile tile;
    int row = kg * ROWS;
    tile.load_k(K, row, last, l16, lq);
    tile.template load_v<QG == 1>(V, row, last, l16, lq);
    typename Tile::Query q[NQ];
    f32x4 o[NQ][E];
    float m[NQ], l[NQ];
#pragma unroll
    for (int i = 0; i < NQ; ++i) {
        const int t = (qg * NQ + i) * 16 + l16;
        Tile::load_query(Q + (size_t)min(t, c.T - 1) * D, lq, t < c.T, q[i]);
        m[i] = -INFINITY;
        l[i] = 0.f;
#pragma unroll
        for (int e = 0; e < E; ++e) o[i][e] = f32x4{0.f, 0.f, 0.f, 0.f};
    }
    for (; row <= last; row += KG * ROWS) {
        const int next = row + KG * ROWS;
        f32x4 s[NQ][KT];
#pragma unroll
        for (int i = 0; i < NQ; ++i) tile.logits(q[i], s[i]);
        tile.load_k(K, next, last, l16, lq);
        const bool whole = row + ROWS - 1 <= last;
#pragma unroll
        for (int i = 0; i < NQ; ++i) {
            float top = -INFINITY;
#pragma unroll
            for (int t = 0; t < KT; ++t)
#pragma unroll
                for (int j = 0; j < 4; ++j) {
                    float z = s[i][t][j] * scale2;
                    if (!whole) z = row + 16 * t + 4 * lq + j > last ? -INFINITY : z;
                    s[i][t][j] = z;
                    top = fmaxf(top, z);
                }
            top = over_quads_max(top);
            // the running maximum follows only where a logit is more than 2^8 above it: weights stay below 2^8
            const bool raise = top > m[i] + 8.f;   // also at the first row (m = -inf)
            if (__any(raise)) {
                const float corr = raise ? __builtin_amdgcn_exp2f(m[i] - top) : 1.f;
                m[i] = raise ? top : m[i];
                l[i] *= corr;
#pragma unroll
                for (int e = 0; e < E; ++e) o[i][e] *= corr;
            }
            const float ref = m[i] == -INFINITY ? 0.f : m[i];
#pragma unroll
            for (int t = 0; t < KT; ++t)
#pragma unroll
                for (int j = 0; j < 4; ++j) {
                    s[i][t][j] = __builtin_amdgcn_exp2f(s[i][t][j] - ref);
                    l[i] += s[i][t][j];
                }
        }
        if (!whole) tile.clear_v(row, last, lq);
        tile.template products<NQ>(s, o);
        tile.template load_v<QG == 1>(V, next, last, l16, lq);
    }
#pragma unroll
    for (int i = 0; i < NQ; ++i) l[i] = over_quads_sum(l[i]);

    // the wavefronts that share queries: the upper half of them hands its result to the lower half, until one is left
#pragma unroll
    for (int half = KG / 2; half >= 1; half /= 2) {
        const int place = qg * half + kg % half;
        static_assert(QG * (KG / 2) <= 2, "slots");
        if (half < KG / 2) __syncthreads();   // the slots have been read
        if (kg >= half && kg < 2 * half) {
#pragma unroll
            for (int i = 0; i < NQ; ++i) {
                s_ml[place][i][0][lane] = m[i];
                s_ml[place][i][1][lane] = l[i];
#pragma unroll
                for (int e = 0; e < E; ++e) s_o[place][i * E + e][lane] = o[i][e];
            }
        }
        __syncthreads();
        if (kg < half) {
#pragma unroll
            for (int i = 0; i < NQ; ++i) {
                const float m2 = s_ml[place][i][0][lane], l2 = s_ml[place][i][1][lane];
                const float top = fmaxf(m[i], m2), ref = top == -INFINITY ? 0.f : top;
                const float w1 = __builtin_amdgcn_exp2f(m[i] - ref), w2 = __builtin_amdgcn_exp2f(m2 - ref);
                m[i] = top;
                l[i] = w1 * l[i] + w2 * l2;
#pragma unroll
                for (int e = 0; e < E; ++e) o[i][e] = w1 * o[i][e] + w2 * s_o[place][i * E + e][lane];
            }
        }
    }
    if (kg != 0) return;
    const size_t part = (size_t)slot * c.T;
#pragma unroll
    for (int i = 0; i < NQ; ++i) {
        const int t = (qg * NQ + i) * 16 + l16;
        if (t >= c.T) continue;
        float* out = c.ws + c.off_part + (part + t) * D;
#pragma unroll
        for (int j = 0; j < 4; ++j)
#pragma unroll
            for (int e = 0; e < E; e += 4)
                *reinterpret_cast<f32x4*>(out + Tile::column(lq, j, e)) = f32x4{o[i][e][j], o[i][e + 1][j], o[i][e + 2][j], o[i][e + 3][j]};
        if (lq == 0) *reinterpret_cast<float2*>(c.ws + c.off_ml + (part + t) * 2) = make_float2(m[i], l[i]);
    }
}

static_assert(TC_THREADS == TL_THREADS, "blocks of either kind in one launch");

// Block x of c.even: an equal share of the rows of all caches, which may begin and end inside one.
template <typename T, int D, int NQ, int QG>
__device__ __forceinline__ void tree_even_block(const TreeCall& c, int x, int heads, CacheLds<D, NQ>& lds) {
    auto length = [&](int h) { return min(max(c.cache_len[h], 0), c.cap); };
    // the caches' units counted by all threads, some caches in a row each
    __shared__ int s_sum[TC_WAVES], s_head, s_unit;
    const int tid = threadIdx.x, lane = tid & 63, wave = tid >> 6;
    const int each = (heads + TC_THREADS - 1) / TC_THREADS, first = min(tid * each, heads), end = min(first + each, heads);
    auto units = [](int rows) { return (rows + TREE_UNIT - 1) / TREE_UNIT; };
    int mine = 0;
    for (int h = first; h < end; ++h) mine += units(length(h));
    const int upto = wave_inclusive_scan_i32(mine);
    if (lane == 63) s_sum[wave] = upto;
    __syncthreads();
    int before = upto - mine, total = 0;
#pragma unroll
    for (int v = 0; v < TC_WAVES; ++v) {
        before += v < wave ? s_sum[v] : 0;
        total += s_sum[v];
    }
    const int share = max((total + c.even - 1) / c.even, TREE_LEAST_UNITS), from = x * share;
    if (x == 0) {   // for the merge
        int at = before;
        for (int h = first; h < end; ++h) {
            c.units()[h] = at;
            at += units(length(h));
        }
        if (tid == 0) {
            c.units()[heads] = total;
            c.units()[heads + 1] = share;
        }
    }
    if (from >= total) return;
    if (before <= from && from < before + mine) {
        int h = first, at = before;
        for (int u = units(length(h)); at + u <= from; u = units(length(h))) {
            at += u;
            ++h;
        }
        s_head = h;
        s_unit = from - at;
    }
    __syncthreads();
    int left = min(share, total - from), unit = s_unit;
    for (int h = s_head; left > 0 && h < heads; ++h, unit = 0) {
        const int n = length(h), take = min(left, units(n) - unit), lo = unit * TREE_UNIT;
        if (take <= 0) continue;   // an empty cache
        tree_cache_block<T, D, NQ, QG>(c, h, lo, min(n - lo, take * TREE_UNIT), h + x, lds);
        left -= take;
        __syncthreads();   // the LDS is free again
    }
}

// Blocks of a CU that the registers are shared out for.  Narrow heads of bf16: four, or in equal shares of more than 16 nodes three, for with
// the weights' three terms four leave some of the registers in memory (us of a call with four / three: 1024 caches of 64 .. 2048 rows, 20
// nodes 97 / 92; 512 of them, 40 nodes 70 / 67; but without equal shares, where blocks are short, 300 caches of up to 1000 rows, 40 nodes
// 34 / 37).
constexpr int narrow_blocks(bool bf16, int T, bool even) { return bf16 && even && T > 16 ? 3 : 4; }

template <typename T, int D, int NT, int TURNS, bool EVEN>
__global__ __launch_bounds__(TC_THREADS, D == 64 ? narrow_blocks(sizeof(T) == 2, 16 * NT, EVEN) : 2) void tree_read_kernel(TreeCall c) {
    constexpr int PARTS = D / (64 * TURNS);   // blocks of a head's linear branch
    constexpr int NQ = NT == 1 ? 1 : 2, QG = NT <= 2 ? 1 : 2;
    __shared__ union {
        LinearLds<NT> linear;
        CacheLds<D, NQ> cache;
    } s;
    const int heads = c.B * c.H * c.G, id = blockIdx.x;
    if (id < heads * PARTS) {
        tree_linear_block<T, D, NT, TURNS>(c, id / PARTS, id % PARTS, s.linear);
        return;
    }
    const int x = id - heads * PARTS;
    auto length = [&](int h) { return min(max(c.cache_len[h], 0), c.cap); };
    if constexpr (!EVEN) {
        const int h = x / c.n_split, lo = x % c.n_split * c.rows, count = min(length(h) - lo, c.rows);
        // (the merge knows from the same length which parts exist)
        if (count > 0) tree_cache_block<T, D, NQ, QG>(c, h, lo, count, x, s.cache);
    } else {
        tree_even_block<T, D, NQ, QG>(c, x, heads, s.cache);
    }
}

template <typename T, int D, int TURNS, bool EVEN>
static void run_tree_read(const TreeCall& c, hipStream_t st) {
    const int heads = c.B * c.H * c.G;
    const dim3 grid(heads * (D / (64 * TURNS)) + (EVEN ? c.even : heads * c.n_split)), block(TC_THREADS);
    if (c.T <= 16) hipLaunchKernelGGL((tree_read_kernel<T, D, 1, TURNS, EVEN>), grid, block, 0, st, c);
    else if (c.T <= 32) hipLaunchKernelGGL((tree_read_kernel<T, D, 2, TURNS, EVEN>), grid, block, 0, st, c);
    else if (c.T <= 48) hipLaunchKernelGGL((tree_read_kernel<T, D, 3, TURNS, EVEN>), grid, block, 0, st, c);
    else hipLaunchKernelGGL((tree_read_kernel<T, D, 4, TURNS, EVEN>), grid, block, 0, st, c);
}

// d = 128 with few heads: a head's linear branch in two blocks, which is the shorter chain
static bool halves(const TreeCall& c) { return (long long)c.B * c.H * c.G <= 128; }

// Parts of the caches.  Large parts make few partial results (4 T d bytes each, written and read) and long runs of rows; small ones fill the
// chip where there are few caches.  us of both kernels with parts of 256 / 512 / 1024 / 2048 rows: 1024 caches of 64 .. 2048 rows, 16 nodes
// 207 / 187 / 176 / 171; 32 of 32000, 64 nodes 227 / 176 / 154 / 140; 96 of 64 .. 1024, 33 nodes 36 / 34 / 41 / 41; 16 of 1000, 16 nodes 17 /
// 18 / 24 / 23 (128 rows: 19).  With many caches the longest decide when parts are caches: then every block that fits the chip at once
// takes the same number of rows (us a call, by caches and by shares: 1024 caches of 64 .. 2048 rows, 16 nodes 158 / 149; 512 of them, 33 nodes
// 130 / 115; 384 in fp32, 20 nodes 175 / 131).  That costs a scan of all lengths per block and shares that end inside a cache: nothing for
// fewer caches, for shorter ones (768 of 64 .. 1024, 64 nodes 148 / 159; 516 of 23 .. 418, d 64, 36 nodes 34 / 39), nor for so many that their
// number evens out.
void tree_cache_parts(TreeCall& c) {
    const long long heads = (long long)c.B * c.H * c.G;
    c.rows = 2048;
    while (c.rows > 256 && heads * ((c.cap + c.rows - 1) / c.rows) < (c.rows > 512 ? 512 : 192)) c.rows /= 2;
    c.n_split = (c.cap + c.rows - 1) / c.rows;
    const int per_cu = c.d == 64 ? (c.T <= 48 ? narrow_blocks(c.dtype == NATS_BF16, c.T, true) : 2) : (c.T <= 16 ? 3 : 2);   // blocks that a CU holds
    c.even = !halves(c) && c.cap > 1024 && heads <= 2048 ? 256 * per_cu : 0;
}

nats_status launch_tree_read(const TreeCall& c, hipStream_t st) {
    ProfScope ps("tree_read", st);
    auto run = [&](auto zero) {
        using T = decltype(zero);
        if (c.d == 64) c.even ? run_tree_read<T, 64, 1, true>(c, st) : run_tree_read<T, 64, 1, false>(c, st);
        else if (halves(c)) run_tree_read<T, 128, 1, false>(c, st);
        else c.even ? run_tree_read<T, 128, 2, true>(c, st) : run_tree_read<T, 128, 2, false>(c, st);
    };
    if (c.dtype == NATS_F32) run(float{});
    else run(bf16_t{});
    return check_launch("tree_read");
}

}  // namespace nats

// Linear branch of a tree of drafted tokens (internal header): the work of a block of four wavefronts for one output head.
//
// With a_i the decay and b_i the write strength of node i, g_i the product of the decays on its path and r_ij that of the decays behind
// ancestor j up to i, the states of all nodes are sums over their ancestors, and S itself is read once:
//   S_i = g_i S + sum_j r_ij u_j k_j^T                              (j: ancestors of i and i)
//   u_i = b_i (v_i - g_i S k_i + sum_{j != i} n_ij u_j / b_i),      n_ij = -b_i r_ij (k_i . k_j)
//   o_i = la_scale (g_i S q_i + sum_j r_ij (q_i . k_j) u_j)
// i.e. (I - N) U = diag(b) (V - diag(g) K S^T) with N strictly lower triangular, since parents come first.  It is solved by blocks of
// 16 nodes, the diagonal blocks' inverses made once per head.
//
// A wavefront takes 16 rows of S (columns of U) at a time and needs nothing of the others': K S^T, the solution and P U are products whose
// result tiles are the next one's operand as they sit in registers.  K S^T and Q S^T run on the bf16 instruction with S as three bf16
// terms (all of its bits), the products with N, P and U, up to 64 x 64, on the fp32 one.
//
// In a product a node that is no ancestor has a coefficient of 0, which an infinity or a NaN in its u turns into NaN.  So a wavefront
// whose u and S q are not all finite does its columns again, ancestor by ancestor, with the products formed on the fp32 instruction: an infinity
// has no three terms that add up to it, nor has a number that bf16 rounds to one.
#pragma once
#include "nats_common.h"
#include "serve.h"
#include "softmax_terms.h"
#include "tree_nodes.h"

namespace nats {

constexpr int TL_THREADS = 256, TL_WAVES = TL_THREADS / 64;

template <int NT>   // tiles of 16 nodes
struct LinearLds {
    static constexpr int N = 16 * NT;
    float n[N][N + 4], p[N][N + 4];      // rows of fp32 operands: 16-byte reads of 16 rows
    float inv[NT][16][20];
    float u[TL_WAVES][N][16];
    float a[64], b[64], g[64];
    double lg[64];                       // log2 g
    uint64_t anc[64];
    int par[64];
    int plain;                           // every decay is an ordinary positive number
    int there;                           // nodes
};

__device__ __forceinline__ float4 as_float4(f32x4 x) { return make_float4(x[0], x[1], x[2], x[3]); }
// four nodes' results, those of nodes from `first` up to `there` finite (what stands in nodes that are not there is of no use)
__device__ __forceinline__ bool all_finite(f32x4 x, int first, int there) {
    bool fine = true;
#pragma unroll
    for (int e = 0; e < 4; ++e) fine = fine && (fabsf(x[e]) < INFINITY || first + e >= there);
    return fine;
}
// four elements of a row as the fp32 instruction takes them
__device__ __forceinline__ float4 row4(const float* p) { return ld4(p); }
__device__ __forceinline__ float4 row4(const bf16_t* p) { return ldb4(reinterpret_cast<const uint16_t*>(p)); }

// TURNS x 64 rows of S, number `part` of them
template <typename T, int D, int NT, int TURNS>
__device__ __forceinline__ void tree_linear_block(const TreeCall& c, int bhg, int part, LinearLds<NT>& s) {
    constexpr int KS = D / 32;
    const int bh = bhg / c.G, b = bh / c.H, N = c.T, lane = threadIdx.x & 63, l16 = lane & 15, lq = lane >> 4;
    const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    const T* q = (const T*)c.q + (size_t)bh * N * D;
    const T* k = (const T*)c.k + (size_t)bh * N * D;
    const T* v = (const T*)c.v + (size_t)bhg * N * D;
    const float* S = c.state + (size_t)bhg * D * D;

    // the first rows of S are on their way while the tree is looked at
    Raw8<float> sr[KS];
    auto load_state = [&](int row0) {
#pragma unroll
        for (int i = 0; i < KS; ++i) sr[i].load(S + (size_t)(row0 + l16) * D + 32 * i + 8 * lq);
    };
    const int row0 = 16 * (part * TURNS * TL_WAVES + wave);   // of the wavefront's first turn
    load_state(row0);
    float vv[NT][4];
    auto load_values = [&](int col) {
#pragma unroll
        for (int t = 0; t < NT; ++t)
#pragma unroll
            for (int e = 0; e < 4; ++e) vv[t][e] = to_float(v[(size_t)min(16 * t + 4 * lq + e, N - 1) * D + col]);
    };
    load_values(row0 + l16);

    // ---- N and P, the products: the lower triangle's tiles, dealt out to the wavefronts; the first tile's rows are asked for before the
    // last two wavefronts, which have the fewest tiles, look at the tree ----
    auto load_nodes = [&](const T* x, int tile, Raw8<T> (&r)[KS]) {
        const T* p = x + (size_t)min(16 * tile + l16, N - 1) * D + 8 * lq;
#pragma unroll
        for (int i = 0; i < KS; ++i) r[i].load(p + 32 * i);
    };
    constexpr int PAIRS = NT * (NT + 1) / 2, PER_WAVE = (PAIRS + TL_WAVES - 1) / TL_WAVES;
    auto tile_row = [](int pair) { return pair < 1 ? 0 : pair < 3 ? 1 : pair < 6 ? 2 : 3; };
    f32x4 kk[PER_WAVE], qk[PER_WAVE];
    Raw8<T> ki[KS], qi[KS], kj[KS];
    auto load_pair = [&](int pair) {
        const int ti = tile_row(pair), tj = pair - ti * (ti + 1) / 2;
        load_nodes(k, ti, ki);
        load_nodes(q, ti, qi);
        load_nodes(k, tj, kj);
    };
    load_pair(min(wave, PAIRS - 1));

    // ---- paths (one wavefront), their decays (another) ----
    if (wave >= TL_WAVES - 2) {
        const int par = parent_of(c.parent, b, N, lane);
        if (wave == TL_WAVES - 1) {
            const uint64_t anc = ancestors(par, lane);
            s.anc[lane] = anc;
            s.par[lane] = par;
            if (lane < N && part == 0 && bhg % (c.H * c.G) == 0) c.anc()[(size_t)b * N + lane] = anc;   // for the merge
        } else {
            const int there = c.n_nodes != nullptr ? min(c.n_nodes[b], N) : N;
            const bool soft = c.mask[(size_t)bh * N + min(lane, N - 1)] != 0;
            float a = c.alpha[(size_t)bh * N + min(lane, N - 1)], bt = c.beta[(size_t)bh * N + min(lane, N - 1)];
            if (lane >= N || (soft && c.freeze)) a = 1.f;
            if (lane >= there || soft) bt = 0.f;
            float g = a;
            double lg = log2((double)a);
            along_paths(par, lane, [&](bool up, int from) {
                const float more = __shfl(g, from);
                const uint64_t l = shfl_u64(__double_as_longlong(lg), from);
                if (up) {
                    g *= more;
                    lg += __longlong_as_double(l);
                }
            });
            const bool plain = __all(a > 0x1p-120f && a < 0x1p120f);
            s.a[lane] = a;
            s.b[lane] = bt;
            s.g[lane] = g;
            s.lg[lane] = lg;
            if (lane == 0) {
                s.plain = plain;
                s.there = there;
            }
        }
    }

#pragma unroll
    for (int x = 0; x < PER_WAVE; ++x) {
        kk[x] = qk[x] = f32x4{0.f, 0.f, 0.f, 0.f};
        if (wave + x * TL_WAVES >= PAIRS) break;
        if (x > 0) load_pair(wave + x * TL_WAVES);
#pragma unroll
        for (int i = 0; i < KS; ++i) {
            u32x4 tk[terms_of<T>()], tq[terms_of<T>()], tb[terms_of<T>()];
            ki[i].terms(tk);
            qi[i].terms(tq);
            kj[i].terms(tb);
            kk[x] = mfma_terms(tk, tb, kk[x]);
            qk[x] = mfma_terms(tq, tb, qk[x]);
        }
    }
    __syncthreads();
    const bool plain = s.plain != 0;
    const int there = s.there;
#pragma unroll
    for (int x = 0; x < PER_WAVE; ++x) {
        const int pair = wave + x * TL_WAVES;
        if (pair >= PAIRS) break;
        const int ti = tile_row(pair), tj = pair - ti * (ti + 1) / 2;
        const int j = 16 * tj + l16;
        if constexpr (sizeof(T) == 4) {
            // (node j is read as an ancestor, so it is there where the others are)
            const int i0 = 16 * ti + 4 * lq;
            if (!__all(j >= there || (all_finite(kk[x], i0, there) && all_finite(qk[x], i0, there)))) {
                const size_t at = (size_t)min(16 * ti + l16, N - 1) * D + 4 * lq, up = (size_t)min(j, N - 1) * D + 4 * lq;
                kk[x] = qk[x] = f32x4{0.f, 0.f, 0.f, 0.f};
#pragma unroll 1
                for (int i = 0; i < D; i += 16) {
                    const float4 kj4 = row4(k + up + i);
                    kk[x] = mac16(row4(k + at + i), kj4, kk[x]);
                    qk[x] = mac16(row4(q + at + i), kj4, qk[x]);
                }
            }
        }
        const double lgj = s.lg[j];
        const bool writes = s.b[j] != 0.f;
#pragma unroll
        for (int e = 0; e < 4; ++e) {
            const int i = 16 * ti + 4 * lq + e;
            const bool on = (s.anc[i] >> j) & 1;
            float r = 0.f;
            if (plain) {
                r = __builtin_amdgcn_exp2f((float)(s.lg[i] - lgj));
            } else if (on) {
                r = 1.f;
                for (int m = i; m != j; m = s.par[m]) r *= s.a[m];
            }
            // (a node that writes nothing, as one that is not there: its key may hold anything)
            s.n[i][j] = on && i != j && writes && s.b[i] != 0.f ? -s.b[i] * r * kk[x][e] : 0.f;
            s.p[i][j] = on && writes ? r * qk[x][e] : 0.f;
        }
    }
    __syncthreads();
    // ---- the diagonal blocks' inverses: lane (tile, column); the first K S^T and Q S^T are done beside them ----
    if (wave == 0 && lane < 16 * NT && c.linear_op == 0) {
        float x[16];
#pragma unroll
        for (int i = 0; i < 16; ++i) {
            float sum = i == l16 ? 1.f : 0.f;
#pragma unroll
            for (int j = 0; j < i; ++j) sum += s.n[16 * lq + i][16 * lq + j] * x[j];
            x[i] = sum;
            s.inv[lq][i][l16] = sum;
        }
    }
    f32x4 w[NT], o[NT];
    auto state_products = [&] {
#pragma unroll
        for (int t = 0; t < NT; ++t) w[t] = o[t] = f32x4{0.f, 0.f, 0.f, 0.f};
#pragma unroll
        for (int i = 0; i < KS; ++i) {
            u32x4 ts[N_TERMS];
            sr[i].terms(ts);
#pragma unroll
            for (int t = 0; t < NT; ++t) {
                Raw8<T> x;
                u32x4 tx[terms_of<T>()];
                const size_t at = (size_t)min(16 * t + l16, N - 1) * D + 32 * i + 8 * lq;
                x.load(k + at);
                x.terms(tx);
                w[t] = mfma_terms(tx, ts, w[t]);
                x.load(q + at);
                x.terms(tx);
                o[t] = mfma_terms(tx, ts, o[t]);
            }
        }
    };
    auto state_products_again = [&](int row0) {   // on the fp32 instruction
#pragma unroll
        for (int t = 0; t < NT; ++t) w[t] = o[t] = f32x4{0.f, 0.f, 0.f, 0.f};
#pragma unroll 1
        for (int i = 0; i < D; i += 16) {
            const float4 s4 = ld4(S + (size_t)(row0 + l16) * D + i + 4 * lq);
#pragma unroll
            for (int t = 0; t < NT; ++t) {
                const size_t at = (size_t)min(16 * t + l16, N - 1) * D + i + 4 * lq;
                w[t] = mac16(row4(k + at), s4, w[t]);
                o[t] = mac16(row4(q + at), s4, o[t]);
            }
        }
    };
    state_products();
    __syncthreads();

    // ---- 16 columns at a time ----
    float* O = c.ws + c.off_ola + (size_t)bhg * N * D;
#pragma unroll
    for (int turn = 0; turn < TURNS; ++turn) {
        const int col = row0 + 16 * TL_WAVES * turn + l16;
        if (turn > 0) {
            load_values(col);
            state_products();
        }
        if (turn + 1 < TURNS) load_state(row0 + 16 * TL_WAVES * (turn + 1));
        f32x4 u[NT];
        bool fine = true;
        auto weigh = [&](int t) {   // w: what the state alone has the nodes write; o: what they read of it
            const f32x4 g = *reinterpret_cast<const f32x4*>(&s.g[16 * t + 4 * lq]), bt = *reinterpret_cast<const f32x4*>(&s.b[16 * t + 4 * lq]);
#pragma unroll
            for (int e = 0; e < 4; ++e) {
                const float x = bt[e] * (c.linear_op == 0 ? vv[t][e] - g[e] * w[t][e] : vv[t][e]);
                w[t][e] = bt[e] == 0.f ? 0.f : x;   // (a softmax token writes nothing, whatever its v)
                o[t][e] *= g[e];
            }
        };
#pragma unroll
        for (int t = 0; t < NT; ++t) {
            weigh(t);
            u[t] = w[t];
            if (c.linear_op == 0) {
#pragma unroll
                for (int x = 0; x < t; ++x) u[t] = mac16(ld4(&s.n[16 * t + l16][16 * x + 4 * lq]), as_float4(u[x]), u[t]);
                u[t] = mac16(ld4(&s.inv[t][l16][4 * lq]), as_float4(u[t]), f32x4{0.f, 0.f, 0.f, 0.f});
            }
            fine = fine && all_finite(u[t], 16 * t + 4 * lq, there) && all_finite(o[t], 16 * t + 4 * lq, there);
        }
        if (__all(fine)) {
#pragma unroll
            for (int t = 0; t < NT; ++t)
#pragma unroll
                for (int x = 0; x <= t; ++x) o[t] = mac16(ld4(&s.p[16 * t + l16][16 * x + 4 * lq]), as_float4(u[x]), o[t]);
        } else {
            state_products_again(row0 + 16 * TL_WAVES * turn);
            load_values(col);
#pragma unroll
            for (int t = 0; t < NT; ++t) weigh(t);
            // ancestor by ancestor: 16 lanes a column each for u, then every lane its results
            float(&su)[16 * NT][16] = s.u[wave];
#pragma unroll
            for (int t = 0; t < NT; ++t)
#pragma unroll
                for (int e = 0; e < 4; ++e) su[16 * t + 4 * lq + e][l16] = w[t][e];
            __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "workgroup");
            __builtin_amdgcn_wave_barrier();
            if (lq == 0 && c.linear_op == 0) {
                for (int i = 0; i < N; ++i) {
                    float sum = su[i][l16];
                    if (s.b[i] == 0.f) continue;
                    for (uint64_t m = s.anc[i] & ~(1ull << i); m; m &= m - 1) {
                        const int j = __builtin_ctzll(m);
                        if (s.b[j] != 0.f) sum += s.n[i][j] * su[j][l16];
                    }
                    su[i][l16] = sum;
                }
            }
            __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "workgroup");
            __builtin_amdgcn_wave_barrier();
#pragma unroll
            for (int t = 0; t < NT; ++t)
#pragma unroll
                for (int e = 0; e < 4; ++e) {
                    const int i = 16 * t + 4 * lq + e;
                    for (uint64_t m = i < N ? s.anc[i] : 0; m; m &= m - 1) {
                        const int j = __builtin_ctzll(m);
                        if (s.b[j] != 0.f) o[t][e] += s.p[i][j] * su[j][l16];
                    }
                }
            __builtin_amdgcn_wave_barrier();
        }
#pragma unroll
        for (int t = 0; t < NT; ++t)
#pragma unroll
            for (int e = 0; e < 4; ++e) {
                const int i = 16 * t + 4 * lq + e;
                if (i < N) O[(size_t)i * D + col] = c.la_scale * o[t][e];
            }
    }
}

}  // namespace nats

// Ancestor sets of a tree of drafted tokens (internal header).
#pragma once
#include "nats_common.h"

namespace nats {

__device__ __forceinline__ uint64_t shfl_u64(uint64_t x, int from) {
    return ((uint64_t)(uint32_t)__shfl((int)(uint32_t)(x >> 32), from) << 32) | (uint32_t)__shfl((int)(uint32_t)x, from);
}

// parent[b][i] as the kernels use it: what is no earlier node counts as the root
__device__ __forceinline__ int parent_of(const int32_t* parent, int b, int T, int i) {
    const int p = i < T ? parent[(size_t)b * T + i] : -1;
    return p >= 0 && p < i ? p : -1;
}

// Folds every node's path to the root, by one wavefront with lane i for node i: step(up, from) is called six times, whatever the tree,
// with the node (lane) that the path so far ends before; the lane then takes that node's path so far too if `up`.
template <typename F>
__device__ __forceinline__ void along_paths(int parent, int lane, F&& step) {
    int at = parent;
#pragma unroll
    for (int r = 0; r < 6; ++r) {
        const int from = at < 0 ? lane : at, next = __shfl(at, from);
        step(at >= 0, from);
        if (at >= 0) at = next;
    }
}

// the set of every node's ancestors, itself among them, as a bit mask
__device__ __forceinline__ uint64_t ancestors(int parent, int lane) {
    uint64_t m = 1ull << lane;
    along_paths(parent, lane, [&](bool up, int from) {
        const uint64_t more = shfl_u64(m, from);
        if (up) m |= more;
    });
    return m;
}

}  // namespace nats

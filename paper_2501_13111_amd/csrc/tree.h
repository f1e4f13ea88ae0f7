// A drafted tree of a chunk: node i of a sequence (its row i) names an earlier node as its parent.
#pragma once
#include "paged.h"

namespace fpk {

constexpr int TREE_MAX = 64;               // nodes of a sequence

// Lane i: the nodes from the root down to node i of sequence sq, itself among them, as bits.  A parent that is no earlier
// node of the sequence is none: the node follows the context.  Paths double their length each round (p: the ancestor
// that a path has not reached yet), so a tree of depth 4 to 7 takes three rounds of three shuffles.
__device__ __forceinline__ uint64_t tree_lines(const int* parent, const Seq& sq) {
    const int lane = threadIdx.x & 63;
    int p = lane < sq.n ? parent[sq.row0 + lane] : -1;
    if (p >= lane) p = -1;
    uint64_t line = lane < sq.n ? 1ull << lane : 0ull;
    while (__ballot(p >= 0) != 0) {
        const int from = max(p, 0);
        const uint64_t up = __shfl(line, from, 64);
        const int pp = __shfl(p, from, 64);
        if (p >= 0) {
            line |= up;
            p = pp;
        }
    }
    return line;
}

// Of 32 positions, the first `at` past the sequence's context (or before it: at < 0), those that a node with this line sees.
__device__ __forceinline__ uint32_t tree_sees(uint64_t line, int at) {
    if (at >= 0) return at < 64 ? (uint32_t)(line >> at) : 0u;
    return at > -32 ? (uint32_t)(line << -at) | ((1u << -at) - 1u) : 0xFFFFFFFFu;
}

}  // namespace fpk

// The ancestors of a node, from its tree's parents.  Plain C++ as well: tests run it on the host.
#pragma once
#include <cstdint>

#ifdef __CUDACC__
#define READER_BOTH __host__ __device__ __forceinline__
#else
#define READER_BOTH inline
#endif

namespace reader {

// Bits 64 half .. + 63 of the 128 that stand for `node` and its ancestors; the root's parent is -1 (as a byte, 255).  The walk goes to lower nodes alone and ends at
// the first parent that is none: whatever the array holds, it ends, and reads nothing behind parents[node].  (A thread block that has given up a wait may come here
// with parents that were not checked, or not written at all.)
template <typename Parent>
READER_BOTH uint64_t ancestors(const Parent *parents, int node, int half) {
    uint64_t seen = 0;
    for (int n = node;;) {
        if ((n >> 6) == half) seen |= 1ull << (n & 63);
        const int next = parents[n];
        if (next < 0 || next >= n) return seen;
        n = next;
    }
}

}  // namespace reader

// How the attention over the paged 8-bit cache is dealt to CTAs and warps, and which rows of a step belong to which request: the
// index arithmetic of aq_kv8.cu and aq_kv8_attn.cu.  Plain C++ (host and device), so it can be unit-tested without a GPU.
//
// The work is a line of tiles of 32 positions: requests in order, within a request (key/value head, block of query rows), within
// such an item its tiles.  The line is cut into one contiguous run per warp, equal to within a tile; neighbouring warps of a CTA
// hold neighbouring runs.
#pragma once
#include <cstdint>

#ifdef __CUDACC__
#define AQ_HD __host__ __device__ __forceinline__
#else
#define AQ_HD inline
#endif

namespace aq {

// First tile of run i of n runs over `total` tiles (i == n: the end).
AQ_HD uint32_t kv8_run_begin(uint32_t total, uint32_t i, uint32_t n) { return (uint32_t)((uint64_t)total * i / n); }

// The run that holds tile x (x < total): the last one that begins at or before it.
AQ_HD uint32_t kv8_run_of(uint32_t total, uint32_t x, uint32_t n) { return (uint32_t)(((uint64_t)(x + 1u) * n - 1u) / total); }

// Rows of request b in a step of T rows: row_start as the caller gave it, held inside the step whatever it says.
struct Kv8Rows { int first, n; };
AQ_HD Kv8Rows kv8_rows(int start, int next, int T) {
    int a = start < 0 ? 0 : (start > T ? T : start);
    int e = next < a ? a : (next > T ? T : next);
    return Kv8Rows{a, e - a};
}

// Largest b in [0, n) with begin[b] <= x, 0 if there is none (begin ascends; n >= 1).
template <typename T>
AQ_HD int kv8_find(const T* begin, int n, T x) {
    int lo = 0, hi = n;
    while (hi - lo > 1) {
        const int mid = (lo + hi) >> 1;
        if (begin[mid] <= x) lo = mid; else hi = mid;
    }
    return lo;
}

// Partial results of an item that n CTAs share are merged in groups of this many, then the groups' results: what one CTA reads
// grows with the square root of n.
AQ_HD int kv8_merge_group(int n) {
    if (n <= 16) return n;
    int g = 4;
    while (g * g < n) ++g;
    return g;
}

}  // namespace aq

// How the attention over the paged 8-bit cache is dealt to CTAs and warps, which rows of a step belong to which request, and how a
// block's scale is rounded: the whole-number arithmetic of aq_kv8.cu and aq_kv8_attn.cuh.  Plain C++ (host and device), so it can be unit-tested without a GPU.
//
// The work is a line: requests in order, within a request its items (key/value head, block of query rows), of each item first
// KV8_ITEM_COST places for what an item costs beside its tiles (queries in, output out), then its tiles of 32 positions.  The line is
// cut into one contiguous run per warp, equal to within one place; neighbouring warps of a CTA hold neighbouring runs.
#pragma once
#include <cstdint>

#ifdef __CUDACC__
#define AQ_HD __host__ __device__ __forceinline__
#else
#define AQ_HD inline
#endif

namespace aq {

constexpr uint32_t KV8_ITEM_COST = 2;

// CTAs of a launch over a line of `total` places, `warps` warps each, at most `most`: so many that a warp has about a place.
AQ_HD uint32_t kv8_even_ctas(uint32_t total, uint32_t warps, uint32_t most) {
    const uint32_t n = (total + warps - 1u) / warps;
    return n < most ? n : most;
}
// The same over `items` items that may be one CTA's each.  Where there is a CTA for every item and its warps have few tiles of it on average
// (five places), one each: nothing is then merged between CTAs, which costs a chain of trips to memory (32 items of 16 tiles: 12.2 us with two
// CTAs per item).
AQ_HD uint32_t kv8_ctas(uint32_t total, uint32_t items, uint32_t warps, uint32_t most) {
    return items <= most && total <= items * warps * 5u ? items : kv8_even_ctas(total, warps, most);
}

// How a line of `total` places is cut into `n` CTAs' shares (1 <= n <= total): the first `more` have one place more than the others.  One
// division for the cut and one per look-up; a 64-bit quotient here was a microsecond of every small call.
struct Kv8Cut { uint32_t each, more; };
AQ_HD Kv8Cut kv8_cut(uint32_t total, uint32_t n) {
    const uint32_t q = total / n;
    return Kv8Cut{q, total - q * n};
}
AQ_HD uint32_t kv8_begin(const Kv8Cut& c, uint32_t i) { return c.each * i + (i < c.more ? i : c.more); }   // (i == n: the end)
AQ_HD uint32_t kv8_cta_of(const Kv8Cut& c, uint32_t x) {
    const uint32_t longer = c.more * (c.each + 1u);
    return x < longer ? x / (c.each + 1u) : c.more + (x - longer) / c.each;
}
// Whether no item need be shared by CTAs: an item of so many tiles at most makes a CTA's share longer by a few tiles per warp, or by a
// sixteenth, and spares the merge between CTAs.
AQ_HD uint32_t kv8_whole_items(const Kv8Cut& c, uint32_t warps) {
    const uint32_t few = 4u * warps, part = c.each / 16u;
    return few > part ? few : part;
}
// Whether items, the longest of so many tiles, are one CTA's each where kv8_ctas says a CTA per item: all are short (kv8_whole_items of a cut
// into `items` shares) or all alike (the cut then falls between them).
AQ_HD bool kv8_stay_whole(uint32_t total, uint32_t items, uint32_t longest, uint32_t warps) {
    return longest <= 4u * warps || (uint64_t)(longest + KV8_ITEM_COST) * items == total;
}
// CTAs of a launch, whatever the items are.  A long item among short ones, which the average hides, would be shared by CTAs all the same, and
// few of them would run (items of 600 and 39 x 29 tiles: 14.3 us on 40 CTAs, 13.5 so; 100 and 31 x 45: 13.5 and 9.3).
AQ_HD uint32_t kv8_launch(uint32_t total, uint32_t items, uint32_t longest, uint32_t warps, uint32_t most) {
    return kv8_stay_whole(total, items, longest, warps) ? kv8_ctas(total, items, warps, most) : kv8_even_ctas(total, warps, most);
}
// Items that are all alike, on two thirds of the CTAs at least: how many whole ones a CTA gets, for two thirds of the SMs draw the memory's
// whole rate and nothing is then merged between CTAs (256 items of 128 tiles: 49.7 us on 148 CTAs, 46.2 on 128; 120 items: 28.4 and
// 25.1; but 192 items of 282 tiles on 96: 75.1 and 77.9).  0: not so.
AQ_HD uint32_t kv8_alike(uint32_t total, uint32_t items, uint32_t longest, uint32_t most) {
    if ((uint64_t)(longest + KV8_ITEM_COST) * items != total) return 0u;
    const uint32_t each = items <= most ? 1u : (items + most - 1u) / most;
    return (uint64_t)items * 3u >= (uint64_t)each * most * 2u ? each : 0u;
}
// The first item that begins at x or later, of a request whose items begin at `first` and have `len` places each.
AQ_HD uint32_t kv8_snap(uint32_t x, uint32_t first, uint32_t len) { return first + (x - first + len - 1u) / len * len; }

// First place of warp w of W in a CTA's share [a, e).
AQ_HD uint32_t kv8_warp_begin(uint32_t a, uint32_t e, uint32_t w, uint32_t W) { return a + (uint32_t)((uint64_t)(e - a) * w / W); }

// x / d for a divisor that the host knows: m = kv8_magic(d), exact for x * d < 2^32 (d > 1).
AQ_HD uint32_t kv8_magic(uint32_t d) { return d == 1 ? 0u : (uint32_t)(((uint64_t)1 << 32) / d) + 1u; }
AQ_HD uint32_t kv8_div(uint32_t x, uint32_t m) { return m == 0u ? x : (uint32_t)((uint64_t)x * m >> 32); }

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
    if (n <= 14) return n;
    int g = 4;
    while (g * g < n) ++g;
    return g;
}

// Of the pattern x of a binary32 number >= 0: the pattern of the next one of 11 significant bits not below it.  A normal number's 13 last
// bits go; of a subnormal, whose pattern is the number itself in steps of 2^-149, what is behind its first 11 bits.
AQ_HD uint32_t kv8_up11(uint32_t x) {
#ifdef __CUDA_ARCH__
    const int top = 31 - __clz((int)x);
#else
    int top = -1;
    while (top < 31 && x >> (top + 1) != 0u) ++top;
#endif
    const int drop = top > 23 ? 13 : top > 10 ? top - 10 : 0;
    const uint32_t low = (1u << drop) - 1u;
    return (x + low) & ~low;
}

}  // namespace aq

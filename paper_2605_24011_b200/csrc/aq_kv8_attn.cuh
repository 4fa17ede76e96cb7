// Attention of a step's new tokens over the paged 8-bit key/value cache:
//     out[t][h] = sum_p softmax_p(scale q[t][h] . K[p]) V[p],   K[p] = ks code_k[p],  V[p] = vs code_v[p],
// over the positions p of the row's request up to the row's own, ks and vs one float32 per 32 positions and head.
//
// Bound: HBM.  Every key and value is read once, D bytes each; per position and head that is 2 D + 0.25 bytes for 4 D G M flops.
//
// Why whole numbers.  The codes are signed bytes and so is what the tensor core multiplies (mma.sync.m16n8k32, 8-bit in, 32-bit sums,
// as fast per instruction as its binary16 form with half the depth): keys go from the cache to the instruction as they are, values after
// one byte permute per four codes; no code is converted, and the sums of products are exact.  Queries and weights are rounded to 16 bits for
// it, below.  (With both made binary16 first, a tile of 128 dims took
// 706 instructions per warp; the kernel waited for its own arithmetic: 32 x 4096 positions x 8 heads 62.6 us, DRAM 48 % busy.)
//   A tile is 32 positions, the span of one scale, so scales touch the sums and not the operands.  Positions (or dims) are the 16 rows
//   of the instruction and its 8 columns are four query rows in two planes, high and low byte:
//   q^ = rint(q 32639 / max|q|) = 256 hi + lo, off by at most 1/65278 of the row's largest magnitude (a binary16 or bfloat16 q is
//       itself known to 2^-11 or 2^-8 of each element: one under 1/32 of the largest keeps less than binary16 had, under 1/256 than bfloat16).
//       hi and lo sums of a query lie in one lane: S = 256 hi + lo.
//   P = rint(65535 exp2(S - the tile's largest S)): 16 bits against the tile's own largest weight, so a tile loses what lies under
//       1/131070 of that and no tile is lost for being light.  Transposed by movmatrix and split into byte planes by a permute.  sum(P) is a
//       product with ones: the normaliser sums what the values are weighted with.
//   O = al O + 2^-16 vs fac (256 hi + lo) in binary32 (2^-16: the sum of weighted values fits where the values' own sum does); ldmatrix.trans on pairs of bytes gives dims 2g, 2g + 1 of two positions per register.
// A NaN (of a scale, of a query row) travels in the scales: F, fac.
// Every warp has a contiguous run of the line (aq_kv8_runs.h) and streams it through its own cp.async ring without waiting for another
// warp; runs differ by one place at most whatever the requests' lengths are.  What a warp finishes alone it writes; pieces of an item are merged
// over the warps of the CTA in shared memory, then over the CTAs in the scratch by the last CTA to arrive (counters; nobody waits), in two
// levels above 14 CTAs.  All sums go in a fixed order.  Where items are short, or all alike, a CTA's share is of whole ones.
// Measured: 32 requests x 4096 positions, 32 heads on 8 of 128, binary16: 46.7 us, 5.75 TB/s, 0.88 of the copy rate (from the L2 instead of
// HBM it takes 32.8: what remains is the start, the unequal speed of the SMs and the merge in the CTA); one request of 512 positions, 32 heads:
// 7.2 us; 100001 positions, 8 heads of 256 on 1: 24.4 us, ten of them merging 148 CTAs' parts; 61 ragged requests of 3 tokens (12 query rows):
// 63.8 us for 296 MB (57.9 from the L2: held up by the arithmetic, 840 instructions a tile at 46 % of the issue slots).
// Fewer warps are slower where the arithmetic counts (61 ragged requests: 66.3 us with 8), more do not fit the registers (168 each
// with 12: with the walks' state in them 148 us).
// (Included by aq_kv8.cu alone, which has the status word and the host calls.)
#pragma once

namespace aq {

constexpr int KA_TILE = AQ_KV8_BLOCK;                 // positions per tile: the span of a scale
constexpr int KA_MAX_CTAS = 192;

// QT: groups of four query rows.  A warp's ring has HALVES places; a place holds a tile's keys or its values and is filled again with what
// comes HALVES later when it has been used: both when the tile is done where HALVES is even, so that its products and weights are one
// stretch of code (ragged requests 70.1 -> 66.8 us), else the keys' before the weights, so that a half more is under way.
// The first of a run's items may leave a piece.  It goes to one of POOL places beside the ring, by turns; when they are out it takes STEAL
// places of the ring, which is that much shorter from then on (and that warp the CTA's last: without the POOL 66.8 us, with it 64.9).
template <int D, int QT>
struct KaShape {
    static constexpr int WARPS = D == 64 ? (QT <= 2 ? 16 : 12) : D == 128 && QT <= 3 ? 12 : 8;
    static constexpr int HALVES = D == 256 ? 3 : D == 64 || QT <= 3 ? 4 : 6;
    static constexpr int ROWS = 4 * QT;               // query rows of an item
    static constexpr int HALF = KA_TILE * D;          // bytes of a tile's keys (or values)
    static constexpr int PITCH = D + 4;               // floats: a row's O, then its maximum and sum
    static constexpr int SLOT = ROWS * PITCH * 4;     // a piece
    static constexpr bool ONCE = HALVES % 2 == 0;     // a place is for keys or for values: a tile is waited for once
    static constexpr int STEAL = ONCE ? 2 : 1;
    // on a line of 128 bytes (with 16 more for the scale between places 32 x 4096 took 53.0 us, so 49.3)
    static constexpr int PLACE = ((HALF > SLOT / STEAL ? HALF : SLOT / STEAL) + 127) / 128 * 128;
    static constexpr int RING = WARPS * HALVES * PLACE;
    static constexpr int TAGS = WARPS * HALVES * 8;   // a place's scale and, with keys, whether the tile may be read
    static constexpr int MERGE = ROWS * 32 * 12;      // a weight, a maximum and a sum per row and part
    static constexpr int FITS = (232448 - 2600 - RING - TAGS - MERGE) / SLOT, POOL = FITS < WARPS ? FITS : WARPS;   // places for pieces beside the ring
    static constexpr int SMEM = RING + MERGE + POOL * SLOT + TAGS;
    static_assert((AQ_KV8_MAX_SEQS + 1) * 4 <= RING && 14 * SLOT <= RING, "the line's marks, and the parts of a group, lie in the ring");
    static_assert(HALVES - STEAL >= 2 && (STEAL == 1 || HALVES % 2 == 0) && 2 * WARPS <= 32, "places can be spared; a lane per piece");
    static_assert(SMEM + 2600 <= 232448 && SLOT % 16 == 0, "shared memory of an SM");
};
// scratch: tickets [2][KA_MAX_CTAS], parts [KA_MAX_CTAS][4][rows][pitch]
constexpr size_t KA_TICKET_BYTES = 2 * KA_MAX_CTAS * 4;
static_assert(KA_TICKET_BYTES % 16 == 0 && KA_TICKET_BYTES + (size_t)KA_MAX_CTAS * 4 * KaShape<128, 4>::SLOT <= AQ_KV8_SCRATCH_BYTES &&
              KA_TICKET_BYTES + (size_t)KA_MAX_CTAS * 4 * KaShape<256, 2>::SLOT <= AQ_KV8_SCRATCH_BYTES, "scratch");

struct KaArgs {
    const void* q;
    void* out;
    const uint8_t* kc;
    const uint8_t* vc;
    const float* ks;
    const float* vs;
    const int32_t* lens;
    const int32_t* row_start;   // or null: n_each rows per request
    const int32_t* table;
    int64_t width, n_pages, q_row, out_row;
    int B, T, n_each, Hkv, G;
    int shift;                  // log2(tiles per page)
    uint32_t G_magic;           // for divisions by G
    int q_bf16, out_dtype;
    float scale_log2;           // scale log2(e)
    unsigned* tickets;
    uint8_t* part;
};

__device__ __forceinline__ void ka_cp16(uint32_t dst, const void* src) {
    asm volatile("cp.async.cg.shared.global [%0], [%1], 16;" ::"r"(dst), "l"(src) : "memory");
}
__device__ __forceinline__ void ka_cp4(uint32_t dst, const void* src) {
    asm volatile("cp.async.ca.shared.global [%0], [%1], 4;" ::"r"(dst), "l"(src) : "memory");
}
__device__ __forceinline__ void ka_commit() { asm volatile("cp.async.commit_group;" ::: "memory"); }
template <int N> __device__ __forceinline__ void ka_wait() { asm volatile("cp.async.wait_group %0;" ::"n"(N) : "memory"); }
__device__ __forceinline__ void ka_ldm(uint32_t addr, uint32_t (&r)[4]) {
    asm volatile("ldmatrix.sync.aligned.m8n8.x4.shared.b16 {%0, %1, %2, %3}, [%4];"
                 : "=r"(r[0]), "=r"(r[1]), "=r"(r[2]), "=r"(r[3]) : "r"(addr) : "memory");
}
__device__ __forceinline__ void ka_ldm_t(uint32_t addr, uint32_t (&r)[4]) {
    asm volatile("ldmatrix.sync.aligned.m8n8.x4.trans.shared.b16 {%0, %1, %2, %3}, [%4];"
                 : "=r"(r[0]), "=r"(r[1]), "=r"(r[2]), "=r"(r[3]) : "r"(addr) : "memory");
}
__device__ __forceinline__ uint32_t ka_transpose(uint32_t a) {
    uint32_t d;
    asm("movmatrix.sync.aligned.m8n8.trans.b16 %0, %1;" : "=r"(d) : "r"(a));
    return d;
}
// signed rows x signed columns, signed rows x unsigned columns
__device__ __forceinline__ void ka_mma_ss(int (&c)[4], const uint32_t (&a)[4], uint32_t b0, uint32_t b1) {
    asm("mma.sync.aligned.m16n8k32.row.col.s32.s8.s8.s32 {%0,%1,%2,%3}, {%4,%5,%6,%7}, {%8,%9}, {%0,%1,%2,%3};"
        : "+r"(c[0]), "+r"(c[1]), "+r"(c[2]), "+r"(c[3]) : "r"(a[0]), "r"(a[1]), "r"(a[2]), "r"(a[3]), "r"(b0), "r"(b1));
}
__device__ __forceinline__ void ka_mma_su(int (&c)[4], const uint32_t (&a)[4], uint32_t b0, uint32_t b1) {
    asm("mma.sync.aligned.m16n8k32.row.col.s32.s8.u8.s32 {%0,%1,%2,%3}, {%4,%5,%6,%7}, {%8,%9}, {%0,%1,%2,%3};"
        : "+r"(c[0]), "+r"(c[1]), "+r"(c[2]), "+r"(c[3]) : "r"(a[0]), "r"(a[1]), "r"(a[2]), "r"(a[3]), "r"(b0), "r"(b1));
}
__device__ __forceinline__ float ka_exp2(float x) {   // 2 ulp; results below 2^-126 are 0
    float y;
    asm("ex2.approx.ftz.f32 %0, %1;" : "=f"(y) : "f"(x));
    return y;
}
// o = f x + o and o = f o, two at a time
__device__ __forceinline__ void ka_fma2(float (&o)[2], float x0, float x1, float f) {
    asm("{.reg .b64 a, b, c;\n mov.b64 a, {%2, %3};\n mov.b64 b, {%4, %4};\n mov.b64 c, {%0, %1};\n fma.rn.f32x2 c, a, b, c;\n mov.b64 {%0, %1}, c;}"
        : "+f"(o[0]), "+f"(o[1]) : "f"(x0), "f"(x1), "f"(f));
}
__device__ __forceinline__ void ka_mul2(float (&o)[2], float f) {
    asm("{.reg .b64 b, c;\n mov.b64 b, {%2, %2};\n mov.b64 c, {%0, %1};\n mul.rn.f32x2 c, c, b;\n mov.b64 {%0, %1}, c;}"
        : "+f"(o[0]), "+f"(o[1]) : "f"(f));
}
// Byte offset of 16-byte piece c of row r in a tile: rows of eight that ldmatrix reads together fall on different banks.
template <int D>
__device__ __forceinline__ uint32_t ka_at(int r, int c) {
    const int x = D == 64 ? c ^ ((r >> 1) & 3) : c ^ (r & 7);
    return (uint32_t)(r * D + x * 16);
}

// A request of the line.
struct KaSeq {
    int b, L, row0, n, nt, rb;   // L: as the caller says; nt: tiles of an item, those that the table has room for; rb: items per key/value head
};
__device__ __forceinline__ KaSeq ka_seq(const KaArgs& a, int b, int rows) {
    KaSeq s;
    s.b = b;
    const Kv8Rows r = a.row_start ? kv8_rows(a.row_start[b], a.row_start[b + 1], a.T) : Kv8Rows{b * a.n_each, a.n_each};
    s.row0 = r.first;
    s.n = r.n;
    s.L = max(a.lens[b], 0);   // (rows' positions follow from it, as the append has them, whether they fit or not)
    const int held = min(s.L, (int)a.width << (a.shift + 5));   // (2^30 at most)
    s.nt = max(1, (held + KA_TILE - 1) / KA_TILE);   // (a request without positions has one tile that is not read: its rows become 0)
    s.rb = (s.n * a.G + rows - 1) / rows;   // (n G <= 2^20)
    return s;
}

// Whether a request has rows and a length that the table has no room for, or a negative one.
__device__ __forceinline__ bool ka_too_long(const KaSeq& s, int len) { return s.n > 0 && (len < 0 || s.L > s.nt * KA_TILE); }

__device__ __forceinline__ uint32_t ka_places(const KaArgs& a, const KaSeq& s) {
    return ((uint32_t)s.nt + KV8_ITEM_COST) * (uint32_t)s.rb * (uint32_t)a.Hkv;
}

// A piece of an item as it is put down for merging.
struct KaPiece {
    uint32_t first;   // the place of the item's first tile on the line
    int nt;           // its tiles (0: no piece here)
    int row0, rows;   // first row of the request, its query rows (G n)
    int hk, q0;       // key/value head, the item's first query row
    uint32_t at;      // where in shared memory
};

// N neighbouring values as the output's type
template <int N>
__device__ __forceinline__ void ka_store(const KaArgs& a, int64_t at, const float (&x)[N]) {
#pragma unroll
    for (int i = 0; i < N; i += 2) {
        if (a.out_dtype == AQ_F32) *reinterpret_cast<float2*>(reinterpret_cast<float*>(a.out) + at + i) = make_float2(x[i], x[i + 1]);
        else if (a.out_dtype == AQ_F16) *reinterpret_cast<__half2*>(reinterpret_cast<__half*>(a.out) + at + i) = __floats2half2_rn(x[i], x[i + 1]);
        else *reinterpret_cast<__nv_bfloat162*>(reinterpret_cast<__nv_bfloat16*>(a.out) + at + i) = __floats2bfloat162_rn(x[i], x[i + 1]);
    }
}
__device__ __forceinline__ int64_t ka_out_at(const KaArgs& a, int row0, int hk, int q, int D) {
    const int tok = (int)kv8_div((uint32_t)q, a.G_magic);
    return (int64_t)(row0 + tok) * a.out_row + (int64_t)(hk * a.G + (q - tok * a.G)) * D;
}
// 2^16 over the normaliser (O was summed with 2^-16); a row that saw nothing is 0
__device__ __forceinline__ float ka_norm(float l) { return l == 0.f ? 0.f : 1.f / l * 65536.f; }

// Arrives at an item's (or a group's) counter: whether this was the last of `want`, who puts it back to zero.  What the CTA wrote before
// the barrier in front of this is visible to whoever arrives later, and what earlier ones wrote to this CTA after the next barrier.
__device__ __forceinline__ bool ka_arrive(unsigned* ticket, unsigned one, unsigned want) {
    unsigned was;
    asm volatile("atom.acq_rel.gpu.global.add.u32 %0, [%1], %2;" : "=r"(was) : "l"(ticket), "r"(one) : "memory");
    const bool last = (one == 1u ? was & 0xffffu : was >> 16) == want - 1u;
    if (last) atomicSub(ticket, one * want);
    return last;
}

template <int D, int QT>
__global__ void __launch_bounds__(KaShape<D, QT>::WARPS * 32, 1) kv8_attn_kernel(const __grid_constant__ KaArgs a) {
    using S = KaShape<D, QT>;
    constexpr int W = S::WARPS, ROWS = S::ROWS;
    extern __shared__ __align__(128) uint8_t smem[];
    __shared__ KaPiece pieces[2 * W];
    __shared__ uint32_t sums[W][4];
    __shared__ int last_flag[2], group_head[32];
    __shared__ KaSeq seqs[2 * W];   // the requests that a warp's copies and its products are at (kept out of the registers)
    __shared__ KaPiece at_work[W];
    __shared__ int pool_used;
    const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
    const int g = lane >> 2, t = lane & 3;

    // ---- the line: first place of each request ---------------------------------------------------------------
    if constexpr (S::POOL < W) {
        if (threadIdx.x == 0) pool_used = 0;
        __syncthreads();
    }
    pdl_wait();
    pdl_launch_dependents();
    if (lane < 2) pieces[2 * warp + lane].nt = 0;
    uint32_t total, items, longest;   // of the line: places, items, tiles of the longest item
    KaSeq sq{};
    uint32_t off = 0;             // the run's first place in its request
    uint32_t c0 = 0, c1 = 0, x0 = 0, x1 = 0;   // the CTA's share, the warp's run
    Kv8Cut cut{};
    bool whole_items = false;     // every item belongs to the CTA whose share holds its first place
    auto my_run = [&] {
        const uint32_t n = kv8_launch(total, items, longest, W, gridDim.x);
        const uint32_t each = n == gridDim.x ? kv8_alike(total, items, longest, n) : 0u;   // (fewer: there is a CTA per item, or a place per warp)
        cut = each ? Kv8Cut{each * (longest + KV8_ITEM_COST), 0u} : kv8_cut(total, n);
        c0 = min(kv8_begin(cut, blockIdx.x), total);
        c1 = min(kv8_begin(cut, blockIdx.x + 1), total);
        whole_items = each != 0u || longest <= kv8_whole_items(cut, W);
    };
    auto cut_warps = [&] {   // (the places in front of the first tile of a share that begins with an item are no warp's work)
        const uint32_t a0 = whole_items ? min(c0 + KV8_ITEM_COST, c1) : c0;
        x0 = kv8_warp_begin(a0, c1, warp, W);
        x1 = kv8_warp_begin(a0, c1, warp + 1, W);
    };
    // Row marks that descend can name more rows than the step has, and the line would be longer than the host could know (it counts in 32
    // bits, and `total` may be anything, 0 too): such a step is not followed.
    auto too_many = [&](uint32_t rows) {
        if (rows <= (uint32_t)a.T) return false;
        if (blockIdx.x == 0 && threadIdx.x == 0) kv8_report(KV8_BAD_LENGTH);
        return true;
    };
    if (a.B <= 32) {   // a lane per request, in every warp: no warp waits for another
        KaSeq s{};
        if (lane < a.B) {
            s = ka_seq(a, lane, ROWS);
            if (ka_too_long(s, a.lens[lane])) kv8_report(KV8_BAD_LENGTH);
        }
        const uint32_t mine = ka_places(a, s);
        total = __reduce_add_sync(0xffffffffu, mine);
        items = __reduce_add_sync(0xffffffffu, (unsigned)(s.rb * a.Hkv));
        longest = __reduce_max_sync(0xffffffffu, s.n > 0 ? (unsigned)s.nt : 0u);
        if (too_many(__reduce_add_sync(0xffffffffu, (unsigned)s.n)) || total == 0) return;
        uint32_t upto = mine;
#pragma unroll
        for (int d = 1; d < 32; d <<= 1) {
            const uint32_t v = __shfl_up_sync(0xffffffffu, upto, d);
            if (lane >= d) upto += v;
        }
        my_run();
        if (c0 >= total) return;
        if (whole_items) {
            auto snap = [&](uint32_t x) -> uint32_t {
                const unsigned at = __ballot_sync(0xffffffffu, upto - mine <= x && x < upto);
                if (!at) return x;   // (the line's end)
                const int b = __ffs(at) - 1;
                return kv8_snap(x, __shfl_sync(0xffffffffu, upto - mine, b), (uint32_t)__shfl_sync(0xffffffffu, s.nt, b) + KV8_ITEM_COST);
            };
            c0 = snap(c0);
            c1 = snap(c1);
        }
        cut_warps();
        const unsigned here = __ballot_sync(0xffffffffu, upto - mine <= x0 && x0 < upto);
        if (here) {
            const int b = __ffs(here) - 1;
            off = x0 - __shfl_sync(0xffffffffu, upto - mine, b);
            sq.b = b;
            sq.L = __shfl_sync(0xffffffffu, s.L, b); sq.row0 = __shfl_sync(0xffffffffu, s.row0, b); sq.n = __shfl_sync(0xffffffffu, s.n, b);
            sq.nt = __shfl_sync(0xffffffffu, s.nt, b); sq.rb = __shfl_sync(0xffffffffu, s.rb, b);
        }
    } else {
        uint32_t* marks = reinterpret_cast<uint32_t*>(smem);
        const int per = (a.B + W * 32 - 1) / (W * 32), b0 = threadIdx.x * per;
        uint32_t mine = 0, my_items = 0, my_longest = 0, my_rows = 0;
        for (int b = b0; b < min(b0 + per, a.B); ++b) {
            const KaSeq s = ka_seq(a, b, ROWS);
            if (s.n > 0) my_longest = max(my_longest, (uint32_t)s.nt);
            if (ka_too_long(s, a.lens[b])) kv8_report(KV8_BAD_LENGTH);
            mine += ka_places(a, s);
            my_rows += (uint32_t)s.n;
            my_items += (uint32_t)s.rb * (uint32_t)a.Hkv;
        }
        uint32_t upto = mine;
#pragma unroll
        for (int d = 1; d < 32; d <<= 1) {
            const uint32_t v = __shfl_up_sync(0xffffffffu, upto, d), w = __shfl_up_sync(0xffffffffu, my_items, d);
            if (lane >= d) { upto += v; my_items += w; }
        }
        my_longest = __reduce_max_sync(0xffffffffu, my_longest);
        my_rows = __reduce_add_sync(0xffffffffu, my_rows);
        if (lane == 31) { sums[warp][0] = upto; sums[warp][1] = my_items; sums[warp][2] = my_longest; sums[warp][3] = my_rows; }
        __syncthreads();
        uint32_t before = upto - mine;
        total = items = longest = 0;
        uint32_t rows = 0;
        for (int w = 0; w < W; ++w) {
            if (w < warp) before += sums[w][0];
            total += sums[w][0];
            items += sums[w][1];
            longest = max(longest, sums[w][2]);
            rows += sums[w][3];
        }
        if (too_many(rows) || total == 0) return;
        for (int b = b0; b < min(b0 + per, a.B); ++b) {
            marks[b] = before;
            before += ka_places(a, ka_seq(a, b, ROWS));
        }
        my_run();
        if (c0 >= total) return;
        __syncthreads();
        if (whole_items) {
            auto snap = [&](uint32_t x) -> uint32_t {
                if (x >= total) return x;
                const int b = kv8_find(marks, a.B, x);
                return kv8_snap(x, marks[b], (uint32_t)ka_seq(a, b, ROWS).nt + KV8_ITEM_COST);
            };
            c0 = snap(c0);
            c1 = snap(c1);
        }
        cut_warps();
        if (x0 < x1) {
            const int b = kv8_find(marks, a.B, x0);
            sq = ka_seq(a, b, ROWS);
            off = x0 - marks[b];
        }
        __syncthreads();   // (the marks lie where tiles will)
    }
    int item = 0, j = 0;          // item of the request (head x block of rows), tile of the item
    if (x0 < x1) {
        const uint32_t len = (uint32_t)sq.nt + KV8_ITEM_COST;
        item = (int)(off / len);
        off -= (uint32_t)item * len;
        if (off < KV8_ITEM_COST) x0 += KV8_ITEM_COST - off;   // (its first tile; past x1 if the run has none)
        else j = (int)(off - KV8_ITEM_COST);
    }

    const uint32_t my_ring = (uint32_t)(warp * S::HALVES * S::PLACE), ring = (uint32_t)__cvta_generic_to_shared(smem) + my_ring;
    const uint32_t tags = (uint32_t)__cvta_generic_to_shared(smem) + S::SMEM - S::TAGS + warp * S::HALVES * 8;

    if (x0 < x1) {
        // ---- copies: a walk of its own, HALVES halves ahead --------------------------------------------------
        KaSeq& ps = seqs[2 * warp];
        KaSeq& cs = seqs[2 * warp + 1];
        if (lane == 0) ps = cs = sq;
        __syncwarp();
        int p_item = item, p_j = j, p_page0 = -1, p_pages = -1;   // lane i holds the number of page p_page0 + i
        int nt = sq.nt;
        uint32_t p_x = x0;
        auto next_item = [&](KaSeq& s, int& it) {   // whether the request is another one now
            if (++it < s.rb * a.Hkv) return false;
            it = 0;
            int b = s.b;
            KaSeq to;
            do { to = ka_seq(a, ++b, ROWS); } while (to.n == 0 && b + 1 < a.B);   // (x < total: there is one)
            __syncwarp();
            if (lane == 0) s = to;
            __syncwarp();
            return true;
        };
        auto touch_queries = [&](const KaSeq& s, int it) {   // a line per lane, so that they are near when the item's turn comes
            constexpr int LINES = D * 2 / 128;
            const int hk = s.rb == 1 ? it : it / s.rb, r = (it - hk * s.rb) * ROWS + lane / LINES;
            if (lane < ROWS * LINES && r < a.G * s.n) {
                const int tok = (int)kv8_div((uint32_t)r, a.G_magic);
                const uint16_t* q = reinterpret_cast<const uint16_t*>(a.q) + (int64_t)(s.row0 + tok) * a.q_row + (int64_t)(hk * a.G + (r - tok * a.G)) * D;
                asm volatile("prefetch.global.L1 [%0];" ::"l"(q + (lane % LINES) * 64));
            }
        };
        // an item's query rows as they come: of row 4 u + g / 2, dims 32 c + 4 t .. and 16 further.  The first item's are asked for before its
        // tiles where there are registers for that.
        constexpr bool EARLY = QT <= 2;
        uint2 raw[EARLY ? QT : 1][D / 32][2];
        auto load_queries = [&](const KaSeq& s, int it, int u0) {
            const int hk = s.rb == 1 ? it : it / s.rb, q0 = (it - hk * s.rb) * ROWS;
#pragma unroll
            for (int u = 0; u < (EARLY ? QT : 1); ++u) {
                const int r = q0 + 4 * (u + u0) + (g >> 1);
                if (r < a.G * s.n) {
                    const int tok = (int)kv8_div((uint32_t)r, a.G_magic);
                    const uint16_t* q = reinterpret_cast<const uint16_t*>(a.q) + (int64_t)(s.row0 + tok) * a.q_row +
                                        (int64_t)(hk * a.G + (r - tok * a.G)) * D + 4 * t;
#pragma unroll
                    for (int c = 0; c < D / 32; ++c) {
                        raw[u][c][0] = *reinterpret_cast<const uint2*>(q + 32 * c);
                        raw[u][c][1] = *reinterpret_cast<const uint2*>(q + 32 * c + 16);
                    }
                } else {
#pragma unroll
                    for (int c = 0; c < D / 32; ++c) raw[u][c][0] = raw[u][c][1] = make_uint2(0u, 0u);
                }
            }
        };
        if constexpr (EARLY) load_queries(cs, item, 0);       // (under way while the first tiles' pages are looked up)
        bool p_ok = false;
        int64_t p_blk = 0;
        auto copy = [&](uint32_t dst, uint32_t tag, const uint8_t* codes, const float* scales) {   // a tile's keys or values, and their scale
            const uint8_t* src = codes + p_blk * S::HALF + lane * 16;
            // (the rows' pattern repeats every eight: a few offsets of the lane, the rest is known when this is compiled)
            constexpr int RPP = 512 / D, REP = RPP >= 8 ? 1 : 8 / RPP;
#pragma unroll
            for (int i = 0; i < S::HALF / 512; ++i)
                ka_cp16(dst + ka_at<D>(lane / (D / 16) + i % REP * RPP, lane % (D / 16)) + i / REP * (REP * 512), src + i * 512);
            if (lane == 0) ka_cp4(tag, scales + p_blk);
        };
        bool p_values = false;   // what is due: a tile's keys, or the values of the tile whose keys came last
        auto issue = [&](int st, bool values) {
            if (values && !p_values) return;   // (the run has no more tiles)
            const uint32_t dst = ring + (uint32_t)(st * S::PLACE), tag = tags + (uint32_t)(st * 8);
            if (!values) {
                if (p_x >= x1) return;
                const int pg = p_j >> a.shift;
                if (p_page0 < 0 || pg >= p_page0 + 32 || pg < p_page0) {
                    p_page0 = pg;
                    const int i = pg + lane;
                    p_pages = (int64_t)i < a.width && (i << (a.shift + 5)) < ps.L ? a.table[(int64_t)ps.b * a.width + i] : -1;
                }
                const int page = __shfl_sync(0xffffffffu, p_pages, pg - p_page0);
                p_ok = page >= 0 && page < a.n_pages;
                const int hk = ps.rb == 1 ? p_item : p_item / ps.rb;
                p_blk = (((int64_t)page * a.Hkv + hk) << a.shift) + (p_j & ((1 << a.shift) - 1));
                if (!p_ok && ps.L > 0 && lane == 0) kv8_report(KV8_BAD_PAGE);
                if (lane == 1) asm volatile("st.shared.u32 [%0], %1;" ::"r"(tag + 4), "r"(p_ok ? 1 : 0) : "memory");
            }
            if (p_ok) copy(dst, tag, values ? a.vc : a.kc, values ? a.vs : a.ks);
            if (values) {
                ++p_x;
                if (++p_j == ps.nt) {
                    p_x += KV8_ITEM_COST;
                    if (p_x < x1) {
                        p_j = 0;
                        if (next_item(ps, p_item)) p_page0 = -1;
                        touch_queries(ps, p_item);
                    }
                }
            }
            p_values = !values;
        };
#pragma unroll 1
        for (int s = 0; s < S::HALVES; ++s) {
            issue(s, S::ONCE ? (s & 1) != 0 : p_values);
            ka_commit();
        }

        uint32_t qf[QT][D / 32][2];
        float o[QT][D / 16][2];       // of query row 4 u + t: dims 16 c + 2 g and the next
        float m[QT], l[QT], fq[QT];
        int lim[QT], lim_min = 0;
        uint32_t first = 0;           // the place of the item's first tile
        bool fresh = true;
        int kst = 0, gone = -1;       // the place of the tile's keys; the first one that a piece has taken
        auto after = [&](int st) {
            st = st + 1 == S::HALVES ? 0 : st + 1;
            if (st == gone) st = st + S::STEAL >= S::HALVES ? st + S::STEAL - S::HALVES : st + S::STEAL;
            return st;
        };
        for (uint32_t x = x0; x < x1;) {
            if (fresh) {   // ---- another item: its queries
                fresh = false;
                __syncwarp();   // (every lane has read the piece before)
                const KaSeq sq = cs;
                KaPiece pc;
                pc.first = first = x - (uint32_t)j;
                pc.nt = nt = sq.nt;
                pc.row0 = sq.row0;
                pc.rows = a.G * sq.n;
                pc.hk = sq.rb == 1 ? item : item / sq.rb;
                pc.q0 = (item - pc.hk * sq.rb) * ROWS;
                pc.at = 0;
                if (lane == 0) at_work[warp] = pc;
                // operand column g of a group of four rows: row g / 2, plane g % 2
                if constexpr (EARLY) { if (x != x0) load_queries(cs, item, 0); }
#pragma unroll
                for (int u = 0; u < QT; ++u) {
                    if constexpr (!EARLY) load_queries(cs, item, u);
                    constexpr int U = EARLY ? 1 : 0;   // (whether raw holds all groups)
                    // magnitudes as whole numbers: of two values of one type the larger has the larger pattern, a NaN the largest
                    uint32_t most = 0;
#pragma unroll
                    for (int c = 0; c < D / 32; ++c)
#pragma unroll
                        for (int h = 0; h < 2; ++h) most = __vmaxu2(most, __vmaxu2(raw[u * U][c][h].x & 0x7fff7fffu, raw[u * U][c][h].y & 0x7fff7fffu));
                    most = __vmaxu2(most, __shfl_xor_sync(0xffffffffu, most, 1));
                    most = __vmaxu2(most, __shfl_xor_sync(0xffffffffu, most, 2));
                    most = max(most & 0xffffu, most >> 16);
                    const bool poison = most >= (a.q_bf16 ? 0x7f80u : 0x7c00u);
                    const float big = a.q_bf16 ? __uint_as_float(most << 16) : __half2float(__ushort_as_half((unsigned short)most));
                    // (a row under 1.1e-34, which bfloat16 can hold, is in steps of 1 / 3e38; rows of zeros are too)
                    const float up = poison ? 0.f : fminf(32639.f / big, 3e38f);
                    // q up + 1.5 * 2^23 has rint(q up) in its low bits; 128 more, and the second byte is the high plane's
                    const float magic = 12582912.f + ((g & 1) ? 0.f : 128.f);
                    const uint32_t pick = (g & 1) ? 0x0040 : 0x0051;
                    auto planes = [&](float y0, float y1, float y2, float y3) -> uint32_t {
                        const uint32_t n0 = __float_as_uint(fmaf(y0, up, magic)), n1 = __float_as_uint(fmaf(y1, up, magic));
                        const uint32_t n2 = __float_as_uint(fmaf(y2, up, magic)), n3 = __float_as_uint(fmaf(y3, up, magic));
                        return __byte_perm(__byte_perm(n0, n1, pick), __byte_perm(n2, n3, pick), 0x5410);
                    };
                    if (a.q_bf16) {
                        auto w = [](uint32_t v) { return make_float2(__uint_as_float(v << 16), __uint_as_float(v & 0xffff0000u)); };
#pragma unroll
                        for (int c = 0; c < D / 32; ++c)
#pragma unroll
                            for (int h = 0; h < 2; ++h) {
                                const float2 e = w(raw[u * U][c][h].x), f = w(raw[u * U][c][h].y);
                                qf[u][c][h] = planes(e.x, e.y, f.x, f.y);
                            }
                    } else {
#pragma unroll
                        for (int c = 0; c < D / 32; ++c)
#pragma unroll
                            for (int h = 0; h < 2; ++h) {
                                const float2 e = __half22float2(*reinterpret_cast<const __half2*>(&raw[u * U][c][h].x));
                                const float2 f = __half22float2(*reinterpret_cast<const __half2*>(&raw[u * U][c][h].y));
                                qf[u][c][h] = planes(e.x, e.y, f.x, f.y);
                            }
                    }
                    // of the query row whose scores this lane holds (row t of the group: lanes of columns 2t and 2t + 1 have it)
                    const float step = poison ? __uint_as_float(0x7fc00000u) : up < 3e38f ? big * (1.f / 32639.f) : 1.f / 3e38f;
                    fq[u] = __shfl_sync(0xffffffffu, step, 8 * t) * a.scale_log2;
                    lim[u] = sq.L - sq.n + (int)kv8_div((uint32_t)min(pc.q0 + 4 * u + t, pc.rows - 1), a.G_magic) + 1;   // positions before this one are seen
                    m[u] = -INFINITY;
                    l[u] = 0.f;
#pragma unroll
                    for (int c = 0; c < D / 16; ++c) o[u][c][0] = o[u][c][1] = 0.f;
                }
                lim_min = sq.L - sq.n + (int)kv8_div((uint32_t)pc.q0, a.G_magic) + 1;
            }

            const bool item_ends = j + 1 == nt;
            const uint32_t next = x + 1 + (item_ends ? KV8_ITEM_COST : 0u);
            const bool run_ends = next >= x1, whole = item_ends && first >= x0, take = item_ends && !run_ends && !whole;
            constexpr int USED = S::ONCE ? 2 : 1;
            if (gone < 0) ka_wait<S::HALVES - USED>(); else ka_wait<S::HALVES - USED - S::STEAL>();
            __syncwarp();   // every lane's copies of the keys have landed
            const int vst = after(kst);
            const uint32_t kt = ring + (uint32_t)(kst * S::PLACE), vt = ring + (uint32_t)(vst * S::PLACE);
            float ks;
            int ok;
            asm volatile("ld.shared.f32 %0, [%1];" : "=f"(ks) : "r"(tags + (uint32_t)(kst * 8)) : "memory");
            asm volatile("ld.shared.s32 %0, [%1];" : "=r"(ok) : "r"(tags + (uint32_t)(kst * 8) + 4) : "memory");
            // (ok is the same for all lanes; a tile that could not be read counts as masked)
            int sc[QT][2][4];
            if (ok) {
                // ---- S = K q: 32 positions x 4 QT query rows x 2 planes
#pragma unroll
                for (int u = 0; u < QT; ++u)
#pragma unroll
                    for (int mt = 0; mt < 2; ++mt) sc[u][mt][0] = sc[u][mt][1] = sc[u][mt][2] = sc[u][mt][3] = 0;
#pragma unroll
                for (int c = 0; c < D / 32; ++c) {
#pragma unroll
                    for (int mt = 0; mt < 2; ++mt) {
                        uint32_t r[4];
                        ka_ldm(kt + ka_at<D>(16 * mt + ((lane >> 3) & 1) * 8 + (lane & 7), 2 * c + (lane >> 4)), r);
#pragma unroll
                        for (int u = 0; u < QT; ++u) ka_mma_ss(sc[u][mt], r, qf[u][c][0], qf[u][c][1]);
                    }
                }
            }
            if constexpr (!S::ONCE) {
                __syncwarp();   // every lane is through with the keys
                issue(kst, p_values);
                ka_commit();
                if (gone < 0) ka_wait<S::HALVES - 1>(); else ka_wait<S::HALVES - 1 - S::STEAL>();
                __syncwarp();   // every lane's copies of the values have landed
            }
            if (ok) {
                float vs;
                asm volatile("ld.shared.f32 %0, [%1];" : "=f"(vs) : "r"(tags + (uint32_t)(vst * 8)) : "memory");
                vs *= 0x1p-16f;
                // ---- weights
                const int pos = j * KA_TILE;
                const bool all_seen = pos + KA_TILE <= lim_min;
                // (Step by step over all groups, each step in one block of code: with the masks' branches inside a loop over groups the warp waited
                // for one group after the other.)
                uint32_t pb[QT][2];
                float al[QT], vf[QT];
                int s[QT][4], top[QT];   // positions g, g + 8, g + 16, g + 24 of row t
#pragma unroll
                for (int u = 0; u < QT; ++u)
#pragma unroll
                    for (int i = 0; i < 4; ++i) s[u][i] = sc[u][i >> 1][2 * (i & 1)] * 256 + sc[u][i >> 1][2 * (i & 1) + 1];
                constexpr int NONE = -0x7fffffff - 1;   // (no score is so low: |S| <= 256 * 128 * 32639)
                if (!all_seen) {
#pragma unroll
                    for (int u = 0; u < QT; ++u)
#pragma unroll
                        for (int i = 0; i < 4; ++i) s[u][i] = pos + 8 * i + g < lim[u] ? s[u][i] : NONE;
                }
#pragma unroll
                for (int u = 0; u < QT; ++u) top[u] = max(max(s[u][0], s[u][1]), max(s[u][2], s[u][3]));
#pragma unroll
                for (int d = 4; d < 32; d <<= 1)
#pragma unroll
                    for (int u = 0; u < QT; ++u) top[u] = max(top[u], __shfl_xor_sync(0xffffffffu, top[u], d));
                uint32_t p[QT][4];   // the low half: rint(65535 weight)
#pragma unroll
                for (int u = 0; u < QT; ++u) {
                    const float F = ks * fq[u];
#pragma unroll
                    for (int i = 0; i < 4; ++i) {
                        const float w = ka_exp2((float)(int)((uint32_t)s[u][i] - (uint32_t)top[u]) * F);
                        p[u][i] = __float_as_uint(fmaf(w, 65535.f, 8388608.f));
                    }
                }
                if (!all_seen) {
#pragma unroll
                    for (int u = 0; u < QT; ++u)
#pragma unroll
                        for (int i = 0; i < 4; ++i) p[u][i] = s[u][i] == NONE ? 0u : p[u][i];
                }
                bool moved = false;
#pragma unroll
                for (int u = 0; u < QT; ++u) {
                    int lt[4] = {0, 0, 0, 0};
                    const uint32_t ones[4] = {0x01010101u, 0x01010101u, 0x01010101u, 0x01010101u};
#pragma unroll
                    for (int h = 0; h < 2; ++h) {
                        // columns 2t, 2t + 1: row t's positions g and g + 8; transposed, lane (g, t) has two of the four positions 2t, 2t + 1, 2t + 8,
                        // 2t + 9 of row g / 2 and its neighbour the other two: even g takes the four high bytes, odd g the low ones
                        const uint32_t mine = ka_transpose(__byte_perm(p[u][2 * h], p[u][2 * h + 1], 0x5410));
                        const uint32_t other = __shfl_xor_sync(0xffffffffu, mine, 4);
                        pb[u][h] = __byte_perm(mine, other, (g & 1) ? 0x2064 : 0x7531);
                    }
                    ka_mma_su(lt, ones, pb[u][0], pb[u][1]);
                    const bool any = top[u] != NONE;
                    const float s_top = any ? (float)top[u] * (ks * fq[u]) : -INFINITY;
                    const float now = fmaxf(m[u], s_top);   // (a NaN leaves the maximum; fac carries it into the sums)
                    al[u] = now == -INFINITY ? 1.f : ka_exp2(m[u] - now);
                    const float fac = any ? ka_exp2(s_top - (now == -INFINITY ? 0.f : now)) : 0.f;
                    moved |= now != m[u];
                    m[u] = now;
                    l[u] = fmaf(l[u], al[u], (float)(lt[0] * 256 + lt[1]) * fac);
                    vf[u] = any ? vs * fac : 0.f;   // (what a row does not see cannot reach it, a NaN among it)
                }
                moved = __any_sync(0xffffffffu, moved);
                if (moved) {
#pragma unroll
                    for (int u = 0; u < QT; ++u)
#pragma unroll
                        for (int c = 0; c < D / 16; ++c) ka_mul2(o[u][c], al[u]);
                }
                // ---- O += vs fac V P
#pragma unroll
                for (int c = 0; c < D / 16; ++c) {
                    uint32_t r[4];
                    ka_ldm_t(vt + ka_at<D>(lane, c), r);
                    // rows 0..7 are even dims, 8..15 odd ones; depth: positions 2t, 2t + 1, 2t + 8, 2t + 9, then those + 16
                    const uint32_t v[4] = {__byte_perm(r[0], r[1], 0x6420), __byte_perm(r[0], r[1], 0x7531), __byte_perm(r[2], r[3], 0x6420),
                                           __byte_perm(r[2], r[3], 0x7531)};
#pragma unroll
                    for (int u = 0; u < QT; ++u) {
                        int ot[4] = {0, 0, 0, 0};
                        ka_mma_su(ot, v, pb[u][0], pb[u][1]);
                        ka_fma2(o[u][c], (float)(ot[0] * 256 + ot[1]), (float)(ot[2] * 256 + ot[3]), vf[u]);
                    }
                }
            }
            __syncwarp();   // every lane is through with the values
            bool steal = false;
            uint32_t piece_at = 0;
            if (take) {   // a place for the piece: beside the ring, or else where this tile was
                int k = warp;
                if constexpr (S::POOL < W) {
                    if (lane == 0) k = atomicAdd(&pool_used, 1);
                    k = __shfl_sync(0xffffffffu, k, 0);
                    steal = k >= S::POOL;
                }
                piece_at = (uint32_t)(S::RING + S::MERGE + k * S::SLOT);
            }
            if (S::ONCE && !(steal && S::STEAL == 2)) {
                issue(kst, false);
                ka_commit();
            }
            if (!steal) {
                issue(vst, S::ONCE ? true : p_values);
                ka_commit();
            }

            // ---- the item's end, or the run's
            if (item_ends || run_ends) {
                KaPiece pc = at_work[warp];
                if (whole) {
#pragma unroll
                    for (int u = 0; u < QT; ++u) {
                        const int r = pc.q0 + 4 * u + t;
                        if (r < pc.rows) {
                            const float inv = ka_norm(l[u]);
                            const int64_t at = ka_out_at(a, pc.row0, pc.hk, r, D) + 2 * g;
#pragma unroll
                            for (int c = 0; c < D / 16; ++c) {
                                const float two[2] = {o[u][c][0] * inv, o[u][c][1] * inv};
                                ka_store(a, at + 16 * c, two);
                            }
                        }
                    }
                } else {
                    // the run's first piece, where this tile was, or its last: all copies have been used by then
                    const int to = S::STEAL == 1 ? vst : kst;   // (places of one tile lie side by side where two are wanted)
                    pc.at = take && !steal ? piece_at : my_ring + (uint32_t)(to * S::PLACE);
#pragma unroll
                    for (int u = 0; u < QT; ++u) {
                        float* row = reinterpret_cast<float*>(smem + pc.at) + (4 * u + t) * S::PITCH;
#pragma unroll
                        for (int c = 0; c < D / 16; ++c) *reinterpret_cast<float2*>(row + 16 * c + 2 * g) = make_float2(o[u][c][0], o[u][c][1]);
                        if (g == 0) *reinterpret_cast<float2*>(row + D) = make_float2(m[u], l[u]);
                    }
                    if (lane == 0) pieces[2 * warp + (run_ends ? 1 : 0)] = pc;
                    if (steal) gone = to;
                }
            }
            kst = after(vst);
            if (item_ends) {
                j = 0;
                if (!run_ends) { next_item(cs, item); fresh = true; }
            } else {
                ++j;
            }
            x = next;
        }
        ka_wait<0>();
    }
    __syncthreads();

    // ---- merging ---------------------------------------------------------------------------------------------
    // Up to 32 parts in shared memory, part k at byte my_at of lane k, neighbours of one item in groups that begin at the lanes of `heads`:
    // first every part's weight (a warp per row, a lane per part), then the sums (a thread per four dims).
    float2 (*stat)[32] = reinterpret_cast<float2 (*)[32]>(smem + S::RING);
    float (*weight)[32] = reinterpret_cast<float (*)[32]>(smem + S::RING + ROWS * 32 * 8);
    auto weigh = [&](unsigned there, unsigned heads, uint32_t my_at, int rows) {
        const unsigned upto = heads & ((2u << lane) - 1u), later = heads & ~((2u << lane) - 1u);
        // (its last part's lane, not the lane before the next group: sums then go in an order of the group's own, whatever lies beside it)
        const int lo = upto ? 31 - __clz(upto) : 0, hi = max(31 - __clz((int)(there & (later ? (later & (0u - later)) - 1u : 0xffffffffu))), 0);
        for (int r = warp; r < rows; r += W) {
            float2 ml = make_float2(-INFINITY, 0.f);
            if (there >> lane & 1u) ml = *reinterpret_cast<const float2*>(smem + my_at + (r * S::PITCH + D) * 4);
            float top = ml.x;
#pragma unroll
            for (int d = 1; d < 32; d <<= 1) {
                const float v = __shfl_up_sync(0xffffffffu, top, d);
                if (lane - d >= lo) top = fmaxf(top, v);
            }
            top = __shfl_sync(0xffffffffu, top, hi);
            const float w = ka_exp2(ml.x - (top == -INFINITY ? 0.f : top));
            float l = ml.y * w;
#pragma unroll
            for (int d = 1; d < 32; d <<= 1) {
                const float v = __shfl_up_sync(0xffffffffu, l, d);
                if (lane - d >= lo) l += v;
            }
            l = __shfl_sync(0xffffffffu, l, hi);
            weight[r][lane] = w;
            if (lane == lo) stat[r][lane] = make_float2(top, l);
        }
    };
    auto sum_parts = [&](unsigned there, int k0, int k1, int r, int d, auto at) -> float4 {   // parts k0 .. k1 - 1, those of `there`
        float4 o = make_float4(0.f, 0.f, 0.f, 0.f);
        for (int k = k0; k < k1; k += 4) {
            float4 y[4];
            float w[4];
#pragma unroll
            for (int i = 0; i < 4; ++i) {
                const bool in = k + i < k1 && (there >> (k + i) & 1u);
                y[i] = in ? *reinterpret_cast<const float4*>(smem + at(k + i) + (r * S::PITCH + d) * 4) : make_float4(0.f, 0.f, 0.f, 0.f);
                w[i] = in ? weight[r][k + i] : 0.f;
            }
#pragma unroll
            for (int i = 0; i < 4; ++i) {
                o.x = fmaf(w[i], y[i].x, o.x); o.y = fmaf(w[i], y[i].y, o.y); o.z = fmaf(w[i], y[i].z, o.z); o.w = fmaf(w[i], y[i].w, o.w);
            }
        }
        return o;
    };
    auto put = [&](const KaPiece& pc, int r, int d, int head, const float4& o, bool final, size_t place) {   // place: of the scratch
        const float2 ml = stat[r][head];
        if (final) {
            const float inv = ka_norm(ml.y), y[4] = {o.x * inv, o.y * inv, o.z * inv, o.w * inv};
            ka_store(a, ka_out_at(a, pc.row0, pc.hk, pc.q0 + r, D) + d, y);
        } else {
            float* to = reinterpret_cast<float*>(a.part + place * S::SLOT) + r * S::PITCH;
            __stcg(reinterpret_cast<float4*>(to + d), o);
            if (d == 0) __stcg(reinterpret_cast<float2*>(to + D), ml);
        }
    };

    // The warps' pieces.  One of an item that other CTAs have parts of goes to the scratch: place 0 if the item began in an earlier CTA, else
    // place 1; the CTA has one of each at most.
    const KaPiece mine = lane < 2 * W ? pieces[lane] : KaPiece{};
    int open0, open1;   // a piece of the item at place 0, 1; -1: none
    {
        auto at = [&](int k) -> uint32_t { return pieces[k].at; };
        const unsigned there = __ballot_sync(0xffffffffu, mine.nt != 0), below = there & ((1u << lane) - 1u);
        const uint32_t before = __shfl_sync(0xffffffffu, mine.first, below ? 31 - __clz(below) : 0);
        const bool head = mine.nt != 0 && (below == 0 || before != mine.first);
        const unsigned heads = __ballot_sync(0xffffffffu, head);
        const bool whole = mine.first >= c0 && mine.first + (uint32_t)mine.nt <= c1;
        open0 = __ffs(__ballot_sync(0xffffffffu, head && !whole && mine.first < c0)) - 1;
        open1 = __ffs(__ballot_sync(0xffffffffu, head && !whole && mine.first >= c0)) - 1;
        if (warp == 0 && head) group_head[__popc(heads & ((1u << lane) - 1u))] = lane;
        weigh(there, heads, mine.at, ROWS);
        __syncthreads();
        const int units = __popc(heads) * ROWS * (D / 4);
        for (int i = threadIdx.x; i < units; i += W * 32) {
            const int r = i / (D / 4) % ROWS, d = i % (D / 4) * 4, e = group_head[i / (ROWS * (D / 4))];
            const KaPiece& pc = pieces[e];
            if (r >= pc.rows - pc.q0) continue;
            const unsigned later = heads & ~((2u << e) - 1u);
            put(pc, r, d, e, sum_parts(there, e, later ? __ffs(later) - 1 : 2 * W, r, d, at), e != open0 && e != open1, (size_t)blockIdx.x * 4 + (e == open0 ? 0 : 1));
        }
    }
    if (open0 < 0 && open1 < 0) return;   // (the same in all threads: every warp has looked at all pieces)

    // Items that several CTAs share: the last CTA of a group to arrive merges the group, the last group's the groups.  An item's entries:
    // its first CTA's place 1, the others' place 0; a group's result: the group's first CTA's place 3 (the item's first CTA) or 2.
    // A counter has two halves: a CTA can be the first of a group of an item that began earlier, and of an item that begins there.
    for (int level = 0; level < 2; ++level) {
        int lo[2] = {0, 0}, entries[2] = {0, 0}, step[2] = {1, 1}, f[2] = {0, 0};
        bool final[2] = {false, false};
#pragma unroll
        for (int k = 0; k < 2; ++k) {
            const int e = k == 0 ? open0 : open1;
            if (e < 0) continue;
            const uint32_t first = pieces[e].first;
            f[k] = (int)kv8_cta_of(cut, first);
            const int n = (int)kv8_cta_of(cut, first + (uint32_t)pieces[e].nt - 1u) - f[k] + 1, group = kv8_merge_group(n);
            lo[k] = level == 0 ? ((int)blockIdx.x - f[k]) / group * group : 0;
            entries[k] = level == 0 ? min(group, n - lo[k]) : (n + group - 1) / group;
            step[k] = level == 0 ? 1 : group;
            final[k] = level == 1 || entries[k] == n;
        }
        __syncthreads();   // (this CTA's parts are written)
        if (threadIdx.x < 2) {
            const int k = threadIdx.x, l = k == 0 ? lo[0] : lo[1], n = k == 0 ? entries[0] : entries[1];
            bool last = false;
            if (n > 0) last = ka_arrive(a.tickets + level * KA_MAX_CTAS + (k == 0 ? f[0] : f[1]) + l, l > 0 ? 0x10000u : 1u, (unsigned)n);
            last_flag[k] = last ? 1 : 0;
        }
        __syncthreads();
        const int n0 = last_flag[0] ? entries[0] : 0, n1 = last_flag[1] ? entries[1] : 0;
        bool more = false;
        // both at once where there is room
        for (int todo = (n0 ? 1 : 0) | (n1 ? 2 : 0); todo;) {
            const int now = todo == 3 && (n0 + n1) * S::SLOT > S::RING ? 1 : todo;
            todo &= ~now;
            const int m0 = now & 1 ? n0 : 0, m = m0 + (now & 2 ? n1 : 0);   // entries 0 .. m0 - 1 of the one item, m0 .. m - 1 of the other
            const uint32_t dst = (uint32_t)__cvta_generic_to_shared(smem);
            auto rows_of = [&](int k) { const KaPiece& pc = pieces[k == 0 ? open0 : open1]; return min(ROWS, pc.rows - pc.q0); };
            for (int e = warp; e < m; e += W) {
                const int k = e < m0 ? 0 : 1, c = (k == 0 ? lo[0] : lo[1]) + (e - (k == 0 ? 0 : m0)) * (k == 0 ? step[0] : step[1]);
                const uint8_t* src = a.part + ((size_t)((k == 0 ? f[0] : f[1]) + c) * 4 + (level == 1 ? 2 : 0) + (c == 0 ? 1 : 0)) * S::SLOT;
                const int pieces16 = rows_of(k) * S::PITCH / 4;   // 16-byte pieces of an entry
#pragma unroll 4
                for (int i = lane; i < pieces16; i += 32) ka_cp16(dst + e * S::SLOT + i * 16, src + i * 16);
            }
            ka_commit();
            ka_wait<0>();
            __syncthreads();
            auto at = [](int e) -> uint32_t { return (uint32_t)(e * S::SLOT); };
            const unsigned there = m == 32 ? 0xffffffffu : (1u << m) - 1u, heads = (m0 ? 1u : 0u) | (m > m0 ? 1u << m0 : 0u);
            weigh(there, heads, at(min(lane, m - 1)), ROWS);   // (what it makes of rows that an item does not have is not used)
            __syncthreads();
            for (int i = threadIdx.x; i < __popc(heads) * ROWS * (D / 4); i += W * 32) {
                const int k = (m0 == 0 || i >= ROWS * (D / 4)) ? 1 : 0, r = i / (D / 4) % ROWS, d = i % (D / 4) * 4;
                if (r >= rows_of(k)) continue;
                const KaPiece& pc = pieces[k == 0 ? open0 : open1];
                put(pc, r, d, k == 0 ? 0 : m0, sum_parts(there, k == 0 ? 0 : m0, k == 0 ? m0 : m, r, d, at), k == 0 ? final[0] : final[1],
                    (size_t)((k == 0 ? f[0] : f[1]) + (k == 0 ? lo[0] : lo[1])) * 4 + ((k == 0 ? lo[0] : lo[1]) == 0 ? 3 : 2));
            }
            __syncthreads();   // (the next merge uses the same shared memory)
        }
        if (n0 && !final[0]) more = true; else open0 = -1;
        if (n1 && !final[1]) more = true; else open1 = -1;
        if (!more) return;
    }
}

template <int D, int QT>
static cudaError_t launch_ka(const KaArgs& a, cudaStream_t s) {
    using S = KaShape<D, QT>;
    static PerDeviceOnce configured;
    const int rc = configured.run(current_device(), [] {
        return (int)cudaFuncSetAttribute(kv8_attn_kernel<D, QT>, cudaFuncAttributeMaxDynamicSharedMemorySize, S::SMEM);
    });
    if (rc != 0) return rc < 0 ? cudaErrorInvalidDevice : (cudaError_t)rc;
    const int grid = sm_count() < KA_MAX_CTAS ? sm_count() : KA_MAX_CTAS;
    const cudaError_t e = launch_pdl(kv8_attn_kernel<D, QT>, dim3((unsigned)grid), dim3(S::WARPS * 32), S::SMEM, s, a);
    count_launch();
    return e;
}

cudaError_t launch_kv8_attn(const aq_kv8_cache_t& c, const aq_kv8_batch_t& b, const void* q, int64_t q_row, void* out, int64_t out_row, int T,
                            int n_heads, float scale, aq_dtype_t dt, aq_dtype_t out_dt, void* scratch, cudaStream_t s) {
    KaArgs a;
    memset(&a, 0, sizeof(a));
    a.q = q; a.out = out;
    a.kc = reinterpret_cast<const uint8_t*>(c.k_dev); a.vc = reinterpret_cast<const uint8_t*>(c.v_dev);
    a.ks = c.k_scale_dev; a.vs = c.v_scale_dev;
    a.lens = b.lens_dev; a.row_start = b.row_start_dev; a.table = b.table_dev;
    a.width = b.table_width; a.n_pages = c.n_pages; a.q_row = q_row; a.out_row = out_row;
    a.B = b.n_seqs; a.T = T; a.n_each = T / b.n_seqs; a.Hkv = c.n_kv_heads; a.G = n_heads / c.n_kv_heads;
    a.shift = 0;
    while ((AQ_KV8_BLOCK << a.shift) < c.page) ++a.shift;
    a.G_magic = kv8_magic((uint32_t)a.G);
    a.q_bf16 = dt == AQ_BF16; a.out_dtype = (int)out_dt;
    a.scale_log2 = scale * 1.4426950408889634f;
    uint8_t* sc = reinterpret_cast<uint8_t*>(scratch);
    a.tickets = reinterpret_cast<unsigned*>(sc);
    a.part = sc + KA_TICKET_BYTES;
    // query rows per pass over a request's keys and values: what it has of them; where requests may differ, half as many again as on average
    // (slots without rows and requests with fewer lie in the average; a second pass over a long request costs more than empty columns).  The
    // host knows the step's rows and not whose they are: rows of nobody count, and a prompt among decodes does.
    const int64_t each = b.row_start_dev ? (T <= a.B ? 1 : ((int64_t)3 * T + a.B) / (2 * (int64_t)a.B)) : a.n_each;
    const int64_t rows = a.G * each;
    const int qt = rows <= 4 ? 1 : rows <= 8 || c.head_dim == 256 ? 2 : rows <= 12 ? 3 : 4;
    switch (c.head_dim + qt) {
        case 65: return launch_ka<64, 1>(a, s);
        case 66: return launch_ka<64, 2>(a, s);
        case 67: return launch_ka<64, 3>(a, s);
        case 68: return launch_ka<64, 4>(a, s);
        case 129: return launch_ka<128, 1>(a, s);
        case 130: return launch_ka<128, 2>(a, s);
        case 131: return launch_ka<128, 3>(a, s);
        case 132: return launch_ka<128, 4>(a, s);
        case 257: return launch_ka<256, 1>(a, s);
        default: return launch_ka<256, 2>(a, s);
    }
}

}  // namespace aq

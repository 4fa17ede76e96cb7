// Attention of a step's new tokens over the paged 8-bit key/value cache:
//     out[t][h] = sum_p softmax_p(scale q[t][h] . K[p]) V[p],   K[p] = ks code_k[p],  V[p] = vs code_v[p],
// over the positions p of the row's request up to the row's own, ks and vs one float32 per 32 positions and head.
//
// Bound: HBM.  Every key and value is read once, D bytes each; per position and head that is 2 D + 0.25 bytes for 4 D G M flops.
//
// Why this layout.  Positions are the rows of the tensor-core tile and query rows its columns (mma.sync.m16n8k16, binary16 in,
// binary32 sums): with one to eight query rows per key/value head no part of a tile is padding but the columns, and a lane holds
// two queries' scores, so a running maximum is two registers.  A tile of the work is 32 positions, the span of one scale, so the
// scales touch the sums and not the operands.
//   S^T = K q^T.  A code byte c + 128 in the low half of a binary16 IS the number (c + 128) 2^-24 (a subnormal): one byte permute
//       per two codes makes the operand.  128 sum(q) is taken off the sum.  A lane's two bytes pairs of a 16-byte piece are dims
//       4t .. 4t + 3 instead of 2t, 2t + 1, 2t + 8, 2t + 9: q is loaded in the same order.  q's row is divided by a power of two
//       first so that its largest magnitude is in [1, 2): then bfloat16 rows fit binary16 too (what is under 2^-24 of the largest
//       is lost, at most 2^-25 of it).
//   P = exp2(S - max + 15), rounded to binary16 (weights down to 2^-39 of the largest keep a value), moved into operand order by
//       movmatrix.  sum(P) is a product with ones, so the normaliser sums exactly what the values are weighted with.
//   O^T += vs (V^T P^T - 128 sum P).  ldmatrix.trans on pairs of bytes gives dims 2g, 2g + 1 of two positions in one register:
//       the even bytes are one operand row, the odd bytes another.
// Every warp has a contiguous run of the line of tiles (aq_kv8_runs.h) and streams it through its own cp.async ring without
// waiting for another warp; runs differ by one tile at most whatever the requests' lengths are.  What a warp finishes alone it
// writes; pieces of an item are merged over the warps of the CTA in shared memory, then over the CTAs in the scratch by the last
// CTA to arrive (tickets; nobody waits).
// (Included by aq_kv8.cu alone, which has the status word and the host calls.)
#pragma once

namespace aq {

constexpr int KA_TILE = AQ_KV8_BLOCK;                 // positions per tile: the span of a scale
constexpr int KA_MAX_CTAS = 192;

template <int D, int NT>
struct KaShape {
    static constexpr int WARPS = D == 256 ? 4 : 8;
    static constexpr int STAGES = D == 64 ? 5 : (NT == 2 ? 2 : 3);
    static constexpr int ROWS = 8 * NT;               // query rows of an item
    static constexpr int HALF = KA_TILE * D;          // bytes of a tile's keys (or values)
    static constexpr int STAGE = 2 * HALF + 16;       // + ks, vs, whether the tile may be read
    static constexpr int PITCH = D + 4;               // floats: a row's O, then its maximum and sum
    static constexpr int SLOT = ROWS * PITCH * 4;
    static constexpr int RING = WARPS * STAGES * STAGE;
    static constexpr int SMEM = RING + WARPS * SLOT;
    static_assert(SLOT <= STAGES * STAGE, "a warp's last piece is put down in its own ring");
    static_assert((AQ_KV8_MAX_SEQS + 1) * 4 <= WARPS * SLOT, "the line's marks lie where pieces will");
    static_assert(WARPS * ROWS * D * 4 + KA_MAX_CTAS * ROWS * 8 <= RING, "the merge works in the ring");
    static_assert(SMEM + 1024 <= 232448, "shared memory of an SM");
};
// scratch: tickets [2][KA_MAX_CTAS][2], (maximum, sum) [KA_MAX_CTAS][2][rows], O [KA_MAX_CTAS][2][rows][D]
constexpr size_t KA_TICKET_BYTES = 2 * KA_MAX_CTAS * 2 * 4;
constexpr size_t KA_ML_BYTES = (size_t)KA_MAX_CTAS * 2 * 16 * 8;
static_assert(KA_TICKET_BYTES + KA_ML_BYTES + (size_t)KA_MAX_CTAS * 2 * 8 * 256 * 4 <= AQ_KV8_SCRATCH_BYTES &&
              KA_TICKET_BYTES + KA_ML_BYTES + (size_t)KA_MAX_CTAS * 2 * 16 * 128 * 4 <= AQ_KV8_SCRATCH_BYTES, "scratch");

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
    int q_bf16, out_dtype;
    float scale_log2;           // scale log2(e)
    unsigned* tickets;
    float* ml;
    float* part;
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
__device__ __forceinline__ void ka_mma(float (&c)[4], uint32_t a0, uint32_t a1, uint32_t a2, uint32_t a3, uint32_t b0, uint32_t b1) {
    asm("mma.sync.aligned.m16n8k16.row.col.f32.f16.f16.f32 {%0,%1,%2,%3}, {%4,%5,%6,%7}, {%8,%9}, {%0,%1,%2,%3};"
        : "+f"(c[0]), "+f"(c[1]), "+f"(c[2]), "+f"(c[3]) : "r"(a0), "r"(a1), "r"(a2), "r"(a3), "r"(b0), "r"(b1));
}
__device__ __forceinline__ float ka_exp2(float x) {   // 2 ulp; results below 2^-126 are 0
    float y;
    asm("ex2.approx.ftz.f32 %0, %1;" : "=f"(y) : "f"(x));
    return y;
}
__device__ __forceinline__ uint32_t ka_pack(float lo, float hi) {
    const __half2 v = __floats2half2_rn(lo, hi);
    return *reinterpret_cast<const uint32_t*>(&v);
}
// Byte offset of 16-byte piece c of row r in a tile: rows of eight that ldmatrix reads together fall on different banks.
template <int D>
__device__ __forceinline__ uint32_t ka_at(int r, int c) {
    const int x = D == 64 ? c ^ ((r >> 1) & 3) : c ^ (r & 7);
    return (uint32_t)(r * D + x * 16);
}

// A request of the line.
struct KaSeq {
    int b, L, row0, n, nt, rb;   // nt: tiles of an item; rb: items per key/value head
};
__device__ __forceinline__ KaSeq ka_seq(const KaArgs& a, int b, int rows) {
    KaSeq s;
    s.b = b;
    const Kv8Rows r = a.row_start ? kv8_rows(__ldg(a.row_start + b), __ldg(a.row_start + b + 1), a.T) : Kv8Rows{b * a.n_each, a.n_each};
    s.row0 = r.first;
    s.n = r.n;
    const int64_t most = a.width << (a.shift + 5);
    s.L = (int)min((int64_t)max(__ldg(a.lens + b), 0), most);
    s.nt = max(1, (s.L + KA_TILE - 1) / KA_TILE);   // (a request without positions has one tile that is not read: its rows become 0)
    s.rb = (int)(((int64_t)s.n * a.G + rows - 1) / rows);
    return s;
}

// A piece of an item as it is put down for merging.
struct KaPiece {
    uint32_t start;   // the item's first tile on the line
    int nt;           // its tiles (0: no piece here)
    int row0, rows;   // first row of the request, its query rows (G n)
    int hk, q0;       // key/value head, the item's first query row
};

// Stores D/32 neighbouring values of a lane as the output's type.
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
    const int tok = q / a.G;
    return (int64_t)(row0 + tok) * a.out_row + (int64_t)(hk * a.G + (q - tok * a.G)) * D;
}
// 2^24 over the normaliser (the sums of V are in units of 2^-24); a row that saw nothing is 0
__device__ __forceinline__ float ka_norm(float l) { return l == 0.f ? 0.f : 16777216.f / l; }

template <int D, int NT>
__global__ void __launch_bounds__(KaShape<D, NT>::WARPS * 32, 1) kv8_attn_kernel(const __grid_constant__ KaArgs a) {
    using S = KaShape<D, NT>;
    constexpr int W = S::WARPS, ROWS = S::ROWS, NV = D / 32;
    extern __shared__ __align__(128) uint8_t smem[];
    __shared__ KaPiece pieces[2 * W];
    __shared__ uint32_t warp_sum[W];
    __shared__ int last_flag;
    const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
    const int g = lane >> 2, t = lane & 3;

    // ---- the line: marks[b] = first tile of request b -------------------------------------------------------
    uint32_t* marks = reinterpret_cast<uint32_t*>(smem + S::RING);
    pdl_wait();
    {
        const int per = (a.B + W * 32 - 1) / (W * 32), b0 = threadIdx.x * per;
        uint32_t mine = 0;
        for (int b = b0; b < min(b0 + per, a.B); ++b) {
            const KaSeq s = ka_seq(a, b, ROWS);
            if (s.n > 0 && s.L != __ldg(a.lens + b)) kv8_report(KV8_BAD_LENGTH);
            mine += (uint32_t)s.nt * (uint32_t)s.rb * (uint32_t)a.Hkv;
        }
        uint32_t upto = mine;
#pragma unroll
        for (int d = 1; d < 32; d <<= 1) {
            const uint32_t v = __shfl_up_sync(0xffffffffu, upto, d);
            if (lane >= d) upto += v;
        }
        if (lane == 31) warp_sum[warp] = upto;
        if (lane < 2) pieces[2 * warp + lane].nt = 0;
        __syncthreads();
        uint32_t before = upto - mine;
        for (int w = 0; w < warp; ++w) before += warp_sum[w];
        for (int b = b0; b < min(b0 + per, a.B); ++b) {
            marks[b] = before;
            const KaSeq s = ka_seq(a, b, ROWS);
            before += (uint32_t)s.nt * (uint32_t)s.rb * (uint32_t)a.Hkv;
        }
    }
    uint32_t total = 0;
    for (int w = 0; w < W; ++w) total += warp_sum[w];
    __syncthreads();
    // CTAs with less than a tile per warp would only add pieces to merge
    const uint32_t n_cta = min(gridDim.x, (total + W - 1) / W);
    if (blockIdx.x >= n_cta) return;
    const uint32_t n_run = n_cta * W, run = blockIdx.x * W + warp;
    const uint32_t x0 = kv8_run_begin(total, run, n_run), x1 = kv8_run_begin(total, run + 1, n_run);
    const uint32_t c0 = kv8_run_begin(total, blockIdx.x * W, n_run), c1 = kv8_run_begin(total, (blockIdx.x + 1) * W, n_run);

    KaSeq sq{};
    int item = 0, j = 0;          // item of the request (head x block of rows), tile of the item
    if (x0 < x1) {
        const int b = kv8_find(marks, a.B, x0);
        sq = ka_seq(a, b, ROWS);
        const uint32_t off = x0 - marks[b];
        item = (int)(off / (uint32_t)sq.nt);
        j = (int)(off - (uint32_t)item * (uint32_t)sq.nt);
    }
    __syncthreads();   // (pieces may be put down where the marks are)

    const uint32_t ring = (uint32_t)__cvta_generic_to_shared(smem) + (uint32_t)warp * S::STAGES * S::STAGE;
    float* slot_a = reinterpret_cast<float*>(smem + S::RING + warp * S::SLOT);
    float* slot_b = reinterpret_cast<float*>(smem + warp * S::STAGES * S::STAGE);

    if (x0 < x1) {
        // ---- copies: a walk of its own, STAGES - 1 tiles ahead ----------------------------------------------
        KaSeq ps = sq;
        int p_item = item, p_j = j, p_page0 = -1, p_pages = -1;   // lane i holds the number of page p_page0 + i
        uint32_t p_x = x0;
        auto next_item = [&](KaSeq& s, int& it) {
            if (++it < s.rb * a.Hkv) return;
            it = 0;
            int b = s.b;
            do { s = ka_seq(a, ++b, ROWS); } while (s.n == 0 && b + 1 < a.B);   // (x < total: there is one)
        };
        auto issue = [&](int st) {
            const uint32_t dst = ring + (uint32_t)st * S::STAGE;
            const int pg = p_j >> a.shift;
            if (p_page0 < 0 || pg >= p_page0 + 32 || pg < p_page0) {
                p_page0 = pg;
                const int i = pg + lane;
                p_pages = (int64_t)i < a.width && (i << (a.shift + 5)) < ps.L ? __ldg(a.table + (int64_t)ps.b * a.width + i) : -1;
            }
            const int page = __shfl_sync(0xffffffffu, p_pages, pg - p_page0);
            const bool ok = page >= 0 && page < a.n_pages;
            if (ok) {
                const int hk = p_item / ps.rb;
                const int64_t blk = (((int64_t)page * a.Hkv + hk) << a.shift) + (p_j & ((1 << a.shift) - 1));
                const uint8_t* sk = a.kc + blk * S::HALF;
                const uint8_t* sv = a.vc + blk * S::HALF;
#pragma unroll
                for (int i = 0; i < S::HALF / 512; ++i) {
                    const int idx = i * 32 + lane, row = idx / (D / 16), c = idx % (D / 16);
                    ka_cp16(dst + ka_at<D>(row, c), sk + idx * 16);
                    ka_cp16(dst + S::HALF + ka_at<D>(row, c), sv + idx * 16);
                }
                if (lane < 2) ka_cp4(dst + 2 * S::HALF + 4 * lane, (lane ? a.vs : a.ks) + blk);
            } else if (ps.L > 0 && lane == 0) {
                kv8_report(KV8_BAD_PAGE);
            }
            if (lane == 2) asm volatile("st.shared.u32 [%0], %1;" ::"r"(dst + 2 * S::HALF + 8), "r"(ok ? 1 : 0) : "memory");
            if (++p_x < x1 && ++p_j == ps.nt) {
                p_j = 0;
                const int was = ps.b;
                next_item(ps, p_item);
                if (ps.b != was) p_page0 = -1;
            }
        };
#pragma unroll
        for (int s = 0; s < S::STAGES - 1; ++s) {
            if (p_x < x1) issue(s);
            ka_commit();
        }

        uint32_t qf[NT][D / 16][2];
        float o[NT][D / 16][4];
        float m[NT][2], l[NT][2], bq[NT][2], fq[NT][2];
        int lim[NT][2], lim_min = 0;
        KaPiece pc{};
        bool fresh = true;
        int st = 0;
        for (uint32_t x = x0; x < x1; ++x) {
            if (fresh) {   // ---- another item: its queries
                fresh = false;
                pc.start = x - (uint32_t)j;
                pc.nt = sq.nt;
                pc.row0 = sq.row0;
                pc.rows = a.G * sq.n;
                pc.hk = item / sq.rb;
                pc.q0 = (item - pc.hk * sq.rb) * ROWS;
#pragma unroll
                for (int nt = 0; nt < NT; ++nt) {
                    const int r = pc.q0 + 8 * nt + g;   // this lane's operand column
                    uint2 raw[D / 16];
                    if (r < pc.rows) {
                        const int tok = r / a.G;
                        const uint16_t* q = reinterpret_cast<const uint16_t*>(a.q) + (int64_t)(pc.row0 + tok) * a.q_row +
                                            (int64_t)(pc.hk * a.G + (r - tok * a.G)) * D + 4 * t;
#pragma unroll
                        for (int c = 0; c < D / 16; ++c) raw[c] = __ldg(reinterpret_cast<const uint2*>(q + 16 * c));
                    } else {
#pragma unroll
                        for (int c = 0; c < D / 16; ++c) raw[c] = make_uint2(0u, 0u);
                    }
                    auto wide = [&](uint32_t v) -> float2 {
                        if (a.q_bf16) return make_float2(__uint_as_float(v << 16), __uint_as_float(v & 0xffff0000u));
                        return __half22float2(*reinterpret_cast<const __half2*>(&v));
                    };
                    float big = 0.f;
#pragma unroll
                    for (int c = 0; c < D / 16; ++c) {
                        const float2 u = wide(raw[c].x), v = wide(raw[c].y);
                        big = fmaxf(big, fmaxf(fmaxf(fabsf(u.x), fabsf(u.y)), fmaxf(fabsf(v.x), fabsf(v.y))));
                    }
                    big = fmaxf(big, __shfl_xor_sync(0xffffffffu, big, 1));
                    big = fmaxf(big, __shfl_xor_sync(0xffffffffu, big, 2));
                    // the power of two under the largest magnitude, as a factor that takes it off (1 for rows of zeros; an infinity stays one)
                    const int e = big > 0.f ? min(max((int)(__float_as_uint(big) >> 23), 1), 253) : 127;
                    const float down = __uint_as_float((uint32_t)(254 - e) << 23), up = __uint_as_float((uint32_t)e << 23);
                    float sum = 0.f;
#pragma unroll
                    for (int c = 0; c < D / 16; ++c) {
                        const float2 u = wide(raw[c].x), v = wide(raw[c].y);
                        qf[nt][c][0] = ka_pack(u.x * down, u.y * down);
                        qf[nt][c][1] = ka_pack(v.x * down, v.y * down);
                        const float2 a2 = __half22float2(*reinterpret_cast<const __half2*>(&qf[nt][c][0]));
                        const float2 b2 = __half22float2(*reinterpret_cast<const __half2*>(&qf[nt][c][1]));
                        sum += (a2.x + a2.y) + (b2.x + b2.y);
                    }
                    sum += __shfl_xor_sync(0xffffffffu, sum, 1);
                    sum += __shfl_xor_sync(0xffffffffu, sum, 2);
                    sum *= 128.f / 16777216.f;   // what the codes' offset of 128 adds to this row's products
#pragma unroll
                    for (int i = 0; i < 2; ++i) {   // and of the two query rows whose scores this lane holds
                        bq[nt][i] = __shfl_sync(0xffffffffu, sum, 4 * (2 * t + i));
                        fq[nt][i] = __shfl_sync(0xffffffffu, up, 4 * (2 * t + i)) * (a.scale_log2 * 16777216.f);
                        const int rr = min(pc.q0 + 8 * nt + 2 * t + i, pc.rows - 1);
                        lim[nt][i] = sq.L - sq.n + rr / a.G + 1;   // positions before this one are seen
                        m[nt][i] = -INFINITY;
                        l[nt][i] = 0.f;
                    }
#pragma unroll
                    for (int c = 0; c < D / 16; ++c) o[nt][c][0] = o[nt][c][1] = o[nt][c][2] = o[nt][c][3] = 0.f;
                }
                lim_min = sq.L - sq.n + pc.q0 / a.G + 1;
            }

            ka_wait<S::STAGES - 2>();
            __syncwarp();   // every lane's copies of this tile have landed, and every lane is through with the tile before
            if (p_x < x1) issue(st == 0 ? S::STAGES - 1 : st - 1);
            ka_commit();
            const uint32_t kt = ring + (uint32_t)st * S::STAGE, vt = kt + S::HALF;
            st = st + 1 == S::STAGES ? 0 : st + 1;
            float ks, vs;
            int ok;
            asm volatile("ld.shared.f32 %0, [%1];" : "=f"(ks) : "r"(kt + 2 * S::HALF) : "memory");
            asm volatile("ld.shared.f32 %0, [%1];" : "=f"(vs) : "r"(kt + 2 * S::HALF + 4) : "memory");
            asm volatile("ld.shared.s32 %0, [%1];" : "=r"(ok) : "r"(kt + 2 * S::HALF + 8) : "memory");

            if (ok) {   // (the same for all lanes; a tile that could not be read counts as masked)
                // ---- S^T = K q^T: 32 positions x 8 NT queries
                float sc[NT][2][4];
#pragma unroll
                for (int nt = 0; nt < NT; ++nt)
#pragma unroll
                    for (int mt = 0; mt < 2; ++mt) sc[nt][mt][0] = sc[nt][mt][1] = sc[nt][mt][2] = sc[nt][mt][3] = 0.f;
#pragma unroll
                for (int cp = 0; cp < D / 32; ++cp) {
#pragma unroll
                    for (int mt = 0; mt < 2; ++mt) {
                        uint32_t r[4];
                        ka_ldm(kt + ka_at<D>(16 * mt + ((lane >> 3) & 1) * 8 + (lane & 7), 2 * cp + (lane >> 4)), r);
#pragma unroll
                        for (int i = 0; i < 4; ++i) r[i] ^= 0x80808080u;
#pragma unroll
                        for (int h = 0; h < 2; ++h) {
                            const uint32_t a0 = __byte_perm(r[2 * h], 0u, 0x4140), a2 = __byte_perm(r[2 * h], 0u, 0x4342);
                            const uint32_t a1 = __byte_perm(r[2 * h + 1], 0u, 0x4140), a3 = __byte_perm(r[2 * h + 1], 0u, 0x4342);
#pragma unroll
                            for (int nt = 0; nt < NT; ++nt) ka_mma(sc[nt][mt], a0, a1, a2, a3, qf[nt][2 * cp + h][0], qf[nt][2 * cp + h][1]);
                        }
                    }
                }
                // ---- weights
                const int pos = j * KA_TILE;
                const bool all_seen = pos + KA_TILE <= lim_min;
                uint32_t pb[NT][2][2];
                float al[NT][2], vq[NT][2], off[NT][2];
                bool moved = false;
#pragma unroll
                for (int nt = 0; nt < NT; ++nt) {
                    if (!all_seen) {
#pragma unroll
                        for (int mt = 0; mt < 2; ++mt)
#pragma unroll
                            for (int i = 0; i < 4; ++i)
                                if (pos + 16 * mt + (i >> 1) * 8 + g >= lim[nt][i & 1]) sc[nt][mt][i] = -INFINITY;
                    }
                    float base[2];
#pragma unroll
                    for (int i = 0; i < 2; ++i) {
                        float mx = fmaxf(fmaxf(sc[nt][0][i], sc[nt][0][i + 2]), fmaxf(sc[nt][1][i], sc[nt][1][i + 2]));
                        mx = fmaxf(mx, __shfl_xor_sync(0xffffffffu, mx, 4));
                        mx = fmaxf(mx, __shfl_xor_sync(0xffffffffu, mx, 8));
                        mx = fmaxf(mx, __shfl_xor_sync(0xffffffffu, mx, 16));
                        const float F = ks * fq[nt][i];
                        const float s = mx == -INFINITY ? -INFINITY : (mx - bq[nt][i]) * F;
                        const float now = fmaxf(m[nt][i], s);   // (a NaN among the scores leaves the maximum and reaches the sums)
                        base[i] = now == -INFINITY ? 0.f : now;
                        al[nt][i] = ka_exp2(m[nt][i] - base[i]);
                        moved |= now != m[nt][i];
                        m[nt][i] = now;
                        const float add = 15.f - base[i];
#pragma unroll
                        for (int mt = 0; mt < 2; ++mt)
#pragma unroll
                            for (int k = i; k < 4; k += 2) {
                                const float raw = sc[nt][mt][k];
                                const float p = ka_exp2(fmaf(raw - bq[nt][i], F, add));
                                sc[nt][mt][k] = raw == -INFINITY ? 0.f : p;
                            }
                    }
                    float lt[4] = {0.f, 0.f, 0.f, 0.f};
#pragma unroll
                    for (int mt = 0; mt < 2; ++mt) {
                        pb[nt][mt][0] = ka_transpose(ka_pack(sc[nt][mt][0], sc[nt][mt][1]));
                        pb[nt][mt][1] = ka_transpose(ka_pack(sc[nt][mt][2], sc[nt][mt][3]));
                        ka_mma(lt, 0x3C003C00u, 0x3C003C00u, 0x3C003C00u, 0x3C003C00u, pb[nt][mt][0], pb[nt][mt][1]);
                    }
#pragma unroll
                    for (int i = 0; i < 2; ++i) {
                        l[nt][i] = fmaf(l[nt][i], al[nt][i], lt[i]);
                        off[nt][i] = lt[i] * (-128.f / 16777216.f);
                        vq[nt][i] = lt[i] == 0.f ? 0.f : vs;   // (what a row gives no weight cannot reach it, a NaN among it)
                    }
                }
                moved = __any_sync(0xffffffffu, moved);
                // ---- O^T = al O^T + vs (V^T P^T - 128 sum P)
#pragma unroll
                for (int c = 0; c < D / 16; ++c) {
                    uint32_t r[4];
                    ka_ldm_t(vt + ka_at<D>(lane, c), r);
#pragma unroll
                    for (int i = 0; i < 4; ++i) r[i] ^= 0x80808080u;
                    uint32_t ev[4], od[4];
#pragma unroll
                    for (int i = 0; i < 4; ++i) {
                        ev[i] = __byte_perm(r[i], 0u, 0x4240);
                        od[i] = __byte_perm(r[i], 0u, 0x4341);
                    }
#pragma unroll
                    for (int nt = 0; nt < NT; ++nt) {
                        float ot[4] = {off[nt][0], off[nt][1], off[nt][0], off[nt][1]};
                        ka_mma(ot, ev[0], od[0], ev[1], od[1], pb[nt][0][0], pb[nt][0][1]);
                        ka_mma(ot, ev[2], od[2], ev[3], od[3], pb[nt][1][0], pb[nt][1][1]);
                        if (moved) {
#pragma unroll
                            for (int i = 0; i < 4; ++i) o[nt][c][i] *= al[nt][i & 1];
                        }
#pragma unroll
                        for (int i = 0; i < 4; ++i) o[nt][c][i] = fmaf(vq[nt][i & 1], ot[i], o[nt][c][i]);
                    }
                }
            }

            // ---- the item's end, or the run's
            const bool item_ends = j + 1 == sq.nt, run_ends = x + 1 == x1;
            if (item_ends || run_ends) {
                const bool whole = item_ends && pc.start >= x0;
                if (whole) {
#pragma unroll
                    for (int nt = 0; nt < NT; ++nt)
#pragma unroll
                        for (int i = 0; i < 2; ++i) {
                            const int r = pc.q0 + 8 * nt + 2 * t + i;
                            if (r < pc.rows) {
                                const float inv = ka_norm(l[nt][i]);
                                const int64_t at = ka_out_at(a, pc.row0, pc.hk, r, D) + 2 * g;
#pragma unroll
                                for (int c = 0; c < D / 16; ++c) {
                                    const float two[2] = {o[nt][c][i] * inv, o[nt][c][i + 2] * inv};
                                    ka_store(a, at + 16 * c, two);
                                }
                            }
                        }
                } else {
                    // a run's first piece goes to a place of its own, its last into the ring, which is done with by then
                    if (run_ends) { ka_wait<0>(); __syncwarp(); }
                    float* to = run_ends ? slot_b : slot_a;
#pragma unroll
                    for (int nt = 0; nt < NT; ++nt)
#pragma unroll
                        for (int i = 0; i < 2; ++i) {
                            float* row = to + (8 * nt + 2 * t + i) * S::PITCH;
#pragma unroll
                            for (int c = 0; c < D / 16; ++c) *reinterpret_cast<float2*>(row + 16 * c + 2 * g) = make_float2(o[nt][c][i], o[nt][c][i + 2]);
                            if (g == 0) *reinterpret_cast<float2*>(row + D) = make_float2(m[nt][i], l[nt][i]);
                        }
                    if (lane == 0) pieces[2 * warp + (run_ends ? 1 : 0)] = pc;
                }
            }
            if (item_ends) {
                j = 0;
                if (!run_ends) { next_item(sq, item); fresh = true; }
            } else {
                ++j;
            }
        }
        ka_wait<0>();
    }
    __syncthreads();

    // ---- pieces of one item lie next to each other in the order of the warps: merge them -----------------------
    // A piece of an item that other CTAs have parts of goes to the scratch: place 0 if the item holds the CTA's first tile, else 1.
    KaPiece open[2];
    open[0].nt = open[1].nt = 0;
    {
        int e = 0, seq = 0;
        while (e < 2 * W) {
            if (pieces[e].nt == 0) { ++e; continue; }
            const KaPiece pc = pieces[e];
            int e1 = e + 1;
            while (e1 < 2 * W && (pieces[e1].nt == 0 || pieces[e1].start == pc.start)) ++e1;
            const bool whole = pc.start >= c0 && pc.start + (uint32_t)pc.nt <= c1;
            const int place = pc.start <= c0 ? 0 : 1;
            if (!whole) open[place] = pc;
            for (int r = 0; r < min(ROWS, pc.rows - pc.q0); ++r, ++seq) {
                if (seq % W != warp) continue;
                float top = -INFINITY;
                for (int i = e; i < e1; ++i)
                    if (pieces[i].nt) {
                        const float* row = ((i & 1) ? reinterpret_cast<float*>(smem + (i >> 1) * S::STAGES * S::STAGE)
                                                    : reinterpret_cast<float*>(smem + S::RING + (i >> 1) * S::SLOT)) + r * S::PITCH;
                        top = fmaxf(top, row[D]);
                    }
                const float base = top == -INFINITY ? 0.f : top;
                float acc[NV], ls = 0.f;
#pragma unroll
                for (int v = 0; v < NV; ++v) acc[v] = 0.f;
                for (int i = e; i < e1; ++i)
                    if (pieces[i].nt) {
                        const float* row = ((i & 1) ? reinterpret_cast<float*>(smem + (i >> 1) * S::STAGES * S::STAGE)
                                                    : reinterpret_cast<float*>(smem + S::RING + (i >> 1) * S::SLOT)) + r * S::PITCH;
                        const float w = ka_exp2(row[D] - base);
                        ls = fmaf(w, row[D + 1], ls);
#pragma unroll
                        for (int v = 0; v < NV; v += 2) {
                            const float2 y = *reinterpret_cast<const float2*>(row + NV * lane + v);
                            acc[v] = fmaf(w, y.x, acc[v]);
                            acc[v + 1] = fmaf(w, y.y, acc[v + 1]);
                        }
                    }
                if (whole) {
                    const float inv = ka_norm(ls);
#pragma unroll
                    for (int v = 0; v < NV; ++v) acc[v] *= inv;
                    ka_store(a, ka_out_at(a, pc.row0, pc.hk, pc.q0 + r, D) + NV * lane, acc);
                } else {
                    const size_t at = ((size_t)blockIdx.x * 2 + place) * ROWS + r;
#pragma unroll
                    for (int v = 0; v < NV; v += 2) __stcg(reinterpret_cast<float2*>(a.part + at * D + NV * lane + v), make_float2(acc[v], acc[v + 1]));
                    if (lane == 0) __stcg(reinterpret_cast<float2*>(a.ml) + at, make_float2(top, ls));
                }
            }
            e = e1;
        }
    }

    // ---- items that several CTAs share: the last one of a group to arrive merges the group ----------------------
    for (int place = 0; place < 2; ++place) {
        if (open[place].nt == 0) continue;   // (the same in all threads: every thread has walked all pieces)
        const KaPiece pc = open[place];
        const int rows = min(ROWS, pc.rows - pc.q0);
        const int f = (int)(kv8_run_of(total, pc.start, n_run) / W), e = (int)(kv8_run_of(total, pc.start + (uint32_t)pc.nt - 1u, n_run) / W);
        const int n = e - f + 1, group = kv8_merge_group(n);
        const int f_place = pc.start <= kv8_run_begin(total, (uint32_t)f * W, n_run) ? 0 : 1;   // (only the first CTA's can be 1)
        int my = (int)blockIdx.x - f;
        // level 0: entries of my group; level 1: the groups' results, each at its first entry
        for (int level = 0; level < 2; ++level) {
            const int step = level == 0 ? 1 : group;
            const int lo = level == 0 ? my / group * group : 0;
            const int count = level == 0 ? min(group, n - lo) : (n + group - 1) / group;
            if (level == 1 && count == 1) break;
            __threadfence();
            __syncthreads();
            if (threadIdx.x == 0) {
                unsigned* ticket = a.tickets + level * KA_MAX_CTAS * 2 + (f + lo) * 2 + (lo == 0 ? f_place : 0);
                const bool last = atomicAdd(ticket, 1u) == (unsigned)count - 1u;
                if (last) *ticket = 0u;   // (as the next call wants it: all have been here)
                last_flag = last ? 1 : 0;
            }
            __syncthreads();
            const bool go = last_flag != 0;
            __syncthreads();
            if (!go) break;
            __threadfence();
            const bool final = level == 1 || count == n;
            float* s_acc = reinterpret_cast<float*>(smem);             // [W][ROWS][D]
            float2* s_ml = reinterpret_cast<float2*>(smem + W * ROWS * D * 4);   // [count][ROWS]
            auto entry = [&](int i) -> size_t {                        // row 0 of entry i
                const int k = lo + i * step;
                return ((size_t)(f + k) * 2 + (k == 0 ? f_place : 0)) * ROWS;
            };
            for (int i = threadIdx.x; i < count * ROWS; i += W * 32)
                if (i % ROWS < rows) s_ml[i] = __ldcg(reinterpret_cast<const float2*>(a.ml) + entry(i / ROWS) + i % ROWS);
            __syncthreads();
            // each warp takes entries warp, warp + W, ... of all rows, four rows' loads in flight
            for (int r0 = 0; r0 < rows; r0 += 4) {
                float base[4], acc[4][NV];
#pragma unroll
                for (int q = 0; q < 4; ++q) {
                    float top = -INFINITY;
                    if (r0 + q < rows)
                        for (int i = lane; i < count; i += 32) top = fmaxf(top, s_ml[i * ROWS + r0 + q].x);
#pragma unroll
                    for (int d = 16; d; d >>= 1) top = fmaxf(top, __shfl_xor_sync(0xffffffffu, top, d));
                    base[q] = top == -INFINITY ? 0.f : top;
#pragma unroll
                    for (int v = 0; v < NV; ++v) acc[q][v] = 0.f;
                }
                for (int i = warp; i < count; i += W) {
                    const size_t at = entry(i);
                    float2 y[4][NV / 2];
#pragma unroll
                    for (int q = 0; q < 4; ++q)
#pragma unroll
                        for (int v = 0; v < NV / 2; ++v)
                            y[q][v] = r0 + q < rows ? __ldcg(reinterpret_cast<const float2*>(a.part + (at + r0 + q) * D + NV * lane) + v) : make_float2(0.f, 0.f);
#pragma unroll
                    for (int q = 0; q < 4; ++q) {
                        if (r0 + q >= rows) continue;
                        const float w = ka_exp2(s_ml[i * ROWS + r0 + q].x - base[q]);
#pragma unroll
                        for (int v = 0; v < NV / 2; ++v) {
                            acc[q][2 * v] = fmaf(w, y[q][v].x, acc[q][2 * v]);
                            acc[q][2 * v + 1] = fmaf(w, y[q][v].y, acc[q][2 * v + 1]);
                        }
                    }
                }
#pragma unroll
                for (int q = 0; q < 4; ++q)
                    if (r0 + q < rows) {
#pragma unroll
                        for (int v = 0; v < NV; v += 2)
                            *reinterpret_cast<float2*>(s_acc + ((size_t)warp * ROWS + r0 + q) * D + NV * lane + v) = make_float2(acc[q][v], acc[q][v + 1]);
                    }
            }
            __syncthreads();
            for (int r = warp; r < rows; r += W) {
                float top = -INFINITY, ls = 0.f, acc[NV];
                for (int i = lane; i < count; i += 32) top = fmaxf(top, s_ml[i * ROWS + r].x);
#pragma unroll
                for (int d = 16; d; d >>= 1) top = fmaxf(top, __shfl_xor_sync(0xffffffffu, top, d));
                const float base = top == -INFINITY ? 0.f : top;
                for (int i = 0; i < count; ++i) ls = fmaf(ka_exp2(s_ml[i * ROWS + r].x - base), s_ml[i * ROWS + r].y, ls);
#pragma unroll
                for (int v = 0; v < NV; ++v) acc[v] = 0.f;
                for (int w = 0; w < min(W, count); ++w)
#pragma unroll
                    for (int v = 0; v < NV; ++v) acc[v] += s_acc[((size_t)w * ROWS + r) * D + NV * lane + v];
                if (final) {
                    const float inv = ka_norm(ls);
#pragma unroll
                    for (int v = 0; v < NV; ++v) acc[v] *= inv;
                    ka_store(a, ka_out_at(a, pc.row0, pc.hk, pc.q0 + r, D) + NV * lane, acc);
                } else {
                    const size_t at = entry(0) + r;
#pragma unroll
                    for (int v = 0; v < NV; v += 2) __stcg(reinterpret_cast<float2*>(a.part + at * D + NV * lane + v), make_float2(acc[v], acc[v + 1]));
                    if (lane == 0) __stcg(reinterpret_cast<float2*>(a.ml) + at, make_float2(top, ls));
                }
            }
            if (final) break;
            my = lo;   // (this CTA goes on for its group)
        }
        __syncthreads();   // (the next place's merge uses the same shared memory)
    }
}

template <int D, int NT>
static cudaError_t launch_ka(const KaArgs& a, cudaStream_t s) {
    using S = KaShape<D, NT>;
    static PerDeviceOnce configured;
    const int rc = configured.run(current_device(), [] {
        return (int)cudaFuncSetAttribute(kv8_attn_kernel<D, NT>, cudaFuncAttributeMaxDynamicSharedMemorySize, S::SMEM);
    });
    if (rc != 0) return rc < 0 ? cudaErrorInvalidDevice : (cudaError_t)rc;
    const int grid = sm_count() < KA_MAX_CTAS ? sm_count() : KA_MAX_CTAS;
    const cudaError_t e = launch_pdl(kv8_attn_kernel<D, NT>, dim3((unsigned)grid), dim3(S::WARPS * 32), S::SMEM, s, a);
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
    a.q_bf16 = dt == AQ_BF16; a.out_dtype = (int)out_dt;
    a.scale_log2 = scale * 1.4426950408889634f;
    uint8_t* sc = reinterpret_cast<uint8_t*>(scratch);
    a.tickets = reinterpret_cast<unsigned*>(sc);
    a.ml = reinterpret_cast<float*>(sc + KA_TICKET_BYTES);
    a.part = reinterpret_cast<float*>(sc + KA_TICKET_BYTES + KA_ML_BYTES);
    // sixteen query rows per pass over a request's keys and values where it has more than eight, on average
    const bool wide = (int64_t)a.G * T > 8 * (int64_t)a.B;
    if (c.head_dim == 64) return wide ? launch_ka<64, 2>(a, s) : launch_ka<64, 1>(a, s);
    if (c.head_dim == 128) return wide ? launch_ka<128, 2>(a, s) : launch_ka<128, 1>(a, s);
    return launch_ka<256, 1>(a, s);
}

}  // namespace aq

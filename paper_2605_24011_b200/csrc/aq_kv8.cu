// The paged 8-bit key/value cache: the step's plan (pages, lengths, row and position maps), the append that quantises, and the
// host side of the attention (aq_kv8_attn.cuh).  (No counterpart in the paper, whose runtime serves one request from a
// half-precision cache; it stands beside aq_kv_append and aq_attn_decode.)
//
// Cache: codes int8 [n_pages][Hkv][page][D], float32 scales [n_pages][Hkv][page / 32]; a value is code * scale.
#include <cuda_bf16.h>
#include <cuda_fp16.h>

#include <cstring>

#include "aq_internal.h"
#include "aq_kv8_runs.h"
#include "aq_per_device.h"

namespace aq {

// What a call met in the caller's device arrays that it could not follow (the host cannot see it); aq_check reports it.
enum { KV8_BAD_PAGE = 1, KV8_BAD_LENGTH = 2, KV8_NO_ROOM = 3 };
__device__ int g_kv8_status = 0;
__device__ __forceinline__ void kv8_report(int code) { atomicCAS(&g_kv8_status, 0, code); }

int read_kv8_status(bool clear) {
    int v = 0;
    cudaMemcpyFromSymbol(&v, g_kv8_status, sizeof(int));
    if (clear && v) { int z = 0; cudaMemcpyToSymbol(g_kv8_status, &z, sizeof(int)); }
    return v;
}

// ---- plan -----------------------------------------------------------------------------------------------------
// One CTA, one thread per request: the whole step is three sums over at most 1024 requests and as many list entries as pages
// change hands, so it is bound by latency: three trips to memory (lengths; the free list; the tables) and the launch.
constexpr int KP_THREADS = 1024;
static_assert(KP_THREADS >= AQ_KV8_MAX_SEQS, "a thread per request");

struct KpArgs {
    const int32_t* lens;
    const int32_t* added;
    int32_t* table;
    int32_t* free_list;
    const int32_t* n_free;
    int32_t* lens_out;
    int32_t* n_free_out;
    int32_t* row_start;
    int32_t* pos;
    int64_t width, free_cap;
    int B, shift, n_rows;   // shift: log2 of the page
};

// Exclusive sums of three values over the CTA's threads; the totals in tot.
__device__ __forceinline__ void kp_scan3(int (&v)[3], int (&tot)[3], int (*sums)[3]) {
    const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
    int up[3] = {v[0], v[1], v[2]};
#pragma unroll
    for (int d = 1; d < 32; d <<= 1)
#pragma unroll
        for (int k = 0; k < 3; ++k) {
            const int o = __shfl_up_sync(0xffffffffu, up[k], d);
            if (lane >= d) up[k] += o;
        }
    if (lane == 31)
#pragma unroll
        for (int k = 0; k < 3; ++k) sums[warp][k] = up[k];
    __syncthreads();
    if (warp < 3) {   // warp k: the warps' sums of value k
        const int x = sums[lane][warp];
        int y = x;
#pragma unroll
        for (int d = 1; d < 32; d <<= 1) {
            const int o = __shfl_up_sync(0xffffffffu, y, d);
            if (lane >= d) y += o;
        }
        sums[lane][warp] = y - x;
        if (lane == 31) sums[32][warp] = y;
    }
    __syncthreads();
#pragma unroll
    for (int k = 0; k < 3; ++k) {
        v[k] = up[k] - v[k] + sums[warp][k];
        tot[k] = sums[32][k];
    }
}

// put(lane of a request, j, get(lane, j)) for j < n: the first FEW by the request's own thread (most requests have one or none), the rest by its
// warp, 32 at a time, four such loads before their stores.  (A search for the request of each row and page instead: 4096 rows and
// 3500 pages of 1000 requests 6.7 us.)
template <int FEW, typename Get, typename Put>
__device__ __forceinline__ void kp_each(int n, Get get, Put put) {
    const int lane = threadIdx.x & 31;
#pragma unroll
    for (int j = 0; j < FEW; ++j)
        if (j < n) put(lane, j, get(lane, j));
    for (unsigned left = __ballot_sync(0xffffffffu, n > FEW); left; left &= left - 1) {
        const int src = __ffs(left) - 1, m = __shfl_sync(0xffffffffu, n, src);
        for (int j0 = FEW + lane; j0 < m; j0 += 128) {
            int v[4];
#pragma unroll
            for (int i = 0; i < 4; ++i) v[i] = j0 + 32 * i < m ? get(src, j0 + 32 * i) : 0;
#pragma unroll
            for (int i = 0; i < 4; ++i)
                if (j0 + 32 * i < m) put(src, j0 + 32 * i, v[i]);
        }
    }
}

__global__ void __launch_bounds__(KP_THREADS, 1) kv8_plan_kernel(const KpArgs a) {
    __shared__ int sums[33][3];
    __shared__ int4 of[KP_THREADS];   // of a request: where its given pages go, where its taken ones come from, its first row; pages held
    __shared__ int length[KP_THREADS];
    const int b = threadIdx.x, P = 1 << a.shift;
    pdl_wait();
    pdl_launch_dependents();
    const int n_free = *a.n_free;
    int len = 0, add = 0;
    if (b < a.B) { len = a.lens[b]; add = a.added[b]; }
    const int64_t most = a.width << a.shift;
    // -1: the request has ended
    bool ok = len >= 0 && len <= most && add >= -1 && (add < 0 || (int64_t)len + add <= most) && add <= a.n_rows;
    const int held = ok ? (int)(((int64_t)len + P - 1) >> a.shift) : 0;
    const int grown = ok && add >= 0 ? (int)(((int64_t)len + add + P - 1) >> a.shift) - held : 0;
    int v[3] = {ok && add < 0 ? held : 0, grown, ok ? max(add, 0) : 0}, tot[3];
    kp_scan3(v, tot, sums);
    of[b] = make_int4(v[0], v[1], v[2], held);   // (read by the warp itself)
    length[b] = len;
    ok = ok && tot[2] <= a.n_rows && n_free >= 0 && (int64_t)n_free + tot[0] <= a.free_cap && (int64_t)tot[1] <= (int64_t)n_free + tot[0];
    ok = __syncthreads_and(ok);
    if (!ok) {   // nothing changes, and the step has no rows
        if (b == 0) kv8_report(KV8_NO_ROOM);
        if (b < a.B) a.lens_out[b] = len;
        if (b == 0) *a.n_free_out = n_free;
        for (int i = b; i <= a.B; i += KP_THREADS) a.row_start[i] = 0;
        for (int i = b; i < a.n_rows; i += KP_THREADS) a.pos[i] = -1;
        return;
    }
    const int b0 = b & ~31;   // the warp's first request
    // pages of ended requests go on the stack, in the order of the requests and their pages
    kp_each<0>(add < 0 ? held : 0, [&](int k, int j) { return a.table[(int64_t)(b0 + k) * a.width + j]; },
               [&](int k, int j, int page) { a.free_list[n_free + of[b0 + k].x + j] = page; });
    if (b < a.B) {
        a.lens_out[b] = add < 0 ? 0 : len + add;
        a.row_start[b] = v[2];
    }
    if (b == 0) {
        *a.n_free_out = n_free + tot[0] - tot[1];
        a.row_start[a.B] = tot[2];
    }
    kp_each<1>(max(add, 0), [&](int k, int j) { return length[b0 + k] + j; }, [&](int k, int j, int p) { a.pos[of[b0 + k].z + j] = p; });
    for (int i = tot[2] + b; i < a.n_rows; i += KP_THREADS) a.pos[i] = -1;
    __syncthreads();   // (pages that have just been given back may be taken)
    // requests that grow take theirs from the top, in the same order
    kp_each<1>(grown, [&](int k, int j) { return a.free_list[n_free + tot[0] - 1 - of[b0 + k].y - j]; },
               [&](int k, int j, int page) { a.table[(int64_t)(b0 + k) * a.width + of[b0 + k].w + j] = page; });
}

cudaError_t launch_kv8_plan(const int32_t* lens, const int32_t* added, int n_seqs, int page, int32_t* table, int64_t width, int32_t* free_list,
                            int64_t free_cap, const int32_t* n_free, int32_t* lens_out, int32_t* n_free_out, int32_t* row_start, int32_t* pos,
                            int n_rows, cudaStream_t s) {
    KpArgs a;
    a.lens = lens; a.added = added; a.table = table; a.free_list = free_list; a.n_free = n_free; a.lens_out = lens_out; a.n_free_out = n_free_out;
    a.row_start = row_start; a.pos = pos; a.width = width; a.free_cap = free_cap; a.B = n_seqs; a.n_rows = n_rows;
    a.shift = 0;
    while ((1 << a.shift) < page) ++a.shift;
    const cudaError_t e = launch_pdl(kv8_plan_kernel, dim3(1), dim3(KP_THREADS), 0, s, a);
    count_launch();
    return e;
}

// ---- append ---------------------------------------------------------------------------------------------------
// A unit of work is what a step brings to one block of 32 positions of one head, keys or values: up to 32 rows that its warps
// hold in registers, so they are read once:
//     need = up11(max |x| / 127),  s = need <= s_old ? s_old : max(need, up11(1.25 s_old)),  code = rint(x / s)
// up11: the next binary32 value of 11 significant bits.  With both x (11 bits at most) and s that short, the binary32 quotient
// is at a half exactly where the true one is, so the rounding is the true quotient's.  A block whose first position is among the
// new rows starts with s_old = 0.  Where the scale of a block under way grows, its older codes become rint(code s_old / s): by a
// quarter at least, so that a code is rounded again few times (off by (1 + 1/1.25 + ...) / 2 < 2.5 steps in all, whatever comes).
// A NaN or an infinity makes the block's scale NaN: its values read as NaN until the block is begun again.
// Bound: HBM for prompts (2 bytes read and 1 written per element), a launch and four dependent trips (row marks, length, page,
// scale) for a decode step.
struct KwArgs {
    uint8_t* codes[2];     // keys, values
    float* scales[2];
    const uint16_t* x[2];
    const int32_t* lens;
    const int32_t* row_start;
    const int32_t* table;
    int64_t width, n_pages, x_row;
    int B, T, n_each, Hkv, shift, chunk, heads;   // shift: log2(blocks per page); rows per CTA; heads per CTA (WPU 4)
};
constexpr int KW_WARPS = 4, KW_CTAS = 6;

__device__ __forceinline__ float kw_up11(float x) { return __uint_as_float(kv8_up11(__float_as_uint(x))); }
__device__ __forceinline__ float kw_up11_normal(float x) { return __uint_as_float((__float_as_uint(x) + 0x1FFFu) & ~0x1FFFu); }   // (of a subnormal: more)

// rint(x / s) for |x / s| < 2^21 as the low bits of a float: the quotient correctly rounded (x inv, corrected by its exact remainder: P. Markstein,
// "Computation of elementary functions on the IBM RISC System/6000 processor", 1990), then rounded to a whole number by adding 1.5 * 2^23.  inv = 1 / s rounded; s in 2^-60 .. 2^125.
__device__ __forceinline__ uint32_t kw_quotient(float x, float s, float inv) {
    const float q = x * inv;
    return __float_as_uint(fmaf(fmaf(-q, s, x), inv, q) + 12582912.f);
}
__device__ __forceinline__ uint32_t kw_bytes(uint32_t a, uint32_t b, uint32_t c, uint32_t d) {   // their low bytes
    return __byte_perm(__byte_perm(a, b, 0x0040), __byte_perm(c, d, 0x0040), 0x5410);
}

// A unit's rows on their way, in the registers of its WPU warps (1, or the CTA's 4): w is this one's number among them.
template <int D, int WPU>
struct KwUnit {
    static constexpr int LPR = D / 8;                // lanes per row (16 bytes each)
    static constexpr int RPP = 32 / LPR * WPU;       // rows per pass
    static constexpr int NV = 32 / RPP;              // passes of a whole block
    uint4 v[NV];
    float s_old;
    int n, at;
    uint8_t* codes;
    float* scale;
    __device__ __forceinline__ void load(const uint16_t* x, int64_t x_row, int n_, int at_, uint8_t* codes_, float* scale_, int w) {
        const int lane = threadIdx.x & 31, sub = w * (32 / LPR) + lane / LPR, c = lane % LPR;
        n = n_; at = at_; codes = codes_; scale = scale_;
#pragma unroll
        for (int i = 0; i < NV; ++i) {
            const int r = i * RPP + sub;
            v[i] = r < n ? reinterpret_cast<const uint4*>(x + r * x_row)[c] : make_uint4(0u, 0u, 0u, 0u);
        }
        s_old = at > 0 ? *scale : 0.f;
    }
};

// Quantises and stores a unit; all of its warps call this together.
template <int D, bool BF16, int WPU>
__device__ __forceinline__ void kw_store(const KwUnit<D, WPU>& u, int w, uint32_t* meet) {
    constexpr int LPR = KwUnit<D, WPU>::LPR, RPP = KwUnit<D, WPU>::RPP, NV = KwUnit<D, WPU>::NV;
    const int lane = threadIdx.x & 31, sub = w * (32 / LPR) + lane / LPR, c = lane % LPR, n = u.n, at = u.at;
    const uint4 (&v)[NV] = u.v;
    const float s_old = u.s_old;
    uint8_t* codes = u.codes;
    float* scale = u.scale;
    // magnitudes as whole numbers: of two values of one 16-bit type the larger has the larger pattern, a NaN the largest
    uint32_t most = 0;
#pragma unroll
    for (int i = 0; i < NV; ++i) {
        const uint32_t u[4] = {v[i].x, v[i].y, v[i].z, v[i].w};
#pragma unroll
        for (int k = 0; k < 4; ++k) most = __vmaxu2(most, u[k] & 0x7fff7fffu);
    }
    most = __reduce_max_sync(0xffffffffu, max(most & 0xffffu, most >> 16));
    if constexpr (WPU > 1) {
        if (lane == 0) meet[w] = most;
        __syncthreads();                      // (and every warp has read the scale)
#pragma unroll
        for (int k = 0; k < WPU; ++k) most = max(most, meet[k]);
        __syncthreads();
    }
    auto wide = [](uint32_t h) -> float {
        if constexpr (BF16) return __uint_as_float(h << 16);
        else return __half2float(__ushort_as_half((unsigned short)h));
    };
    const bool poison = most >= (BF16 ? 0x7f80u : 0x7c00u) || !(s_old == s_old);
    const float asked = wide(most) / 127.f;
    const float need = kw_up11_normal(asked);
    float s = need <= s_old ? s_old : fmaxf(need, kw_up11_normal(1.25f * s_old));
    // The short form differs for subnormals alone, and then s is under 2^-125 (bfloat16 only; with the whole form for all a prompt of 4000 rows
    // took 22.1 us, 21.5 so).
    if (s < 2.35098870164457501594e-38f) {
        const float exact = kw_up11(asked);
        s = exact <= s_old ? s_old : fmaxf(exact, kw_up11(1.25f * s_old));
    }
    if (poison) s = __uint_as_float(0x7fc00000u);
    // A scale under 2^-60 (bfloat16 only) has no reciprocal to work with: both sides of the quotient times 2^100 then.  s = 0 is a block of
    // zeros; of a NaN the codes do not matter, they become 0, as do those of an infinite scale (a caller's; quotients by it).
    const float lift = s < 8.67361737988403547e-19f ? 1.2676506002282294e30f : 1.f;
    const bool endless = s > 3.402823466e38f;
    const float fit = s > 0.f && !endless ? s * lift : 1.f, inv = poison || endless ? 0.f : 1.f / fit;
    auto pair = [&](uint32_t u, uint32_t& a, uint32_t& b) {
        float e, f;
        if constexpr (BF16) { e = __uint_as_float(u << 16); f = __uint_as_float(u & 0xffff0000u); }
        else {
            const float2 h = __half22float2(*reinterpret_cast<const __half2*>(&u));
            e = h.x; f = h.y;
        }
        if (BF16 && lift != 1.f) { e *= lift; f *= lift; }
        a = kw_quotient(e, fit, inv);
        b = kw_quotient(f, fit, inv);
    };
#pragma unroll
    for (int i = 0; i < NV; ++i) {
        const int r = i * RPP + sub;
        if (r < n) {
            const uint32_t u[4] = {v[i].x, v[i].y, v[i].z, v[i].w};
            uint32_t o[2];
#pragma unroll
            for (int k = 0; k < 2; ++k) {
                uint32_t a, b, e, f;
                pair(u[2 * k], a, b);
                pair(u[2 * k + 1], e, f);
                o[k] = poison ? 0u : kw_bytes(a, b, e, f);
            }
            *reinterpret_cast<uint2*>(codes + (at + r) * D + 8 * c) = make_uint2(o[0], o[1]);
        }
    }
    if (s > s_old && at > 0 && !poison) {   // the older positions' codes on the larger scale
        const float was_fit = s_old * lift;
        for (int r = sub; r < at; r += RPP) {
            uint2* p = reinterpret_cast<uint2*>(codes + r * D + 8 * c);
            const uint2 u = *p;
            uint32_t o[2];
#pragma unroll
            for (int h = 0; h < 2; ++h) {
                uint32_t b[4];
#pragma unroll
                for (int k = 0; k < 4; ++k) b[k] = kw_quotient((float)(int)(int8_t)((h ? u.y : u.x) >> (8 * k)) * was_fit, fit, inv);
                o[h] = kw_bytes(b[0], b[1], b[2], b[3]);
            }
            *p = make_uint2(o[0], o[1]);
        }
    }
    if constexpr (WPU == 1) __syncwarp();   // (every lane has read the scale)
    if (w == 0 && lane == 0 && (at == 0 || !(s == s_old))) *scale = s;
}

// WPU 1: a warp per unit, two heads' keys and values per CTA (decode steps: units of a row or a few).  WPU 4: the CTA's warps share each
// unit, keys or values of a few heads per CTA (prompts: one warp per unit left an SM with a few thousand instructions in a row, 9 requests'
// chunks of 333 rows of one head of 256 took 14.0 us).
template <int D, bool BF16, int WPU>
__global__ void __launch_bounds__(KW_WARPS * 32) kv8_append_kernel(const __grid_constant__ KwArgs a) {
    __shared__ int begin[AQ_KV8_MAX_SEQS + 1];
    __shared__ uint32_t meet[KW_WARPS];
    const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
    const int kv = WPU == 1 ? warp & 1 : (int)blockIdx.z, hk = WPU == 1 ? 2 * blockIdx.y + (warp >> 1) : (int)blockIdx.y * a.heads;
    const int t0 = blockIdx.x * a.chunk;
    pdl_wait();
    pdl_launch_dependents();
    if (a.row_start) {
        for (int i = threadIdx.x; i <= a.B; i += KW_WARPS * 32) begin[i] = a.row_start[i];
        __syncthreads();
    }
    if (hk >= a.Hkv) return;
    // lane: one row of the chunk.  The rows that are the first of this step in their block lead a unit.
    const int t = t0 + lane;
    int at = 0, n = 0;            // its place in its block; rows of the unit (0: not a leader)
    int64_t blk = 0;              // the block's number with head 0 (page, head, block of the page)
    if (lane < a.chunk && t < a.T) {
        int b;
        Kv8Rows rows;
        if (a.row_start) {
            b = kv8_find(begin, a.B, t);
            rows = kv8_rows(begin[b], begin[b + 1], a.T);
        } else {
            b = t / a.n_each;
            rows = Kv8Rows{b * a.n_each, a.n_each};
        }
        const int i = t - rows.first;
        if (i >= 0 && i < rows.n) {
            const int64_t pos = (int64_t)a.lens[b] - rows.n + i;
            at = (int)(pos & (AQ_KV8_BLOCK - 1));
            const int64_t tile = pos >> 5, pg = tile >> a.shift;
            if (pos < 0 || pg >= a.width) {
                kv8_report(KV8_BAD_LENGTH);
            } else if (i == 0 || at == 0) {
                const int page = a.table[(int64_t)b * a.width + pg];
                if (page < 0 || page >= a.n_pages) {
                    kv8_report(KV8_BAD_PAGE);
                } else {
                    n = min(AQ_KV8_BLOCK - at, rows.n - i);
                    blk = (((int64_t)page * a.Hkv) << a.shift) + (tile & ((1 << a.shift) - 1));
                }
            }
        }
    }
    unsigned leaders = __ballot_sync(0xffffffffu, n > 0);   // (with WPU 4 the same in every warp)
    if (!leaders) return;
    // (leader, head) pairs in turn, the next one's rows asked for while one is quantised
    int src = __ffs(leaders) - 1, h = hk;
    auto load = [&](KwUnit<D, WPU>& u) {
        const int64_t b = __shfl_sync(0xffffffffu, blk, src) + ((int64_t)h << a.shift);
        u.load(a.x[kv] + (int64_t)(t0 + src) * a.x_row + (int64_t)h * D, a.x_row, __shfl_sync(0xffffffffu, n, src), __shfl_sync(0xffffffffu, at, src),
               a.codes[kv] + b * AQ_KV8_BLOCK * D, a.scales[kv] + b, WPU == 1 ? 0 : warp);
    };
    auto next = [&] {   // whether there is another pair
        if (++h < min(hk + a.heads, a.Hkv)) return true;
        h = hk;
        leaders &= leaders - 1;
        src = __ffs(leaders) - 1;
        return leaders != 0;
    };
    KwUnit<D, WPU> u;
    load(u);
    for (;;) {
        if (WPU == 1) {   // (no registers for two)
            kw_store<D, BF16, WPU>(u, 0, meet);
            if (!next()) break;
            load(u);
        } else {
            const KwUnit<D, WPU> now = u;
            const bool more = next();
            if (more) load(u);
            kw_store<D, BF16, WPU>(now, warp, meet);
            if (!more) break;
        }
    }
}

template <int D, bool BF16>
static cudaError_t launch_kw(KwArgs& a, cudaStream_t s) {
    // four rows or more per request on average: prompts or chunks of them
    if ((int64_t)a.T >= 4 * (int64_t)a.B) {
        a.chunk = 32;
        const int64_t blocks = (a.T + 31) / 32;
        // per CTA: as many as leave each SM several CTAs, so that one's look-ups serve them all, but four at most: with up to eight the last CTAs
        // run alone (32 heads of 64, 4000 rows: 21.1 us, 15.5 so; 8 chunks of 500 rows of 32 heads of 128: 31.8 and 27.2; one of 4000: 21.4 and 21.5)
        a.heads = 1;
        while (a.heads < 4 && blocks * 2 * ((a.Hkv + 2 * a.heads - 1) / (2 * a.heads)) >= KW_CTAS * sm_count()) a.heads *= 2;
        return launch_pdl(kv8_append_kernel<D, BF16, 4>, dim3((unsigned)blocks, (unsigned)((a.Hkv + a.heads - 1) / a.heads), 2), dim3(KW_WARPS * 32), 0, s, a);
    }
    // a decode step's rows are a unit each: a CTA each while there are few
    const int pairs = (a.Hkv + 1) / 2;
    a.chunk = 1;
    a.heads = 1;
    while (a.chunk < 32 && (int64_t)((a.T + a.chunk - 1) / a.chunk) * pairs > 4 * sm_count()) a.chunk *= 2;
    return launch_pdl(kv8_append_kernel<D, BF16, 1>, dim3((unsigned)((a.T + a.chunk - 1) / a.chunk), (unsigned)pairs), dim3(KW_WARPS * 32), 0, s, a);
}

cudaError_t launch_kv8_append(const aq_kv8_cache_t& c, const aq_kv8_batch_t& b, const void* k, const void* v, int64_t x_row, int T, aq_dtype_t dt,
                              cudaStream_t s) {
    KwArgs a;
    a.codes[0] = reinterpret_cast<uint8_t*>(c.k_dev); a.codes[1] = reinterpret_cast<uint8_t*>(c.v_dev);
    a.scales[0] = c.k_scale_dev; a.scales[1] = c.v_scale_dev;
    a.x[0] = reinterpret_cast<const uint16_t*>(k); a.x[1] = reinterpret_cast<const uint16_t*>(v);
    a.lens = b.lens_dev; a.row_start = b.row_start_dev; a.table = b.table_dev;
    a.width = b.table_width; a.n_pages = c.n_pages; a.x_row = x_row;
    a.B = b.n_seqs; a.T = T; a.n_each = T / b.n_seqs; a.Hkv = c.n_kv_heads;
    a.shift = 0;
    while ((AQ_KV8_BLOCK << a.shift) < c.page) ++a.shift;
    const bool bf = dt == AQ_BF16;
    cudaError_t e;
    if (c.head_dim == 64) e = bf ? launch_kw<64, true>(a, s) : launch_kw<64, false>(a, s);
    else if (c.head_dim == 128) e = bf ? launch_kw<128, true>(a, s) : launch_kw<128, false>(a, s);
    else e = bf ? launch_kw<256, true>(a, s) : launch_kw<256, false>(a, s);
    count_launch();
    return e;
}

}  // namespace aq

#include "aq_kv8_attn.cuh"

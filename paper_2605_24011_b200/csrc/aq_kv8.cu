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

__global__ void __launch_bounds__(KP_THREADS, 1) kv8_plan_kernel(const KpArgs a) {
    __shared__ int sums[33][3];
    __shared__ int back_at[AQ_KV8_MAX_SEQS + 1], take_at[AQ_KV8_MAX_SEQS + 1], row_at[AQ_KV8_MAX_SEQS + 1];
    __shared__ int s_len[AQ_KV8_MAX_SEQS], s_held[AQ_KV8_MAX_SEQS];
    const int b = threadIdx.x, P = 1 << a.shift;
    pdl_wait();
    const int n_free = __ldg(a.n_free);
    int len = 0, add = 0;
    if (b < a.B) { len = __ldg(a.lens + b); add = __ldg(a.added + b); }
    const int64_t most = a.width << a.shift;
    // -1: the request has ended
    bool ok = len >= 0 && len <= most && add >= -1 && (add < 0 || (int64_t)len + add <= most) && add <= a.n_rows;
    const int held = ok ? (int)(((int64_t)len + P - 1) >> a.shift) : 0;
    const int grown = ok && add >= 0 ? (int)(((int64_t)len + add + P - 1) >> a.shift) - held : 0;
    int v[3] = {ok && add < 0 ? held : 0, grown, ok ? max(add, 0) : 0}, tot[3];
    kp_scan3(v, tot, sums);
    if (b < a.B) {
        back_at[b] = v[0]; take_at[b] = v[1]; row_at[b] = v[2];
        s_len[b] = len; s_held[b] = held;
    }
    if (b == 0) { back_at[a.B] = tot[0]; take_at[a.B] = tot[1]; row_at[a.B] = tot[2]; }
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
    // pages of ended requests go on the stack, in the order of the requests and their pages
    for (int i = b; i < tot[0]; i += KP_THREADS) {
        const int r = kv8_find(back_at, a.B, i);
        a.free_list[n_free + i] = a.table[(int64_t)r * a.width + (i - back_at[r])];
    }
    if (b < a.B) a.lens_out[b] = add < 0 ? 0 : len + add;
    if (b == 0) *a.n_free_out = n_free + tot[0] - tot[1];
    for (int i = b; i <= a.B; i += KP_THREADS) a.row_start[i] = row_at[i];
    for (int i = b; i < a.n_rows; i += KP_THREADS) {
        int p = -1;
        if (i < tot[2]) {
            const int r = kv8_find(row_at, a.B, i);
            p = s_len[r] + i - row_at[r];
        }
        a.pos[i] = p;
    }
    __syncthreads();   // (pages that have just been given back may be taken)
    // requests that grow take theirs from the top, in the same order
    for (int i = b; i < tot[1]; i += KP_THREADS) {
        const int r = kv8_find(take_at, a.B, i);
        a.table[(int64_t)r * a.width + s_held[r] + (i - take_at[r])] = a.free_list[n_free + tot[0] - 1 - i];
    }
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
// A unit of work is what a step brings to one block of 32 positions of one head, keys or values: up to 32 rows that one warp
// holds in registers, so they are read once:
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
    int B, T, n_each, Hkv, shift, chunk;   // shift: log2(blocks per page); chunk: rows per CTA
};
constexpr int KW_WARPS = 4;

__device__ __forceinline__ float kw_up11(float x) { return __uint_as_float((__float_as_uint(x) + 0x1FFFu) & ~0x1FFFu); }

template <int D, bool BF16>
__device__ __forceinline__ void kw_unit(const uint16_t* x, int64_t x_row, int n, int at, uint8_t* codes, float* scale) {
    constexpr int LPR = D / 8;          // lanes per row (16 bytes each)
    constexpr int RPP = 32 / LPR;       // rows per pass
    constexpr int NV = 32 / RPP;        // passes of a whole block
    const int lane = threadIdx.x & 31, sub = lane / LPR, c = lane % LPR;
    uint4 v[NV];
#pragma unroll
    for (int i = 0; i < NV; ++i) {
        const int r = i * RPP + sub;
        v[i] = r < n ? __ldg(reinterpret_cast<const uint4*>(x + r * x_row) + c) : make_uint4(0u, 0u, 0u, 0u);
    }
    const float s_old = at > 0 ? *scale : 0.f;
    // magnitudes as whole numbers: of two values of one 16-bit type the larger has the larger pattern, a NaN the largest
    uint32_t most = 0;
#pragma unroll
    for (int i = 0; i < NV; ++i) {
        const uint32_t w[4] = {v[i].x, v[i].y, v[i].z, v[i].w};
#pragma unroll
        for (int k = 0; k < 4; ++k) most = __vmaxu2(most, w[k] & 0x7fff7fffu);
    }
#pragma unroll
    for (int d = 16; d; d >>= 1) most = __vmaxu2(most, __shfl_xor_sync(0xffffffffu, most, d));
    const uint32_t big = max(most & 0xffffu, most >> 16);
    auto wide = [](uint32_t h) -> float {
        if constexpr (BF16) return __uint_as_float(h << 16);
        else return __half2float(__ushort_as_half((unsigned short)h));
    };
    const bool poison = big >= (BF16 ? 0x7f80u : 0x7c00u) || !(s_old == s_old);
    const float need = kw_up11(wide(big) / 127.f);
    float s = need <= s_old ? s_old : fmaxf(need, kw_up11(1.25f * s_old));
    if (poison) s = __uint_as_float(0x7fc00000u);
    const float fit = s > 0.f ? s : 1.f;   // (0: a block of zeros; NaN: the codes do not matter, they become 0)
    auto code = [&](uint32_t h) -> uint32_t {
        const float q = rintf(__fdiv_rn(wide(h), fit));
        return poison ? 0u : (uint32_t)(int)q & 0xffu;
    };
#pragma unroll
    for (int i = 0; i < NV; ++i) {
        const int r = i * RPP + sub;
        if (r < n) {
            const uint32_t w[4] = {v[i].x, v[i].y, v[i].z, v[i].w};
            uint32_t o[2];
#pragma unroll
            for (int k = 0; k < 2; ++k)
                o[k] = code(w[2 * k] & 0xffffu) | code(w[2 * k] >> 16) << 8 | code(w[2 * k + 1] & 0xffffu) << 16 | code(w[2 * k + 1] >> 16) << 24;
            *reinterpret_cast<uint2*>(codes + (at + r) * D + 8 * c) = make_uint2(o[0], o[1]);
        }
    }
    if (s > s_old && at > 0 && !poison) {   // the older positions' codes on the larger scale
        for (int r = sub; r < at; r += RPP) {
            uint2* p = reinterpret_cast<uint2*>(codes + r * D + 8 * c);
            const uint2 u = *p;
            uint32_t o[2] = {0u, 0u};
#pragma unroll
            for (int k = 0; k < 8; ++k) {
                const int was = (int)(int8_t)((k < 4 ? u.x : u.y) >> (8 * (k & 3)));
                const uint32_t now = (uint32_t)(int)rintf(__fdiv_rn((float)was * s_old, s)) & 0xffu;
                o[k >> 2] |= now << (8 * (k & 3));
            }
            *p = make_uint2(o[0], o[1]);
        }
    }
    __syncwarp();   // (every lane has read the scale)
    if (lane == 0 && (at == 0 || !(s == s_old))) *scale = s;
}

template <int D, bool BF16>
__global__ void __launch_bounds__(KW_WARPS * 32) kv8_append_kernel(const __grid_constant__ KwArgs a) {
    __shared__ int begin[AQ_KV8_MAX_SEQS + 1];
    const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
    const int kv = warp & 1, hk = 2 * blockIdx.y + (warp >> 1);   // two heads' keys and values per CTA
    const int t0 = blockIdx.x * a.chunk;
    pdl_wait();
    if (a.row_start) {
        for (int i = threadIdx.x; i <= a.B; i += KW_WARPS * 32) begin[i] = __ldg(a.row_start + i);
        __syncthreads();
    }
    if (hk >= a.Hkv) return;
    // lane: one row of the chunk.  The rows that are the first of this step in their block lead a unit.
    const int t = t0 + lane;
    int at = 0, n = 0;            // its place in its block; rows of the unit (0: not a leader)
    int64_t blk = 0;              // the block's number (page, head, block of the page)
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
            const int64_t pos = (int64_t)__ldg(a.lens + b) - rows.n + i;
            at = (int)(pos & (AQ_KV8_BLOCK - 1));
            const int64_t tile = pos >> 5, pg = tile >> a.shift;
            if (pos < 0 || pg >= a.width) {
                kv8_report(KV8_BAD_LENGTH);
            } else if (i == 0 || at == 0) {
                const int page = __ldg(a.table + (int64_t)b * a.width + pg);
                if (page < 0 || page >= a.n_pages) {
                    kv8_report(KV8_BAD_PAGE);
                } else {
                    n = min(AQ_KV8_BLOCK - at, rows.n - i);
                    blk = (((int64_t)page * a.Hkv + hk) << a.shift) + (tile & ((1 << a.shift) - 1));
                }
            }
        }
    }
    for (unsigned leaders = __ballot_sync(0xffffffffu, n > 0); leaders; leaders &= leaders - 1) {
        const int src = __ffs(leaders) - 1;
        const int u_at = __shfl_sync(0xffffffffu, at, src), u_n = __shfl_sync(0xffffffffu, n, src);
        const int64_t u_blk = __shfl_sync(0xffffffffu, blk, src);
        kw_unit<D, BF16>(a.x[kv] + (int64_t)(t0 + src) * a.x_row + (int64_t)hk * D, a.x_row, u_n, u_at, a.codes[kv] + u_blk * AQ_KV8_BLOCK * D,
                         a.scales[kv] + u_blk);
    }
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
    // rows per CTA: a decode step's rows are a unit each and get a CTA each; of a prompt's rows one in 32 leads a unit
    const int pairs = (c.n_kv_heads + 1) / 2;
    a.chunk = 1;
    while (a.chunk < 32 && (int64_t)((T + a.chunk - 1) / a.chunk) * pairs > 4 * sm_count()) a.chunk *= 2;
    const dim3 grid((unsigned)((T + a.chunk - 1) / a.chunk), (unsigned)pairs), block(KW_WARPS * 32);
    cudaError_t e;
    const bool bf = dt == AQ_BF16;
    if (c.head_dim == 64) e = bf ? launch_pdl(kv8_append_kernel<64, true>, grid, block, 0, s, a) : launch_pdl(kv8_append_kernel<64, false>, grid, block, 0, s, a);
    else if (c.head_dim == 128) e = bf ? launch_pdl(kv8_append_kernel<128, true>, grid, block, 0, s, a) : launch_pdl(kv8_append_kernel<128, false>, grid, block, 0, s, a);
    else e = bf ? launch_pdl(kv8_append_kernel<256, true>, grid, block, 0, s, a) : launch_pdl(kv8_append_kernel<256, false>, grid, block, 0, s, a);
    count_launch();
    return e;
}

}  // namespace aq

#include "aq_kv8_attn.cuh"

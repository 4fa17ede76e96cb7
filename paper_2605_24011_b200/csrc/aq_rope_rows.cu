// Rotary positions of a step's rows: out[t][h] = x[t][h] with pair i of the first `rot` dims rotated by pos[t] * f_i (and multiplied
// by a magnitude), the other dims as they are.  Pairs (i, i + rot/2) or (2i, 2i + 1); frequencies from aq_rope_setup.  (No counterpart
// in the paper; aq_rope's many-row form.)
//
// Bound: HBM, each element read and written once.  The angle is formed in turns: pos * (f_i / 2 pi) in binary64, its whole part
// taken off exactly, the rest (half a turn at most, so an error of 2^-25 turns in binary32) into sincospif: far positions cost one
// multiplication in binary64 and no argument reduction.  A CTA has consecutive (row, head) pairs, forms its rows' angles once
// in shared memory for all of their heads, and asks for its elements before that.
#include <cuda_bf16.h>
#include <cuda_fp16.h>

#include <cmath>
#include <cstring>
#include <type_traits>

#include "aq_internal.h"

namespace aq {

struct RrArgs {
    const void* x;
    void* out;
    const int32_t* pos;
    int64_t x_row, out_row, pairs;   // pairs: rows * heads
    int heads, D, rot, per;          // per: (row, head) pairs per CTA
    float magnitude;
    double turns[AQ_ROPE_MAX_PAIRS];
};
constexpr int RR_THREADS = 256;
constexpr int RR_SMEM = 48 * 1024;

template <typename T> __device__ __forceinline__ float rr_wide(T v);
template <> __device__ __forceinline__ float rr_wide<float>(float v) { return v; }
template <> __device__ __forceinline__ float rr_wide<__half>(__half v) { return __half2float(v); }
template <> __device__ __forceinline__ float rr_wide<__nv_bfloat16>(__nv_bfloat16 v) { return __bfloat162float(v); }
template <typename T> __device__ __forceinline__ T rr_cast(float v);
template <> __device__ __forceinline__ float rr_cast<float>(float v) { return v; }
template <> __device__ __forceinline__ __half rr_cast<__half>(float v) { return __float2half_rn(v); }
template <> __device__ __forceinline__ __nv_bfloat16 rr_cast<__nv_bfloat16>(float v) { return __float2bfloat16_rn(v); }

// N neighbouring elements, N * sizeof(T) a multiple of 16 bytes and so aligned, or N = 1
template <typename T, int N>
struct alignas(N == 1 ? sizeof(T) : 16) RrVec { T v[N]; };

template <typename TS, typename TD, int N, bool HALF>
__global__ void __launch_bounds__(RR_THREADS) rope_rows_kernel(const __grid_constant__ RrArgs a) {
    extern __shared__ float2 table[];   // [rows of the CTA][rot / 2]: (cosine, sine) times the magnitude
    const int half = a.rot / 2;
    const int64_t p0 = (int64_t)blockIdx.x * a.per;
    const int64_t p1 = p0 + a.per < a.pairs ? p0 + a.per : a.pairs;
    const int row0 = (int)(p0 / a.heads), n_rows = (int)((p1 - 1) / a.heads) - row0 + 1;
    pdl_wait();
    for (int i = threadIdx.x; i < n_rows * half; i += RR_THREADS) {
        const int r = i / half, k = i - r * half;
        const double turn = (double)__ldg(a.pos + row0 + r) * a.turns[k];
        float s, c;
        sincospif((float)(2.0 * (turn - rint(turn))), &s, &c);
        table[i] = make_float2(c * a.magnitude, s * a.magnitude);
    }
    __syncthreads();
    // units of a head: rotated ones first, then the copied rest
    const int turned = HALF ? half / N : (N == 1 ? half : a.rot / N), units = turned + (a.D - a.rot) / N;
    const int n = (int)(p1 - p0) * units, base = (int)(p0 - (int64_t)row0 * a.heads);
#pragma unroll 2
    for (int i = threadIdx.x; i < n; i += RR_THREADS) {
        const int p = i / units, u = i - p * units;
        const int dr = (base + p) / a.heads, row = row0 + dr, h = base + p - dr * a.heads;
        if (__ldg(a.pos + row) < 0) continue;
        const TS* x = reinterpret_cast<const TS*>(a.x) + row * a.x_row + (int64_t)h * a.D;
        TD* y = reinterpret_cast<TD*>(a.out) + row * a.out_row + (int64_t)h * a.D;
        const float2* cs = table + dr * half;
        if (u < turned && (HALF || N == 1)) {
            // N pairs: elements lo + k and hi + k
            const int lo = HALF ? u * N : 2 * u, hi = HALF ? lo + half : lo + 1, k0 = HALF ? lo : u;
            const RrVec<TS, N> va = *reinterpret_cast<const RrVec<TS, N>*>(x + lo), vb = *reinterpret_cast<const RrVec<TS, N>*>(x + hi);
            RrVec<TD, N> oa, ob;
#pragma unroll
            for (int k = 0; k < N; ++k) {
                const float2 t = cs[k0 + k];
                const float c = rr_wide(va.v[k]), d = rr_wide(vb.v[k]);
                oa.v[k] = rr_cast<TD>(fmaf(c, t.x, -d * t.y));
                ob.v[k] = rr_cast<TD>(fmaf(d, t.x, c * t.y));
            }
            *reinterpret_cast<RrVec<TD, N>*>(y + lo) = oa;
            *reinterpret_cast<RrVec<TD, N>*>(y + hi) = ob;
        } else if (u < turned) {
            // N / 2 neighbouring pairs
            const int lo = u * N;
            const RrVec<TS, N> v = *reinterpret_cast<const RrVec<TS, N>*>(x + lo);
            RrVec<TD, N> o;
#pragma unroll
            for (int k = 0; k < N; k += 2) {
                const float2 t = cs[(lo + k) >> 1];
                const float c = rr_wide(v.v[k]), d = rr_wide(v.v[(k + 1) % N]);
                o.v[k] = rr_cast<TD>(fmaf(c, t.x, -d * t.y));
                o.v[(k + 1) % N] = rr_cast<TD>(fmaf(d, t.x, c * t.y));
            }
            *reinterpret_cast<RrVec<TD, N>*>(y + lo) = o;
        } else {
            const int lo = a.rot + (u - turned) * N;
            const RrVec<TS, N> v = *reinterpret_cast<const RrVec<TS, N>*>(x + lo);
            RrVec<TD, N> o;
#pragma unroll
            for (int k = 0; k < N; ++k) o.v[k] = rr_cast<TD>(rr_wide(v.v[k]));
            *reinterpret_cast<RrVec<TD, N>*>(y + lo) = o;
        }
    }
}

template <typename TS, typename TD>
static cudaError_t launch_rr(RrArgs& a, bool pairs_halved, cudaStream_t s) {
    // eight elements at a time where every such group is 16-byte aligned in both arrays
    const bool wide = ((reinterpret_cast<uintptr_t>(a.x) | reinterpret_cast<uintptr_t>(a.out)) & 15u) == 0 && a.x_row % 8 == 0 && a.out_row % 8 == 0 &&
                      a.D % 8 == 0 && a.rot % (pairs_halved ? 16 : 8) == 0;
    const unsigned grid = (unsigned)((a.pairs + a.per - 1) / a.per);
    const size_t smem = (size_t)((a.per - 1) / a.heads + 2) * (a.rot / 2) * sizeof(float2);
    cudaError_t e;
    if (wide) e = pairs_halved ? launch_pdl(rope_rows_kernel<TS, TD, 8, true>, dim3(grid), dim3(RR_THREADS), smem, s, a)
                               : launch_pdl(rope_rows_kernel<TS, TD, 8, false>, dim3(grid), dim3(RR_THREADS), smem, s, a);
    else e = pairs_halved ? launch_pdl(rope_rows_kernel<TS, TD, 1, true>, dim3(grid), dim3(RR_THREADS), smem, s, a)
                          : launch_pdl(rope_rows_kernel<TS, TD, 1, false>, dim3(grid), dim3(RR_THREADS), smem, s, a);
    count_launch();
    return e;
}

cudaError_t launch_rope_rows(const aq_rope_t& rope, const void* x, aq_dtype_t dt, int64_t x_row, void* out, aq_dtype_t out_dt, int64_t out_row,
                             int rows, int heads, int D, const int32_t* pos, cudaStream_t s) {
    RrArgs a;
    a.x = x; a.out = out; a.pos = pos; a.x_row = x_row; a.out_row = out_row; a.pairs = (int64_t)rows * heads;
    a.heads = heads; a.D = D; a.rot = rope.rot_dim; a.magnitude = rope.magnitude;
    memcpy(a.turns, rope.turns, sizeof(a.turns));
    // enough CTAs for every SM to have some, otherwise as many pairs as share a row's angles well; at most what the table holds
    const int most = RR_SMEM / (int)sizeof(float2) / (rope.rot_dim / 2) - 1;   // rows in a CTA's table, one of them broken at each end
    int64_t per = (a.pairs + 4 * sm_count() - 1) / (4 * sm_count());
    if (per > 64) per = 64;
    if (per > (int64_t)(most - 1) * heads) per = (int64_t)(most - 1) * heads;
    a.per = (int)(per < 1 ? 1 : per);
    const bool halves = rope.layout == AQ_ROPE_HALF;
    if (dt == AQ_F16) return launch_rr<__half, __half>(a, halves, s);
    if (dt == AQ_BF16) return launch_rr<__nv_bfloat16, __nv_bfloat16>(a, halves, s);
    if (out_dt == AQ_F16) return launch_rr<float, __half>(a, halves, s);
    if (out_dt == AQ_BF16) return launch_rr<float, __nv_bfloat16>(a, halves, s);
    return launch_rr<float, float>(a, halves, s);
}

// Frequencies, host only: f_i = theta^(-2i/r) over 2 pi, in turns per position.
void rope_setup(int rot, int layout, double theta, int scaling, double factor, double trained, double low, double high, double magnitude, aq_rope_t* out) {
    memset(out, 0, sizeof(*out));
    out->rot_dim = rot;
    out->layout = layout;
    const double two_pi = 6.283185307179586476925286766559;
    if (scaling == AQ_ROPE_BASE && rot > 2) theta *= std::pow(factor, (double)rot / (rot - 2));
    const double step = -2.0 / rot * std::log2(theta);
    for (int i = 0; i < rot / 2; ++i) {
        double f = std::exp2(step * i);
        if (scaling == AQ_ROPE_LINEAR) f /= factor;
        if (scaling == AQ_ROPE_PARTS) {
            double keep = (trained * f / two_pi - low) / (high - low);
            keep = keep < 0 ? 0 : (keep > 1 ? 1 : keep);
            f = f * keep + f / factor * (1 - keep);
        }
        out->turns[i] = f / two_pi;
    }
    if (magnitude > 0) out->magnitude = (float)magnitude;
    else out->magnitude = scaling == AQ_ROPE_PARTS ? (float)(0.1 * std::log(factor) + 1.0) : 1.0f;
}

}  // namespace aq

// Rotary positions of a step's rows: out[t][h] = x[t][h] with pair i of the first `rot` dims rotated by pos[t] * f_i (and multiplied
// by a magnitude), the other dims as they are.  Pairs (i, i + rot/2) or (2i, 2i + 1); frequencies from aq_rope_setup.  (No counterpart
// in the paper; aq_rope's many-row form.)
//
// Bound: HBM, each element read and written once.  The angle is formed in turns: pos * (f_i / 2 pi) in binary64, its whole part
// taken off exactly, the rest (half a turn at most, so an error of 2^-25 turns in binary32) into sincospif: far positions cost one
// multiplication in binary64 and no argument reduction.  A CTA has consecutive (row, head) pairs, one wave of CTAs all of them; it forms
// its rows' angles once for all of their heads, in shared memory, so laid out that neighbouring threads read neighbouring entries.
// 4000 rows x 40 heads of 128, bfloat16: 15.1 us, 0.83 of the measured copy rate.  With more units per thread or fewer CTAs per SM it is
// slower (4 units held while the angles are formed: 28.8 us): issue slots and threads, not bytes in flight, are what it runs out of.
#include <cuda_bf16.h>
#include <cuda_fp16.h>

#include <cmath>
#include <cstring>
#include <type_traits>

#include "aq_internal.h"
#include "aq_kv8_runs.h"

namespace aq {

struct RrArgs {
    const void* x;
    void* out;
    const int32_t* pos;
    int64_t x_row, out_row, pairs;   // pairs: rows * heads
    int heads, D, rot, per;          // per: (row, head) pairs per CTA
    int units, turned;               // units of a head: rotated ones first, then the copied rest
    uint32_t heads_magic, units_magic;
    float magnitude;
    double turns[AQ_ROPE_MAX_PAIRS];
};
constexpr int RR_THREADS = 256, RR_UNITS = 2;   // units per thread and turn
constexpr int RR_SMEM = 40 * 1024, RR_CTAS = 5;   // per SM
constexpr int RR_AHEAD = 32 * 1024;

// N neighbouring elements as they lie in memory (N = 8: 16-byte aligned; N = 1), and as float32.
template <typename T, int N>
struct RrVec {
    uint4 w[N * sizeof(T) / 16];
    __device__ __forceinline__ void load(const T* p) {
#pragma unroll
        for (int i = 0; i < (int)(N * sizeof(T) / 16); ++i) w[i] = reinterpret_cast<const uint4*>(p)[i];
    }
    __device__ __forceinline__ void store(T* p) const {
#pragma unroll
        for (int i = 0; i < (int)(N * sizeof(T) / 16); ++i) reinterpret_cast<uint4*>(p)[i] = w[i];
    }
    __device__ __forceinline__ uint32_t& word(int i) { return reinterpret_cast<uint32_t*>(w)[i]; }
    __device__ __forceinline__ void get(float (&f)[N]) {
        if constexpr (sizeof(T) == 4) {
#pragma unroll
            for (int i = 0; i < N; ++i) f[i] = __uint_as_float(word(i));
        } else {
#pragma unroll
            for (int i = 0; i < N / 2; ++i) {
                const uint32_t v = word(i);
                if constexpr (std::is_same<T, __half>::value) {
                    const float2 h = __half22float2(*reinterpret_cast<const __half2*>(&v));
                    f[2 * i] = h.x; f[2 * i + 1] = h.y;
                } else {
                    f[2 * i] = __uint_as_float(v << 16); f[2 * i + 1] = __uint_as_float(v & 0xffff0000u);
                }
            }
        }
    }
    __device__ __forceinline__ void set(const float (&f)[N]) {
        if constexpr (sizeof(T) == 4) {
#pragma unroll
            for (int i = 0; i < N; ++i) word(i) = __float_as_uint(f[i]);
        } else {
#pragma unroll
            for (int i = 0; i < N / 2; ++i) {
                if constexpr (std::is_same<T, __half>::value) {
                    const __half2 h = __floats2half2_rn(f[2 * i], f[2 * i + 1]);
                    word(i) = *reinterpret_cast<const uint32_t*>(&h);
                } else {
                    const __nv_bfloat162 h = __floats2bfloat162_rn(f[2 * i], f[2 * i + 1]);
                    word(i) = *reinterpret_cast<const uint32_t*>(&h);
                }
            }
        }
    }
};
template <typename T>
struct RrVec<T, 1> {
    T w;
    __device__ __forceinline__ void load(const T* p) { w = *p; }
    __device__ __forceinline__ void store(T* p) const { *p = w; }
    __device__ __forceinline__ void get(float (&f)[1]) { f[0] = (float)w; }
    __device__ __forceinline__ void set(const float (&f)[1]) {
        if constexpr (sizeof(T) == 4) w = f[0];
        else if constexpr (std::is_same<T, __half>::value) w = __float2half_rn(f[0]);
        else w = __float2bfloat16_rn(f[0]);
    }
};

// A unit: N pairs (HALF, or N = 1: elements lo + k and hi + k), or N neighbouring elements.
template <typename TS, typename TD, int N, bool HALF>
__global__ void __launch_bounds__(RR_THREADS, RR_CTAS) rope_rows_kernel(const __grid_constant__ RrArgs a) {
    extern __shared__ float2 table[];   // [rows of the CTA][rot / 2]: (cosine, sine) times the magnitude
    constexpr bool TWO = HALF || N == 1;
    const int half = a.rot / 2;
    const int64_t p0 = (int64_t)blockIdx.x * a.per;
    const int count = (int)(p0 + a.per < a.pairs ? a.per : a.pairs - p0);
    const int row0 = (int)(p0 / a.heads), base = (int)(p0 - (int64_t)row0 * a.heads);
    const int n_rows = (int)kv8_div((uint32_t)(base + count - 1), a.heads_magic) + 1, n = count * a.units;
    const TS* x0 = reinterpret_cast<const TS*>(a.x) + (int64_t)row0 * a.x_row;
    TD* y0 = reinterpret_cast<TD*>(a.out) + (int64_t)row0 * a.out_row;
    pdl_wait();
    pdl_launch_dependents();
    // a CTA with work for several turns asks for its first 32 KB while the angles are formed (4000 rows x 40 heads: 16.9 -> 15.1 us, 20000 rows
    // 76.8 -> 75.8, with all of them on their way at once 81.0; with fewer turns the extra instructions cost more than they save)
    if (n > 2 * RR_UNITS * RR_THREADS) {
        for (int p = threadIdx.x; p < min(count, RR_AHEAD / (a.D * (int)sizeof(TS))); p += RR_THREADS) {
            const int dr = (int)kv8_div((uint32_t)(base + p), a.heads_magic), h = base + p - dr * a.heads;
            const TS* x = x0 + (int64_t)dr * a.x_row + h * a.D;
            for (int k = 0; k < a.D; k += 128 / (int)sizeof(TS)) asm volatile("prefetch.global.L2 [%0];" ::"l"(x + k));
        }
    }
    // pair e of unit u lies at e * turned + u: neighbouring threads read neighbouring entries
    constexpr int PPU = TWO ? N : N / 2;   // pairs per unit
    for (int i = threadIdx.x; i < n_rows * half; i += RR_THREADS) {
        const int r = i / half, k = i - r * half;
        const double turn = (double)a.pos[row0 + r] * a.turns[k];
        float s, c;
        sincospif((float)(2.0 * (turn - rint(turn))), &s, &c);
        table[r * half + k % PPU * a.turned + k / PPU] = make_float2(c * a.magnitude, s * a.magnitude);
    }
    __syncthreads();
    for (int i0 = threadIdx.x; i0 < n; i0 += RR_UNITS * RR_THREADS) {
        // all loads first (the compiler cannot know that one unit's stores are not another's elements)
        int lo[RR_UNITS], angle[RR_UNITS];   // first element; its angle in the table, -1: copied, -2: nothing to do
        TD* y[RR_UNITS];
        RrVec<TS, N> va[RR_UNITS], vb[TWO ? RR_UNITS : 1];
#pragma unroll
        for (int k = 0; k < RR_UNITS; ++k) {
            const int i = min(i0 + k * RR_THREADS, n - 1);
            const int p = (int)kv8_div((uint32_t)i, a.units_magic), u = i - p * a.units;
            const int dr = (int)kv8_div((uint32_t)(base + p), a.heads_magic), h = base + p - dr * a.heads;
            const TS* x = x0 + (int64_t)dr * a.x_row + h * a.D;
            y[k] = y0 + (int64_t)dr * a.out_row + h * a.D;
            const bool turned = u < a.turned;
            lo[k] = turned ? (HALF || N > 1 ? u * N : 2 * u) : a.rot + (u - a.turned) * N;
            angle[k] = turned ? dr * half + u : -1;
            if (i0 + k * RR_THREADS >= n || a.pos[row0 + dr] < 0) angle[k] = -2;
            va[k].load(x + lo[k]);
            if (TWO) vb[TWO ? k : 0].load(x + (turned ? lo[k] + (HALF ? half : 1) : lo[k]));
        }
#pragma unroll
        for (int k = 0; k < RR_UNITS; ++k) {
            if (angle[k] == -2) continue;
            float fa[N], fb[N];
            RrVec<TD, N> o;
            va[k].get(fa);
            if (angle[k] >= 0) {
                if (TWO) {
                    vb[TWO ? k : 0].get(fb);
#pragma unroll
                    for (int e = 0; e < N; ++e) {
                        const float2 t = table[angle[k] + e * a.turned];
                        const float c = fa[e], d = fb[e];
                        fa[e] = fmaf(c, t.x, -d * t.y);
                        fb[e] = fmaf(d, t.x, c * t.y);
                    }
                    o.set(fb);
                    o.store(y[k] + lo[k] + (HALF ? half : 1));
                } else {
#pragma unroll
                    for (int e = 0; e < N; e += 2) {
                        const float2 t = table[angle[k] + e / 2 * a.turned];
                        const float c = fa[e], d = fa[(e + 1) % N];
                        fa[e] = fmaf(c, t.x, -d * t.y);
                        fa[(e + 1) % N] = fmaf(d, t.x, c * t.y);
                    }
                }
            }
            o.set(fa);
            o.store(y[k] + lo[k]);
        }
    }
}

template <typename TS, typename TD>
static cudaError_t launch_rr(RrArgs& a, bool pairs_halved, cudaStream_t s) {
    // eight elements at a time where every such group is 16-byte aligned in both arrays
    const bool wide = ((reinterpret_cast<uintptr_t>(a.x) | reinterpret_cast<uintptr_t>(a.out)) & 15u) == 0 && a.x_row % 8 == 0 && a.out_row % 8 == 0 &&
                      a.D % 8 == 0 && a.rot % (pairs_halved ? 16 : 8) == 0;
    const int N = wide ? 8 : 1;
    a.turned = pairs_halved || !wide ? a.rot / 2 / N : a.rot / N;
    a.units = a.turned + (a.D - a.rot) / N;
    a.units_magic = kv8_magic((uint32_t)a.units);
    a.heads_magic = kv8_magic((uint32_t)a.heads);
    // one wave of CTAs; no more rows than the table has room for
    const int64_t rows = RR_SMEM / (int64_t)sizeof(float2) / (a.rot / 2) - 1;   // in a CTA's table, broken ones at both ends
    int64_t per = (a.pairs + RR_CTAS * sm_count() - 1) / (RR_CTAS * sm_count());
    if (per > 1024) per = 1024;
    if (per > (rows - 1) * a.heads) per = (rows - 1) * a.heads;
    a.per = (int)(per < 1 ? 1 : per);
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

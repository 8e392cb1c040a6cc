// Projections in 8-bit integers (include/ebrl_i8.h): rows to codes, and the
// product of two operands of codes.  Three kernels multiply, by the shape (i8_plan):
// 256 x 256 tiles, LDS rings of smaller ones, and slices of the weights for few rows.
#include <hip/hip_runtime.h>

#include <type_traits>

#include "../../include/ebrl.h"
#include "../../include/ebrl_i8.h"
#include "kernels.h"
#include "tile.h"

namespace ebrl {

typedef int i32x4 __attribute__((ext_vector_type(4)));

// Vectors that lie in memory at the alignment of an element: global loads and stores
// take any, and a row segment stays one instruction.  9216 rows of 4095 columns, fp32, normed
// 38 us (of 4096 39), bf16, gated 63 (42); read by elements they took 76 and 102.
typedef f32x4 f32x4_any __attribute__((aligned(4)));
typedef u32x4 u32x4_any __attribute__((aligned(2)));
typedef uint32_t u32x2_any __attribute__((ext_vector_type(2), aligned(2)));
typedef __bf16 bf16x4_any __attribute__((ext_vector_type(4), aligned(2)));
template <typename T> EBRL_DEV void st4_any(T* p, f32x4 v) {
    if constexpr (sizeof(T) == 4) *reinterpret_cast<f32x4_any*>(p) = v;
    else *reinterpret_cast<bf16x4_any*>(p) = bf16x4_any{(__bf16)v[0], (__bf16)v[1], (__bf16)v[2], (__bf16)v[3]};
}

constexpr int I8_MAX_COLS = 1 << 20;
constexpr int I8_MAX_K = 131056;            // 2^14 K < 2^31, K a multiple of 16
constexpr int64_t I8_MAX_LD = 1 << 23;      // a tile's byte offsets are 32-bit numbers
constexpr int64_t I8_MAX_TILES = 1 << 23;

// ------------------------------------------------------- rows to codes --
// y, its largest size and the quotients are 64-bit: a code is off by one where y /
// s is nearer to a border than its error, and one such code moves a product by
// about 1e-4 of its size.  With 32-bit y that is one code in 1e5, with 64-bit ones
// none.  The vector units do 64-bit adds and products at the rate of 32-bit ones.
//
// Bound by memory from some thousand rows on: 9216 fp32 rows of 4092, normed, 37 us (5.1
// TB/s; of 4096, whose rows start on the same channels, 39), as they are 32 (5.9), bf16 ones as
// they are 20 (5.7); bf16 ones, normed, by their vector instructions, 30 (of 4096 33); a row
// alone 2.7 us, a launch and two memory latencies.

// 1 / d and 1 / sqrt(d): two steps of Newton's, 2^-23, 2^-46, then all bits.
EBRL_DEV double i8_rcp(double d) {
    double r = __builtin_amdgcn_rcp(d);
    r = fma(r, fma(-d, r, 1.0), r);
    return fma(r, fma(-d, r, 1.0), r);
}
EBRL_DEV double i8_rsqrt(double d) {
    double r = __builtin_amdgcn_rsq(d);
    r = fma(0.5 * r, fma(-d * r, r, 1.0), r);
    return fma(0.5 * r, fma(-d * r, r, 1.0), r);
}
// silu(g) u.  exp(-g) = 2^n 2^f, |f| <= 1/2, 2^f by its Taylor series: the first
// term left out is 2e-16.  The exponent is held to +-690, where silu is g or below
// every scale.  1 / ln(2) in two parts keeps f to all its bits.
EBRL_DEV double i8_gate(float g32, float u32) {
    const double g = g32, h = fmin(fmax(g, -690.0), 690.0);
    const double n = rint(h * -1.4426950408889634);
    const double f = fma(h, -2.0355273740931033e-17, fma(h, -1.4426950408889634, -n));
    double p = 2.5678435993488205141e-11;       // ln(2)^k / k!, k = 12 .. 0
    p = fma(p, f, 4.4455382718708114976e-10);
    p = fma(p, f, 7.0549116208011233299e-9);
    p = fma(p, f, 1.0178086009239699728e-7);
    p = fma(p, f, 1.3215486790144309488e-6);
    p = fma(p, f, 1.5252733804059840280e-5);
    p = fma(p, f, 1.5403530393381609954e-4);
    p = fma(p, f, 1.3333558146428443423e-3);
    p = fma(p, f, 9.6181291076284771619e-3);
    p = fma(p, f, 5.5504108664821579953e-2);
    p = fma(p, f, 2.4022650695910071233e-1);
    p = fma(p, f, 6.9314718055994530942e-1);
    p = fma(p, f, 1.0);
    return g * i8_rcp(1.0 + ldexp(p, (int)n)) * (double)u32;
}
// The same in 32 bits, for |g| <= 80, off by less than 2^-17 of its size: the
// exponent by 2^-18 and the constant's 2^-20, the others by a few ulps.  The gate
// comes last: what is below the normal floats before it, off by 2^-149, stays below
// any code of rows that this is used for; silu(g) of a denormal g would lose bits
// that a large u brings up again.
EBRL_DEV float i8_gate_fast(float g, float u) {
    return g * (__builtin_amdgcn_rcpf(1.0f + __builtin_amdgcn_exp2f(g * -1.44269504f)) * u);
}
// y / s to the nearest whole number, ties to even.
EBRL_DEV uint32_t i8_code(double y, double s) { return (uint32_t)(int)rint(y / s); }
// The low bytes of four words.
EBRL_DEV uint32_t i8_pack(uint32_t a, uint32_t b, uint32_t c, uint32_t d) {
    return __builtin_amdgcn_perm(__builtin_amdgcn_perm(d, c, 0x0c0c0400), __builtin_amdgcn_perm(b, a, 0x0c0c0400), 0x05040100);
}
// The scale that rows with |y| <= top need; infinity: none, the row is not finite.
EBRL_DEV float i8_scale(double top, bool bad) {
    const float s = fmaxf((float)(top / 127.0), 0x1p-100f);
    return bad || !(s <= 3.40282347e38f) ? INFINITY : s;
}
// As wave_sum, on both halves of a double.
template <int CTRL> EBRL_DEV double i8_dpp(double v) {
    const uint2 w = __builtin_bit_cast(uint2, v);
    return __builtin_bit_cast(double, make_uint2(
        (unsigned)__builtin_amdgcn_update_dpp(0, (int)w.x, CTRL, 0xF, 0xF, false),
        (unsigned)__builtin_amdgcn_update_dpp(0, (int)w.y, CTRL, 0xF, 0xF, false)));
}
template <typename F> EBRL_DEV double i8_over_wave(double v, F op) {
    v = op(v, i8_dpp<DPP_SWAP1>(v));
    v = op(v, i8_dpp<DPP_SWAP2>(v));
    v = op(v, i8_dpp<DPP_HALF_MIRROR>(v));
    v = op(v, i8_dpp<DPP_MIRROR>(v));
    const uint2 w = __builtin_bit_cast(uint2, v);
    auto lane = [&](int l) {
        return __builtin_bit_cast(double, make_uint2((unsigned)__builtin_amdgcn_readlane((int)w.x, l),
                                                     (unsigned)__builtin_amdgcn_readlane((int)w.y, l)));
    };
    return op(op(lane(0), lane(16)), op(lane(32), lane(48)));
}
EBRL_DEV double i8_wave_sum(double v) { return i8_over_wave(v, [](double a, double b) { return a + b; }); }
EBRL_DEV double i8_wave_max(double v) { return i8_over_wave(v, [](double a, double b) { return fmax(a, b); }); }

// Eight neighbours of a row; those from `left` on are zeros.
template <typename T> EBRL_DEV void i8_load8(const T* p, int left, float (&v)[8]) {
    if (left >= 8) {
        if constexpr (sizeof(T) == 4) {
            const f32x4 a = *reinterpret_cast<const f32x4_any*>(p), b = *reinterpret_cast<const f32x4_any*>(p + 4);
#pragma unroll
            for (int e = 0; e < 4; ++e) { v[e] = a[e]; v[4 + e] = b[e]; }
        } else {
            const u32x4 w = *reinterpret_cast<const u32x4_any*>(p);
#pragma unroll
            for (int e = 0; e < 4; ++e) {
                v[2 * e] = __uint_as_float(w[e] << 16);
                v[2 * e + 1] = __uint_as_float(w[e] & 0xFFFF0000u);
            }
        }
    } else {
#pragma unroll
        for (int e = 0; e < 8; ++e) v[e] = e < left ? ld_elem<T>(p + e) : 0.f;
    }
}
// The codes of eight neighbours in each of CHUNKS places, `step` columns apart from j on (those
// of columns past the last are codes of zeros); columns from `wide` on are left as they are.
// Adding 1.5 * 2^20 and a half rounds y inv + 1/2 to 2^-32ths, with the whole number in the high
// word's low byte and the fraction in the low word.  The product is off by less than 2^-36 (of
// which a sum of 2^20 squares is most), so that is the one nearest to y / s unless the fraction
// is 0: then y / s may be a tie, or on either side of one, and `exactly(column)` gives its code by
// divisions, stored over the first (one in 2^32, but for data of few bits).
template <int CHUNKS, typename F>
EBRL_DEV void i8_store(int8_t* out, const double (&y)[CHUNKS][8], int j, int step, int wide, double inv, bool bad, F exactly) {
    auto code = [&](int c, int e) { return __builtin_bit_cast(uint2, fma(y[c][e], inv, 1572864.5)); };
    uint32_t least = ~0u;
#pragma unroll
    for (int c = 0; c < CHUNKS; ++c) {
        uint32_t k[8];
#pragma unroll
        for (int e = 0; e < 8; ++e) {
            const uint2 w = code(c, e);
            k[e] = w.y;
            least = min(least, w.x);
        }
        const uint32_t lo = i8_pack(k[0], k[1], k[2], k[3]), hi = i8_pack(k[4], k[5], k[6], k[7]);
        if (j + c * step < wide) *reinterpret_cast<uint2*>(out + j + c * step) = bad ? make_uint2(0, 0) : make_uint2(lo, hi);
    }
    if (least == 0 && !bad) {
        unsigned these = 0;
#pragma unroll
        for (int c = 0; c < CHUNKS; ++c)
#pragma unroll
            for (int e = 0; e < 8; ++e) these |= (code(c, e).x == 0 ? 1u : 0u) << (8 * c + e);
        for (; these; these &= these - 1) {
            const int i = __builtin_ctz(these), at = j + (i >> 3) * step + (i & 7);
            out[at] = (int8_t)exactly(at);
        }
    }
}

// y of a row as it is or normed, read again; ss: its sum of squares.  With the division
// last, y is exact wherever it and the root are numbers of 64 bits.
template <typename T, int OP> EBRL_DEV double i8_value(const ebrl_i8_quant_args& a, const T* x, int j, double ss) {
    const double v = ld_elem<T>(x + j);
    if constexpr (OP == EBRL_I8_ROWS) return v;
    else return (a.gain ? v * (double)a.gain[j] : v) / sqrt(ss / a.cols + (double)a.eps);
}
// The largest value, and the sum, over a row's waves; `red`: a word for each.
template <int WAVES, typename V> EBRL_DEV V i8_over_waves(V v, V* red, bool sum) {
    if constexpr (WAVES > 1) {
        __syncthreads();
        if ((threadIdx.x & 63) == 0) red[threadIdx.x >> 6] = v;
        __syncthreads();
        v = red[0];
#pragma unroll
        for (int w = 1; w < WAVES; ++w) v = sum ? v + red[w] : (V)fmax(v, red[w]);
    }
    return v;
}
EBRL_DEV float i8_most(float m, float v) { return __builtin_elementwise_maximum(m, fabsf(v)); }   // NaN stays

// Rows of at most 512 CHUNKS columns a wave, held in registers from one read to the
// codes: a thread has eight neighbours in each of CHUNKS places.  One wave: four rows a
// workgroup, else a workgroup a row.  Rows of 1025 to 2048 columns on four waves with
// one place (591 rows of 1283: 3.8 us; three with two 4.8); the count of waves is a
// constant, because a loop over it waits for each wave's word in turn (a row of 4096 3.2
// us against 3.6) and sixteen doubles at once take the registers of a wave in four.
//
// Plain and normed rows are 64-bit throughout, but for the maximum of plain ones, which is a
// float.  A row's waves meet once (9216 normed fp32 rows of 11008: 114 us; sum and maximum one
// after the other 161).  Gated rows, whose 64-bit exponentials would take twice the
// time of reading them, have 32-bit values, maximum and codes; what
// lies nearer to a border than these are exact (EB, twice their error) is computed once
// more in 64 bits, one code in 1e4, and so is a whole row where 32 bits do not do
// (near the ends of their range, or not finite).  9216 rows of 11008 (bf16): 124 us, 4.1
// TB/s, 195 with 64 bits throughout.  Two workgroups of twelve waves share a CU, whose
// vector units are busy 73 % of the cycles: the rest is the wait for a row and the exchange.
// Eight waves with three places 149 (159 held to three workgroups a CU), six with four
// 186; persistent workgroups with the next row in flight 152.
template <typename T, int OP, int WAVES, int CHUNKS>
__global__ __launch_bounds__(WAVES == 1 ? 256 : 64 * WAVES) void i8_quant_kernel(ebrl_i8_quant_args a)
{
    constexpr bool ONE = WAVES == 1;
    constexpr int threads = 64 * WAVES;
    constexpr bool GATE = OP == EBRL_I8_SWIGLU;
    constexpr float EB = 0x1p-16f;
    __shared__ double red_sum[WAVES], red_top[WAVES];
    __shared__ float red_max[WAVES], red_scale[WAVES];
    const int tid = ONE ? threadIdx.x & 63 : threadIdx.x;
    const int row = ONE ? blockIdx.x * 4 + (threadIdx.x >> 6) : blockIdx.x;
    if (row >= a.rows) return;
    const T* const x = (const T*)a.x + (size_t)row * a.ldx;
    const T* const up = GATE ? (const T*)a.up + (size_t)row * a.ldup : nullptr;
    int8_t* const out = a.codes + (size_t)row * a.ldc;
    const int wide = (a.cols + 15) / 16 * 16;
    float z[CHUNKS][8], u[CHUNKS][8];     // u: the gated rows' other factor, or the norm's gain
#pragma unroll
    for (int c = 0; c < CHUNKS; ++c) {
        const int j = (c * threads + tid) * 8;
        i8_load8<T>(x + j, a.cols - j, z[c]);
        if constexpr (GATE) i8_load8<T>(up + j, a.cols - j, u[c]);
        if constexpr (OP == EBRL_I8_RMSNORM)
            if (a.gain) i8_load8<float>(a.gain + j, a.cols - j, u[c]);
    }
    if constexpr (!GATE) {
        // normed rows: factor x gain, whose product x gain is exact in 64 bits, so that the
        // largest is known with the sum of squares, in one exchange
        double y[CHUNKS][8], top = 0.0, ss = 0.0, factor = 1.0;
        float most = 0.f;       // of what is not finite wherever a y is, for all that ss does not tell
        const double mean = 1.0 / a.cols;
#pragma unroll
        for (int c = 0; c < CHUNKS; ++c)
#pragma unroll
            for (int e = 0; e < 8; ++e) {
                y[c][e] = z[c][e];
                if constexpr (OP == EBRL_I8_RMSNORM) {
                    ss = fma(y[c][e], y[c][e], ss);
                    if (a.gain) {
                        y[c][e] *= (double)u[c][e];
                        most = i8_most(most, u[c][e]);
                    }
                    top = fmax(top, fabs(y[c][e]));
                } else {
                    most = i8_most(most, z[c][e]);
                }
            }
        float s;
        if constexpr (OP == EBRL_I8_RMSNORM) {
            ss = i8_wave_sum(ss);
            top = i8_wave_max(most < INFINITY ? top : (double)INFINITY);
            if constexpr (WAVES > 1) {
                if ((threadIdx.x & 63) == 0) {
                    red_sum[threadIdx.x >> 6] = ss;
                    red_top[threadIdx.x >> 6] = top;
                }
                __syncthreads();
                ss = red_sum[0];
                top = red_top[0];
#pragma unroll
                for (int w = 1; w < WAVES; ++w) {
                    ss += red_sum[w];
                    top = fmax(top, red_top[w]);
                }
            }
            factor = i8_rsqrt(fma(ss, mean, (double)a.eps));
            top *= factor;      // NaN for squares that are none or infinite
            s = i8_scale(top, !(top < (double)INFINITY));
        } else {
            s = i8_over_waves<WAVES>(wave_max(i8_scale(most, !(most < INFINITY))), red_max, false);
        }
        const bool bad = s == INFINITY;
        const double sd = s, inv = factor * i8_rcp(sd);
        if (tid == 0) a.scales[row] = bad ? __builtin_nanf("") : s;
        i8_store<CHUNKS>(out, y, tid * 8, threads * 8, wide, inv, bad,
                         [&](int j) { return i8_code(i8_value<T, OP>(a, x, j, ss), sd); });
    } else {
        auto exactly = [&](int j) { return i8_gate(ld_elem<T>(x + j), ld_elem<T>(up + j)); };
        float most = 0.f, gate = 0.f;
#pragma unroll
        for (int c = 0; c < CHUNKS; ++c)
#pragma unroll
            for (int e = 0; e < 8; ++e) {
                gate = i8_most(gate, z[c][e]);
                z[c][e] = i8_gate_fast(z[c][e], u[c][e]);
                most = i8_most(most, z[c][e]);
            }
        const bool fits = most <= 0x1p120f && gate <= 80.f;
        float m = wave_max(fits ? most : INFINITY), s = 0.f;
        if (m <= 0x1p120f && m >= 0x1p-81f) {
            // what may be the wave's largest one, from the row read again; those of waves
            // that are left out are below every wave's that counts
            const float may = m * (1.0f - EB);
            double top = 0.0;
            if (most >= may) {
#pragma unroll
                for (int c = 0; c < CHUNKS; ++c) {
                    unsigned these = 0;
#pragma unroll
                    for (int e = 0; e < 8; ++e) these |= (fabsf(z[c][e]) >= may ? 1u : 0u) << e;
                    for (; these; these &= these - 1)
                        top = fmax(top, fabs(exactly((c * threads + tid) * 8 + __builtin_ctz(these))));
                }
            }
            s = wave_max(i8_scale(top, false));
        }
        if constexpr (WAVES > 1) {
            if ((threadIdx.x & 63) == 0) {
                red_max[threadIdx.x >> 6] = m;
                red_scale[threadIdx.x >> 6] = s;
            }
            __syncthreads();
            m = red_max[0];
            s = red_scale[0];
#pragma unroll
            for (int w = 1; w < WAVES; ++w) {
                m = fmaxf(m, red_max[w]);
                s = fmaxf(s, red_scale[w]);
            }
        }
        if (m <= 0x1p120f && m >= 0x1p-80f) {
            const double sd = s;
            const float invf = (float)i8_rcp(sd), eb = invf * EB;
            if (tid == 0) a.scales[row] = s;
#pragma unroll
            for (int c = 0; c < CHUNKS; ++c) {
                const int j = (c * threads + tid) * 8;
                uint32_t k[8];
                float border[8], near = 0.f;
#pragma unroll
                for (int e = 0; e < 8; ++e) {
                    // adding 1.5 * 2^23 rounds to a whole number in the low bits
                    const float t = fmaf(z[c][e], invf, 12582912.0f);
                    k[e] = __float_as_uint(t);
                    border[e] = fmaf(fabsf(z[c][e]), eb, fabsf(fmaf(z[c][e], invf, -(t - 12582912.0f))));
                    near = fmaxf(near, border[e]);
                }
                uint32_t lo = i8_pack(k[0], k[1], k[2], k[3]), hi = i8_pack(k[4], k[5], k[6], k[7]);
                if (near >= 0.5f) {
                    unsigned these = 0;
#pragma unroll
                    for (int e = 0; e < 8; ++e) these |= (border[e] >= 0.5f ? 1u : 0u) << e;
                    for (; these; these &= these - 1) {
                        const int e = __builtin_ctz(these), at = (e & 3) * 8;
                        const uint32_t code = i8_code(exactly(j + e), sd) & 255;
                        if (e < 4) lo = (lo & ~(255u << at)) | code << at;
                        else hi = (hi & ~(255u << at)) | code << at;
                    }
                }
                if (j < wide) *reinterpret_cast<uint2*>(out + j) = make_uint2(lo, hi);
            }
            return;
        }
        double top = 0.0, nan = 0.0;
#pragma unroll 1
        for (int j = tid; j < a.cols; j += threads) {
            const double y = exactly(j);
            top = fmax(top, fabs(y));
            nan = fma(y, 0.0, nan);
        }
        s = i8_over_waves<WAVES>(wave_max(i8_scale(top, !(nan == 0.0))), red_max, false);
        const bool bad = s == INFINITY;
        const double sd = s;
        if (tid == 0) a.scales[row] = bad ? __builtin_nanf("") : s;
#pragma unroll 1
        for (int j = tid; j < wide; j += threads)
            out[j] = j < a.cols && !bad ? (int8_t)i8_code(exactly(j), sd) : (int8_t)0;
    }
}

// Longer rows: read once more for each step.
template <typename T, int OP>
__global__ __launch_bounds__(1024) void i8_quant_long_kernel(ebrl_i8_quant_args a)
{
    __shared__ double red_sum[16];
    __shared__ float red_max[16];
    const int tid = threadIdx.x, row = blockIdx.x;
    const T* const x = (const T*)a.x + (size_t)row * a.ldx;
    double factor = 1.0, ss = 0.0;
    if constexpr (OP == EBRL_I8_RMSNORM) {
        for (int j = tid * 8; j < a.cols; j += 8192) {
            float v[8];
            i8_load8<T>(x + j, a.cols - j, v);
#pragma unroll
            for (int e = 0; e < 8; ++e) ss = fma((double)v[e], (double)v[e], ss);
        }
        ss = i8_over_waves<16>(i8_wave_sum(ss), red_sum, true);
        factor = 1.0 / sqrt(ss / a.cols + (double)a.eps);
    }
    auto values = [&](int j, double (&y)[8]) {
        float v[8], u[8];
        i8_load8<T>(x + j, a.cols - j, v);
        if constexpr (OP == EBRL_I8_SWIGLU)
            i8_load8<T>((const T*)a.up + (size_t)row * a.ldup + j, a.cols - j, u);
        if constexpr (OP == EBRL_I8_RMSNORM)
            if (a.gain) i8_load8<float>(a.gain + j, a.cols - j, u);
#pragma unroll
        for (int e = 0; e < 8; ++e) {
            if constexpr (OP == EBRL_I8_SWIGLU) y[e] = i8_gate(v[e], u[e]);
            else if constexpr (OP == EBRL_I8_RMSNORM) {
                y[e] = v[e] * factor;
                if (a.gain) y[e] *= (double)u[e];
            } else y[e] = v[e];
        }
    };
    double top = 0.0, nan = 0.0;
    for (int j = tid * 8; j < a.cols; j += 8192) {
        double y[8];
        values(j, y);
#pragma unroll
        for (int e = 0; e < 8; ++e) {
            top = fmax(top, fabs(y[e]));
            nan = fma(y[e], 0.0, nan);
        }
    }
    const float s = i8_over_waves<16>(wave_max(i8_scale(top, !(nan == 0.0))), red_max, false);
    const bool bad = s == INFINITY;
    const double sd = s, inv = 1.0 / sd;
    if (tid == 0) a.scales[row] = bad ? __builtin_nanf("") : s;
    int8_t* const out = a.codes + (size_t)row * a.ldc;
    const int wide = (a.cols + 15) / 16 * 16;
    for (int j = tid * 8; j < wide; j += 8192) {
        double y[1][8];
        values(j, y[0]);
        i8_store<1>(out, y, j, 0, wide, inv, bad, [&](int at) {
            if constexpr (OP == EBRL_I8_SWIGLU)
                return i8_code(i8_gate(ld_elem<T>(x + at), ld_elem<T>((const T*)a.up + (size_t)row * a.ldup + at)), sd);
            else return i8_code(i8_value<T, OP>(a, x, at, ss), sd);
        });
    }
}

// -------------------------------------------------------------- product --
// All kernels hold the weights' rows as the first operand of
// v_mfma_i32_16x16x64_i8: a lane (r, g) gives bytes 16 g .. of row r, and gets
// outputs n = 4 g .. of row m = r.  Sums are whole numbers: any order gives the
// same, so tiles and cuts of K are free to follow the size of a call.
//
// K tiles are 128 bytes, a cache line of each row.  The last one may be shorter:
// its loads past K repeat the last 16 bytes of the row, and the first operand's
// fragments past K are zeros.

// The outputs that a lane stores: four neighbours of a row.
template <typename T> struct I8Epi {
    const float *scale_a, *scale_b, *bias;
    const T* residual;
    T* c;
    int64_t ldr, ldc;

    struct Cols { f32x4 s, b; };
    EBRL_DEV Cols cols(int n, int N) const {
        Cols k;
        if (n + 4 <= N) {
            k.s = *reinterpret_cast<const f32x4_any*>(scale_b + n);
            k.b = bias ? *reinterpret_cast<const f32x4_any*>(bias + n) : f32x4{0.f, 0.f, 0.f, 0.f};
            return k;
        }
#pragma unroll
        for (int e = 0; e < 4; ++e) {
            const int at = min(n + e, N - 1);
            k.s[e] = scale_b[at];
            k.b[e] = bias ? bias[at] : 0.f;
        }
        return k;
    }
    EBRL_DEV f32x4 value(i32x4 sum, const Cols& k, float sa) const {
#pragma clang fp contract(off)
        f32x4 v;
#pragma unroll
        for (int e = 0; e < 4; ++e) v[e] = (float)sum[e] * k.s[e] * sa;
        if (bias) {
#pragma unroll
            for (int e = 0; e < 4; ++e) v[e] += k.b[e];
        }
        return v;
    }
    // Four neighbours of the residual, as they lie in memory, and as floats.
    typedef typename std::conditional<sizeof(T) == 4, f32x4, uint2>::type Four;
    static EBRL_DEV Four load4(const T* p) {
        if constexpr (sizeof(T) == 4) {
            return *reinterpret_cast<const f32x4_any*>(p);
        } else {
            const u32x2_any w = *reinterpret_cast<const u32x2_any*>(p);
            return make_uint2(w[0], w[1]);
        }
    }
    EBRL_DEV Four load_residual(int m, int n) const { return load4(residual + (size_t)m * ldr + n); }
    static EBRL_DEV f32x4 floats(f32x4 v) { return v; }
    static EBRL_DEV f32x4 floats(uint2 v) {
        return f32x4{__uint_as_float(v.x << 16), __uint_as_float(v.x & 0xFFFF0000u), __uint_as_float(v.y << 16),
                     __uint_as_float(v.y & 0xFFFF0000u)};
    }
    // Up to four outputs, those that are inside: v but for the residual.
    EBRL_DEV void store_some(int m, int n, int M, int N, f32x4 v) const {
        if (m >= M || n >= N) return;
        if (n + 4 <= N) {
            if (residual) v += floats(load_residual(m, n));
            st4_any<T>(c + (size_t)m * ldc + n, v);
            return;
        }
#pragma unroll
        for (int e = 0; e < 4; ++e)
            if (n + e < N) {
                float x = v[e];
                if (residual) x += ld_elem<T>(residual + (size_t)m * ldr + n + e);
                st_elem<T>(c + (size_t)m * ldc + n + e, x);
            }
    }
    EBRL_DEV void store(int m, int n, int M, int N, i32x4 sum, const Cols& k, float sa) const {
        store_some(m, n, M, N, value(sum, k, sa));
    }
    // What four outputs need beside their sums, asked for before these are there, and
    // their store.
    struct Ahead { Cols k; float sa; Four r; };
    EBRL_DEV Ahead ahead(int m, int n, int M, int N) const {
        Ahead x{};
        if (m < M && n < N) {
            x.k = cols(n, N);
            x.sa = scale_a[m];
            if (residual && n + 4 <= N) {
                x.r = load_residual(m, n);
            } else if (residual) {
                const T* p = residual + (size_t)m * ldr + n;
                T some[4];
#pragma unroll
                for (int e = 0; e < 4; ++e) some[e] = n + e < N ? p[e] : T{};
                x.r = __builtin_bit_cast(Four, some);
            }
        }
        return x;
    }
    EBRL_DEV void store(int m, int n, int M, int N, i32x4 sum, const Ahead& x) const {
        if (m >= M || n >= N) return;
        f32x4 v = value(sum, x.k, x.sa);
        if (residual) v += floats(x.r);
        T* p = c + (size_t)m * ldc + n;
        if (n + 4 <= N) {
            st4_any<T>(p, v);
            return;
        }
#pragma unroll
        for (int e = 0; e < 3; ++e)
            if (n + e < N) st_elem<T>(p + e, v[e]);
    }
};

EBRL_DEV i32x4 i8_fragment(const char* lds) { return *reinterpret_cast<const i32x4*>(lds); }

// 256 x 256 tiles, eight waves of 128 x 64 in two groups of four that run half a
// phase apart, as in the large bf16 kernel: while one group multiplies from
// registers, the other reads its next fragments from LDS and issues DMA.  A K tile
// is two phases: all of a wave's columns with its first 64 rows, then its last 64.
// Two LDS stages of 64 KB, refilled by half operands as soon as both groups have
// read them.  Workgroups are persistent; the next tile's first DMAs go out before
// the epilogue, whose stores drain behind them.  `full` tiles are dealt evenly, those
// of the last round cut in `split`.
//  * What bounds it: power.  8192 x 8192 x 8192 takes 362 us, 3.04 POPS (the library's
//    product of that size 511 to 540, 2.04 to 2.15); 9216 x 12288 x 4096 330 with two sets of
//    operands in turn (411 to 431), 345 with three, which no cache holds.  There the matrix
//    units are busy 73 % of the cycles, at a clock that the card holds at 1.75 GHz; a K tile
//    takes 1.3 us with one on every CU, of which 1.1 are products.
//  * The epilogue loads nothing that the compiler waits for, since its waits count the
//    DMAs too, which it does not see: scales and bias come through LDS, the residual is
//    asked for three row groups ahead, the next tile's DMAs go out behind its last
//    loads (9216 x 12288 x 4096 380 -> 361 us, 5476 x 8192 x 1024 62 -> 53).  Scaled
//    results are staged, bf16 ones as such: half the LDS traffic, 16 bytes a store.
//    Tiles at the edges do the same with what is there, four columns at a time (9216 x
//    4095 x 4096, fp32 with a residual, 179 us; 224 by elements, one load after the other;
//    4096 columns 176).
//  * What a tile derives from the lane is made anew each time: kept in registers it was
//    spilled, and each reload waited for every DMA (35 spilled registers, 374 us at 8192^3;
//    none in the K loop, 364).  The multiplying group goes first (s_setprio: 5476 x 8192 x
//    1024 51 -> 48, nothing at long K).
//  * With a residual the tiles of a round meet in memory at the end: 9216 x 4096 x 11008,
//    fp32, 348 us, of which 302 MB of residual and results are 63.  Half the XCDs
//    taking their part of the last round first, so that the rounds do not end together:
//    425 us (the code of the parts twice in the loop, and spills); starts 1 to 20 us
//    apart: no change.
template <typename T, bool RES, bool STREAM>
__global__ __launch_bounds__(512, 2) void i8_big_kernel(const int8_t* __restrict__ A, uint32_t lda,
                                                        const int8_t* __restrict__ B, uint32_t ldb, int M, int N, int K,
                                                        int full, int split, I8Epi<T> epi)
{
    constexpr int STAGES = 2 * 65536;   // operand stages; 4 KB of epilogue staging per wave follow
    __shared__ __attribute__((aligned(1024))) char smem[STAGES + 8 * 4096];
    const int tid = threadIdx.x, lane = tid & 63;
    const int wave = __builtin_amdgcn_readfirstlane(tid >> 6);
    const int wr = wave >> 2, wc = wave & 3;   // group (row half of the tile) and column quarter
    const int r = lane & 15, g = lane >> 4;
    const int tiles_m = (M + 255) >> 8, tiles_n = (N + 255) >> 8;
    const int nk = (K + 127) >> 7, rest = K - (nk - 1) * 128;
    const uint32_t lds0 = __builtin_amdgcn_readfirstlane((uint32_t)(uintptr_t)(lds_ptr_t)smem);
    // The lane, made anew: what is derived from it once a tile would otherwise be kept in
    // registers through the K loop, that is, spilled, and its way back waits for every
    // load in flight.
    auto fresh_lane = [&]() {
        int l = 0;
        asm volatile("" : "+v"(l));
        return (int)__builtin_amdgcn_mbcnt_hi(~0u, __builtin_amdgcn_mbcnt_lo(~0u, (uint32_t)l));
    };
    // How far past the end of the last K tile, if it is a short one, this lane's bytes are.
    auto past = [&]() {
        const int l = fresh_lane();
        return (uint32_t)max(0, ((l & 7) ^ (l >> 3)) * 16 - (rest - 16));
    };

    auto run = [&](auto FAC, auto FBC, int m0, int n0, auto next) {
        constexpr int FA = decltype(FAC)::value, FB = decltype(FBC)::value;
        constexpr int HA = 16 * FA, HB = 16 * FB;        // a wave's rows / columns per half
        constexpr int NA = FA / 2, NB = FB;              // DMA instructions per wave and half
        constexpr int AHALF = 2 * HA * 128, BHALF = 4 * HB * 128, SB = 2 * (AHALF + BHALF);
        constexpr int W = 2 * NA + 2 * NB;               // DMA instructions per wave and K tile
        static_assert(2 * SB <= STAGES, "stages");
        // The epilogue's 16-row groups, the group before which the next tile's first
        // loads go out (RES: when the residual's are all on their way), and the stores
        // of an interior tile behind those, which may still be in flight with them.
        constexpr int GROUPS = 2 * FA, AT = RES ? GROUPS - 3 : 0;
        constexpr int HALF = sizeof(T) == 2 && !RES;     // staged as results, not as floats
        constexpr int PASSES = FB * (HALF ? 1 : 2);
        constexpr int EST = (GROUPS - AT) * PASSES;
        // scales that are loaded behind them, without the bias
        constexpr int RV = FA / 2, SCL = RV + 1;
        static_assert(W + EST + SCL < 64, "vmcnt range");
        uint32_t va[2][NA], vb[2][NB];
        const char *pA, *pB;
        auto dmaA = [&](int t, int h) {
            const char* p = pA + (size_t)t * 128;
            const uint32_t l = lds0 + (t & 1) * SB + h * AHALF + wave * NA * 1024;
            if (rest < 128 && t == nk - 1) {
                const uint32_t back = past();
#pragma unroll
                for (int j = 0; j < NA; ++j) dma16_to_lds_s(p, va[h][j] - back, l + j * 1024);
            } else {
#pragma unroll
                for (int j = 0; j < NA; ++j) dma16_to_lds_s(p, va[h][j], l + j * 1024);
            }
        };
        auto dmaB = [&](int t, int h) {
            const char* p = pB + (size_t)t * 128;
            const uint32_t l = lds0 + (t & 1) * SB + 2 * AHALF + h * BHALF + wave * NB * 1024;
            if (rest < 128 && t == nk - 1) {
                const uint32_t back = past();
#pragma unroll
                for (int j = 0; j < NB; ++j) dma16_to_lds_s(p, vb[h][j] - back, l + j * 1024);
            } else {
#pragma unroll
                for (int j = 0; j < NB; ++j) dma16_to_lds_s(p, vb[h][j], l + j * 1024);
            }
        };
        // K tiles 0 and 1 but for the second half of A's tile 1; rows past the
        // operand repeat its last one.  LDS row q of a half h holds tile row
        // (q / HA) 2 HA + h HA + q % HA: each wave's rows are contiguous.
        auto prologue = [&]() {
            const int lane = fresh_lane();
            const uint32_t kb = ((lane & 7) ^ (lane >> 3)) * 16;
#pragma unroll
            for (int h = 0; h < 2; ++h) {
#pragma unroll
                for (int j = 0; j < NA; ++j) {
                    const int q = (wave * NA + j) * 8 + (lane >> 3);
                    const int row = (q / HA) * 2 * HA + h * HA + q % HA;
                    va[h][j] = (uint32_t)min(row, M - 1 - m0) * lda + kb;
                }
#pragma unroll
                for (int j = 0; j < NB; ++j) {
                    const int q = (wave * NB + j) * 8 + (lane >> 3);
                    const int row = (q / HB) * 2 * HB + h * HB + q % HB;
                    vb[h][j] = (uint32_t)min(row, N - 1 - n0) * ldb + kb;
                }
            }
            pA = uniform_ptr(A + (size_t)m0 * lda);
            pB = uniform_ptr(B + (size_t)n0 * ldb);
            dmaB(0, 0); dmaA(0, 0); dmaB(0, 1); dmaA(0, 1);
            if (nk > 1) { dmaB(1, 0); dmaA(1, 0); dmaB(1, 1); }
        };
        uint32_t a_off[2], b_off[2];
#pragma unroll
        for (int ks = 0; ks < 2; ++ks) {
            a_off[ks] = (uint32_t)((wr * HA + r) * 128 + (((ks * 4 + g) ^ (r & 7)) << 4));
            b_off[ks] = (uint32_t)(2 * AHALF + (wc * HB + r) * 128 + (((ks * 4 + g) ^ (r & 7)) << 4));
        }
        i32x4 acc[2][2][FA][FB];
        i32x4 fa[2][FA], fb0[2][FB], fb1[2][FB];
        auto readA = [&](int st, int h) {
#pragma unroll
            for (int ks = 0; ks < 2; ++ks)
#pragma unroll
                for (int i = 0; i < FA; ++i) fa[ks][i] = i8_fragment(smem + st + a_off[ks] + h * AHALF + i * 2048);
        };
        auto readB = [&](int st, int h, i32x4 (&f)[2][FB]) {
#pragma unroll
            for (int ks = 0; ks < 2; ++ks)
#pragma unroll
                for (int j = 0; j < FB; ++j) f[ks][j] = i8_fragment(smem + st + b_off[ks] + h * BHALF + j * 2048);
        };
        // fragments past K to zero
        auto cut = [&](i32x4 (&f)[2][FB]) {
#pragma unroll
            for (int ks = 0; ks < 2; ++ks)
                if (ks * 64 + g * 16 >= rest) {
#pragma unroll
                    for (int j = 0; j < FB; ++j) f[ks][j] = i32x4{0, 0, 0, 0};
                }
        };
        auto mma = [&](i32x4 (&c)[FA][FB], const i32x4 (&f)[2][FB]) {
#pragma unroll
            for (int ks = 0; ks < 2; ++ks)
#pragma unroll
                for (int i = 0; i < FA; ++i)
#pragma unroll
                    for (int j = 0; j < FB; ++j)
                        c[i][j] = __builtin_amdgcn_mfma_i32_16x16x64_i8(f[ks][j], fa[ks][i], c[i][j], 0, 0, 0);
        };
        // Phase p of a group: read fragments, issue DMA, wait for the DMA that
        // phase p + 1 reads, barrier, multiply, barrier.  A group's reads are
        // complete before its first barrier, so what phase p reads may be refilled
        // from phase p + 1 on, by either group.  One K tile with L further ones (0,
        // 1, 2 = two or more); first, ov: the scales', and the previous output tile's
        // stores, sit between this tile's DMAs.
        auto wait = [&](bool first, bool ov) {
            if (!first) wait_vmcnt<W>();
            else if (ov) wait_vmcnt<W + EST + SCL>();
            else wait_vmcnt<W + SCL>();
        };
        auto ktile = [&](int t, bool first, bool ov, auto LC) {
            constexpr int L = decltype(LC)::value;
            const int st = (t & 1) * SB;
            readB(st, 0, fb0); readA(st, 0); readB(st, 1, fb1);
            if constexpr (L >= 1) dmaA(t + 1, 1);
            if constexpr (L >= 2) wait(first, ov);
            else if constexpr (L == 1) wait_vmcnt<W>();
            else wait_vmcnt<0>();
            wait_lds();
            wg_barrier();
            if constexpr (L == 0) { cut(fb0); cut(fb1); }
            __builtin_amdgcn_s_setprio(1);
            mma(acc[0][0], fb0); mma(acc[0][1], fb1);
            __builtin_amdgcn_s_setprio(0);
            wg_barrier();
            readA(st, 1);
            if constexpr (L >= 2) {
                dmaB(t + 2, 0); dmaA(t + 2, 0); dmaB(t + 2, 1);
                wait(first, ov);
            } else if constexpr (L == 1) wait_vmcnt<NA>();
            wait_lds();
            wg_barrier();
            __builtin_amdgcn_s_setprio(1);
            mma(acc[1][0], fb0); mma(acc[1][1], fb1);
            __builtin_amdgcn_s_setprio(0);
            wg_barrier();
        };
        prologue();
        bool over = false;   // an interior tile's stores were issued behind the prologue
        for (;;) {
#pragma unroll
            for (int a = 0; a < 2; ++a)
#pragma unroll
                for (int b = 0; b < 2; ++b)
#pragma unroll
                    for (int i = 0; i < FA; ++i)
#pragma unroll
                        for (int j = 0; j < FB; ++j) acc[a][b][i][j] = i32x4{0, 0, 0, 0};
            // The scales of the wave's rows and columns, and the bias, into its staging
            // LDS: loads of the compiler's would wait for the DMAs that it does not see.
            const int mw = m0 + wr * 2 * HA, nw = n0 + wc * 2 * HB;
            const uint32_t stage0 = lds0 + STAGES + wave * 4096;
            char* const stage = smem + STAGES + wave * 4096;
            const int early = fresh_lane();
#pragma unroll
            for (int v = 0; v < RV; ++v) dma4_to_lds(epi.scale_a + min(mw + v * 64 + early, M - 1), stage0 + v * 256);
            const int at_col = min(nw + early % (2 * HB), N - 1);
            dma4_to_lds(epi.scale_b + at_col, stage0 + 512);
            if (epi.bias) dma4_to_lds(epi.bias + at_col, stage0 + 768);
            // first B halves and first A half of K tile 0
            if (nk > 1) wait(true, over);
            else wait_vmcnt<0>();
            wg_barrier();
            if (wr == 1) wg_barrier();   // the second group runs half a phase behind
            int t = 0;
            for (; t + 2 < nk; ++t) ktile(t, t == 0, over, std::integral_constant<int, 2>{});
            if (t + 1 < nk) { ktile(t, false, false, std::integral_constant<int, 1>{}); ++t; }
            ktile(t, false, false, std::integral_constant<int, 0>{});
            if (wr == 0) wg_barrier();   // both groups are done with the stages
            const bool inside = m0 + 4 * HA <= M && n0 + 8 * HB <= N;
            const int lane = fresh_lane(), r = lane & 15, g = lane >> 4;
            float sa[GROUPS];
            f32x4 sb[2 * FB], bias[2 * FB];
#pragma unroll
            for (int k = 0; k < GROUPS; ++k) sa[k] = *reinterpret_cast<const float*>(stage + (k * 16 + r) * 4);
#pragma unroll
            for (int j = 0; j < 2 * FB; ++j) {
                sb[j] = *reinterpret_cast<const f32x4*>(stage + 512 + (j * 16 + 4 * g) * 4);
                if (epi.bias) bias[j] = *reinterpret_cast<const f32x4*>(stage + 768 + (j * 16 + 4 * g) * 4);
            }
            wait_lds();
            const bool more = next(m0, n0);
            // Sixteen rows at a time, scaled, through the staging LDS, so that stores are
            // of whole row segments; 16-byte chunks swizzled by row, which spreads the
            // writes (a lane a row) and the reads (several a row) over all banks.
            auto value = [&](int k, int j) {
#pragma clang fp contract(off)
                const i32x4 sum = acc[k / FA][j / FB][k % FA][j % FB];
                f32x4 v;
#pragma unroll
                for (int e = 0; e < 4; ++e) v[e] = (float)sum[e] * sb[j][e] * sa[k];
                if (epi.bias) v += bias[j];
                return v;
            };
            auto swz = [](int row) { return ((row & 1) << 2) | ((row >> 1) & 3) | (row & 8); };
            auto put = [&](int k) {
#pragma unroll
                for (int j = 0; j < 2 * FB; ++j)
                    *reinterpret_cast<f32x4*>(stage + r * 256 + (((j * 4 + g) ^ swz(r)) << 4)) = value(k, j);
            };
            auto get = [&](int row, int ch) {
                return *reinterpret_cast<const f32x4*>(stage + row * 256 + ((ch ^ swz(row)) << 4));
            };
            constexpr int LPR = 2 * HB / 4, RPP = 64 / LPR;   // lanes a row of floats, rows a pass
            const int lr = lane / LPR, lc = lane % LPR;
            // Edges: rows and columns that are there; a lane whose four columns end past
            // the last one takes the last four (those that its neighbour has too are the
            // same, and loaded before either stores).
            auto rows = [&](auto EDGE) {
                constexpr bool edge = decltype(EDGE)::value;
                constexpr int DEPTH = edge ? 1 : 3;              // row groups of the residual in flight
                typename I8Epi<T>::Four ahead[4][16 / RPP];
                const int col = edge ? min(lc * 4, N - 4 - nw) : lc * 4;
                const int there = !edge ? 16 * GROUPS : nw + lc * 4 < N ? M - mw - lr : 0;
                T* to = epi.c + (size_t)(mw + lr) * epi.ldc + nw + col;
                const T* from = RES ? epi.residual + (size_t)(mw + lr) * epi.ldr + nw + col : nullptr;
                const int64_t step = RPP * epi.ldc, step_r = RPP * epi.ldr;
                auto fetch = [&](int k) {
#pragma unroll
                    for (int p = 0; p < 16 / RPP; ++p) {
                        if (!edge || k * 16 + p * RPP < there)
                            ahead[k & 3][p] = I8Epi<T>::load4(from);
                        from += step_r;
                        asm volatile("" : "+v"(from));   // the next rows' addresses are not kept
                    }
                };
                if constexpr (RES) {
#pragma unroll
                    for (int k = 0; k < DEPTH && k < GROUPS; ++k) fetch(k);
                }
#pragma unroll
                for (int k = 0; k < GROUPS; ++k) {
                    if (k == (RES ? GROUPS - DEPTH : 0) && more) prologue();
                    put(k);
                    if constexpr (RES) { if (k + DEPTH < GROUPS) fetch(k + DEPTH); }
#pragma unroll
                    for (int p = 0; p < 16 / RPP; ++p) {
                        const int row = p * RPP + lr;
                        f32x4 v;
                        if constexpr (edge) {
                            int at = col;
                            asm volatile("" : "+v"(at));         // nor those in LDS
#pragma unroll
                            for (int e = 0; e < 4; ++e, ++at)
                                v[e] = *reinterpret_cast<const float*>(stage + row * 256 + (((at >> 2) ^ swz(row)) << 4) +
                                                                       (at & 3) * 4);
                        } else {
                            v = get(row, lc);
                        }
                        if (!edge || k * 16 + p * RPP < there) {
                            if constexpr (RES) v += I8Epi<T>::floats(ahead[k & 3][p]);
                            if constexpr (STREAM && sizeof(T) == 4 && !edge)
                                __builtin_nontemporal_store(v, reinterpret_cast<f32x4_any*>(to));
                            else
                                st4_any<T>(to, v);
                        }
                        to += step;
                        asm volatile("" : "+v"(to));
                    }
                }
            };
            if (inside && HALF) {
                // results of 2 bytes: eight neighbours a lane
                constexpr int L8 = 2 * HB / 8, R8 = 64 / L8;
                T* to = epi.c + (size_t)(mw + lane / L8) * epi.ldc + nw + lane % L8 * 8;
                const int64_t step = R8 * epi.ldc;
                if (more) prologue();
#pragma unroll
                for (int k = 0; k < GROUPS; ++k) {
#pragma unroll
                    for (int j = 0; j < 2 * FB; ++j) {
                        const f32x4 v = value(k, j);
                        st4<bf16_t>(reinterpret_cast<bf16_t*>(stage + r * 128 + (((j * 2 + (g >> 1)) ^ (r & 7)) << 4) + (g & 1) * 8),
                                    v[0], v[1], v[2], v[3]);
                    }
#pragma unroll
                    for (int p = 0; p < 16 / R8; ++p) {
                        const int row = p * R8 + lane / L8;
                        const u32x4 v = *reinterpret_cast<const u32x4*>(stage + row * 128 + (((lane % L8) ^ (row & 7)) << 4));
                        if constexpr (STREAM) __builtin_nontemporal_store(v, reinterpret_cast<u32x4_any*>(to));
                        else *reinterpret_cast<u32x4_any*>(to) = v;
                        to += step;
                        asm volatile("" : "+v"(to));     // the next rows' addresses are not kept
                    }
                }
            } else if (inside) {
                rows(std::integral_constant<bool, false>{});
            } else if (N - nw >= 4) {
                rows(std::integral_constant<bool, true>{});
            } else {
                if (more) prologue();
#pragma unroll
                for (int k = 0; k < GROUPS; ++k) {
                    put(k);
#pragma unroll 1
                    for (int p = 0; p < 16 / RPP; ++p) {
                        const int row = p * RPP + lr;
                        epi.store_some(mw + k * 16 + row, nw + lc * 4, M, N, get(row, lc));
                    }
                }
            }
            if (!more) break;
            over = inside;
        }
    };

    using I1 = std::integral_constant<int, 1>;
    using I2 = std::integral_constant<int, 2>;
    using I4 = std::integral_constant<int, 4>;
    // The dispatcher deals workgroup ids round-robin over the 8 XCDs: XCD x's
    // workgroups walk a contiguous range of tiles together and share its L2.
    const int P = gridDim.x, bid = blockIdx.x;
    if (full > 0) {
        const int rounds = full / P;
        int i = 0;
        auto origin = [&](int k, int& m, int& n) {
            const int v = (P & 7) == 0 ? (bid & 7) * (full >> 3) + k * (P >> 3) + (bid >> 3) : k * P + bid;
            tile_origin(v, tiles_m, tiles_n, 256, 256, m, n);
        };
        int m0, n0;
        origin(0, m0, n0);
        run(I4{}, I2{}, m0, n0, [&](int& m, int& n) {
            if (++i >= rounds) return false;
            origin(i, m, n);
            return true;
        });
    }
    // The last round: at most one (part of a) tile per workgroup.
    const int items = (tiles_m * tiles_n - full) * split;
    if (bid >= items) return;
    const int x = bid & 7;
    const int s = x * (items >> 3) + min(x, items & 7) + (bid >> 3);
    int m0, n0;
    tile_origin(full + s / split, tiles_m, tiles_n, 256, 256, m0, n0);
    auto none = [](int&, int&) { return false; };
    const int part = s % split;
    m0 += (part & 1) * 128;
    n0 += (part >> 1) * 128;
    if (m0 >= M || n0 >= N) return;
    if (split == 1) run(I4{}, I2{}, m0, n0, none);
    else if (split == 2) run(I2{}, I2{}, m0, n0, none);
    else run(I2{}, I1{}, m0, n0, none);
}

// Small outputs (fewer 256 x 256 tiles than CUs): BM x BN tiles on four waves
// (2 x 2), a ring of ST K tiles in LDS with ST - 1 of them in flight, one barrier a
// K tile; scales and residual ahead of the first operands.  Bound by what a CU draws
// into LDS, by the times of the sizes 70 to 90 GB/s (at 591 x 1003 x 1296 the matrix units
// are busy 4 % of the cycles, the vector units 9, LDS reads 7): a K tile takes 0.2 (32 x 64),
// 0.3 (64 x 64) and 0.42 us (64 x 128) with one workgroup on a CU, 0.3, 0.39 and 0.7 with
// two.  800 x 1024 x 4096 12.9 us, 591 x 1003 x 1296 8.0.
template <typename T, int BM, int BN, int ST>
__global__ __launch_bounds__(256, 2) void i8_ring_kernel(const int8_t* __restrict__ A, uint32_t lda,
                                                         const int8_t* __restrict__ B, uint32_t ldb, int M, int N, int K,
                                                         I8Epi<T> epi)
{
    constexpr int WTM = BM / 2, WTN = BN / 2, TM = WTM / 16, TN = WTN / 16;
    constexpr int SB = (BM + BN) * 128;                // bytes of a stage
    constexpr int PER = (BM + BN) / 32;                // DMA instructions per wave and K tile
    static_assert((BM + BN) % 32 == 0 && BM % 8 == 0 && ST >= 2 && ST <= 4, "ring");
    __shared__ __attribute__((aligned(1024))) char smem[ST * SB];
    const int tiles_m = (M + BM - 1) / BM, tiles_n = (N + BN - 1) / BN;
    int bid = blockIdx.x;
    {
        // XCD x takes the x-th contiguous range of tiles
        const int nb = gridDim.x, x = bid & 7;
        bid = x * (nb >> 3) + min(x, nb & 7) + (bid >> 3);
    }
    int m0, n0;
    tile_origin(bid, tiles_m, tiles_n, BM, BN, m0, n0);
    const int nk = (K + 127) >> 7, rest = K - (nk - 1) * 128;
    const int tid = threadIdx.x, lane = tid & 63;
    const int wave = __builtin_amdgcn_readfirstlane(tid >> 6);
    const int wm = wave >> 1, wn = wave & 1;
    const int r = lane & 15, g = lane >> 4;
    const uint32_t kb = ((lane & 7) ^ (lane >> 3)) * 16;
    const uint32_t past = (uint32_t)max(0, (int)kb - (rest - 16));

    // 8-row groups of a stage, A's first: PER per wave
    uint32_t vo[PER];
    const char* base[PER];
    const uint32_t lds0 = __builtin_amdgcn_readfirstlane((uint32_t)(uintptr_t)(lds_ptr_t)smem + wave * PER * 1024);
    const char* const pA = uniform_ptr(A + (size_t)m0 * lda);
    const char* const pB = uniform_ptr(B + (size_t)n0 * ldb);
#pragma unroll
    for (int j = 0; j < PER; ++j) {
        const int q0 = (wave * PER + j) * 8, q = q0 + (lane >> 3);
        vo[j] = (q0 < BM ? (uint32_t)min(q, M - 1 - m0) * lda : (uint32_t)min(q - BM, N - 1 - n0) * ldb) + kb;
        base[j] = q0 < BM ? pA : pB;
    }
    auto dma = [&](int t, int st) {
        const uint32_t back = t == nk - 1 ? past : 0u;
#pragma unroll
        for (int j = 0; j < PER; ++j) dma16_to_lds_s(base[j] + (size_t)t * 128, vo[j] - back, lds0 + st * SB + j * 1024);
    };
    uint32_t a_off[2], b_off[2];
#pragma unroll
    for (int ks = 0; ks < 2; ++ks) {
        a_off[ks] = (uint32_t)((wm * WTM + r) * 128 + (((ks * 4 + g) ^ (r & 7)) << 4));
        b_off[ks] = (uint32_t)((BM + wn * WTN + r) * 128 + (((ks * 4 + g) ^ (r & 7)) << 4));
    }
    i32x4 acc[TM][TN];
#pragma unroll
    for (int i = 0; i < TM; ++i)
#pragma unroll
        for (int j = 0; j < TN; ++j) acc[i][j] = i32x4{0, 0, 0, 0};
    // the epilogue's scales and residual, ahead of the operands
    constexpr int SROW = WTN + 4, LPR = WTN / 4, RPP = 64 / LPR, PASSES = 16 / RPP;
    static_assert(4 * 16 * SROW * 4 <= ST * SB, "staging space");
    const int col = n0 + wn * WTN + lane % LPR * 4;
    typename I8Epi<T>::Ahead ahead[TM][PASSES];
#pragma unroll
    for (int i = 0; i < TM; ++i)
#pragma unroll
        for (int p = 0; p < PASSES; ++p)
            ahead[i][p] = epi.ahead(m0 + wm * WTM + i * 16 + p * RPP + lane / LPR, col, M, N);
    for (int p = 0; p < ST - 1 && p < nk; ++p) dma(p, p);
    int st = 0, nst = ST - 1;
    for (int t = 0; t < nk; ++t) {
        // this wave's part of tile t has landed (the tiles issued after it may
        // stay in flight); after the barrier every wave's has, and all have
        // read tile t - 1, whose stage is refilled next
        const int later = min(ST - 2, nk - 1 - t);
        if (ST >= 4 && later >= 2) wait_vmcnt<2 * PER>();
        else if (ST >= 3 && later >= 1) wait_vmcnt<PER>();
        else wait_vmcnt<0>();
        wg_barrier();
        if (t + ST - 1 < nk) dma(t + ST - 1, nst);
        const char* const s = smem + st * SB;
        i32x4 w[2][TN], x[2][TM];
#pragma unroll
        for (int ks = 0; ks < 2; ++ks) {
#pragma unroll
            for (int j = 0; j < TN; ++j) w[ks][j] = i8_fragment(s + b_off[ks] + j * 2048);
#pragma unroll
            for (int i = 0; i < TM; ++i) x[ks][i] = i8_fragment(s + a_off[ks] + i * 2048);
        }
        if (t == nk - 1) {
#pragma unroll
            for (int ks = 0; ks < 2; ++ks)
                if (ks * 64 + g * 16 >= rest) {
#pragma unroll
                    for (int j = 0; j < TN; ++j) w[ks][j] = i32x4{0, 0, 0, 0};
                }
        }
#pragma unroll
        for (int ks = 0; ks < 2; ++ks)
#pragma unroll
            for (int i = 0; i < TM; ++i)
#pragma unroll
                for (int j = 0; j < TN; ++j)
                    acc[i][j] = __builtin_amdgcn_mfma_i32_16x16x64_i8(w[ks][j], x[ks][i], acc[i][j], 0, 0, 0);
        nst = st;
        st = st + 1 == ST ? 0 : st + 1;
    }
    wg_barrier();
    // epilogue staging in the stages: rows padded by one chunk
    int* const stage = reinterpret_cast<int*>(smem) + wave * 16 * SROW;
#pragma unroll
    for (int i = 0; i < TM; ++i) {
#pragma unroll
        for (int j = 0; j < TN; ++j) *reinterpret_cast<i32x4*>(stage + r * SROW + j * 16 + 4 * g) = acc[i][j];
#pragma unroll
        for (int p = 0; p < PASSES; ++p) {
            const int row = p * RPP + lane / LPR;
            const i32x4 sum = *reinterpret_cast<const i32x4*>(stage + row * SROW + lane % LPR * 4);
            epi.store(m0 + wm * WTM + i * 16 + row, col, M, N, sum, ahead[i][p]);
        }
    }
}

// Few rows, or few outputs of a long sum: the weights are streamed once.  A workgroup has a slice of BN columns, at
// most 16 TM rows and a range of K; its waves split that range and run pipelines of
// their own: each DMAs its weights' and activations' rows into LDS of its own, one
// instruction 8 rows x 128 bytes, STAGES - 1 K tiles ahead, and multiplies from
// there.  XR rows of activations are loaded, 8 of them for up to 8 rows (the upper
// half of the fragment then repeats the lower one and is not stored).  The waves'
// tiles are summed through LDS.  With several ranges of K (splits) the sums go to the
// workspace and i8_join_kernel adds them up.  NT: each weight is read by one workgroup.
//
// Bound by memory where the slices fill the chip in one round (1 x 12288 x 4096 10.2 us,
// 4.9 TB/s with launch and tail; 8 x 4096 x 11008 10.4, 8.9 in a row of them, 5.1), by what a CU
// draws into LDS, by the times 57 to 70 GB/s, where activations are half of it and more (64 x
// 12288 x 4096 14 to 15; at 37 x 22016 x 4096 the matrix units are busy 9 % of the cycles, the
// vector units 12, LDS reads 6).
// Slices of 16, 48 or 96 columns are those that make one round of 256 workgroups of 4096,
// 12288 and 22016 outputs: 37 x 22016 x 4096 19.8 us with 96, 22.2 with 48, 25 with 64; 17 x
// 4096 x 4096 6.2 with 16, 7.8 with 32.  Eight waves instead of four: never faster (1 x
// 12288 x 4096 13.0, 10.9 and 11.3 us with slices of 16, 48 and 64 against 9.8, 9.9 and 10.2).
template <typename T, int XR, int BN, int STAGES, bool NT>
__global__ __launch_bounds__(256) void i8_decode_kernel(const int8_t* __restrict__ A, uint32_t lda,
                                                               const int8_t* __restrict__ B, uint32_t ldb, int M, int N,
                                                               int K, int tiles_per_split, int splits, int m_tiles,
                                                               int* __restrict__ ws, I8Epi<T> epi)
{
    constexpr int WAVES = 4;
    constexpr int TM = XR < 16 ? 1 : XR / 16, TN = BN / 16, FR = TM * TN;
    constexpr int WI = BN / 8, XI = XR / 8;                  // DMA instructions per K tile
    constexpr int STAGE = (BN + XR) * 128;                   // bytes per wave and K tile
    constexpr int RB = FR * 1024;                            // bytes of a wave's sums
    constexpr int LDS = WAVES * (STAGES * STAGE > RB ? STAGES * STAGE : RB);
    static_assert(LDS <= 160 * 1024 && STAGES >= 2, "LDS");
    __shared__ __attribute__((aligned(1024))) char smem[LDS];
    const int tid = threadIdx.x, lane = tid & 63;
    const int wave = __builtin_amdgcn_readfirstlane(tid >> 6);
    const int r = lane & 15, g = lane >> 4;
    // XCD x takes the x-th contiguous range of units, so that the row tiles of one
    // slice, which read the same weights, run on one XCD
    int bid = blockIdx.x;
    {
        const int nb = gridDim.x, x = bid & 7;
        bid = x * (nb >> 3) + min(x, nb & 7) + (bid >> 3);
    }
    const int mt = bid % m_tiles, unit = bid / m_tiles;
    const int split = unit % splits, nt = unit / splits;
    const int m0 = mt * 16 * TM, n0 = nt * BN;
    const int nk = (K + 127) >> 7, rest = K - (nk - 1) * 128;
    const int s_begin = split * tiles_per_split, s_end = min(nk, s_begin + tiles_per_split);
    const int per_wave = (s_end - s_begin + WAVES - 1) / WAVES;
    const int w_begin = min(s_end, s_begin + wave * per_wave), w_end = min(s_end, w_begin + per_wave);
    const uint32_t kb = ((lane & 7) ^ (lane >> 3)) * 16;
    const uint32_t past = (uint32_t)max(0, (int)kb - (rest - 16));

    uint32_t vw[WI], vx[XI];
#pragma unroll
    for (int j = 0; j < WI; ++j) vw[j] = (uint32_t)min(j * 8 + (lane >> 3), N - 1 - n0) * ldb + kb;
#pragma unroll
    for (int j = 0; j < XI; ++j) vx[j] = (uint32_t)min(j * 8 + (lane >> 3), M - 1 - m0) * lda + kb;
    const char* const pB = uniform_ptr(B + (size_t)n0 * ldb);
    const char* const pA = uniform_ptr(A + (size_t)m0 * lda);
    const uint32_t lds0 =
        __builtin_amdgcn_readfirstlane((uint32_t)(uintptr_t)(lds_ptr_t)smem + wave * STAGES * STAGE);
    auto dma = [&](int t, int st) {
        const uint32_t back = t == nk - 1 ? past : 0u;
        const uint32_t l = lds0 + st * STAGE;
#pragma unroll
        for (int j = 0; j < WI; ++j) {
            if constexpr (NT) dma16_to_lds_s_nt(pB + (size_t)t * 128, vw[j] - back, l + j * 1024);
            else dma16_to_lds_s(pB + (size_t)t * 128, vw[j] - back, l + j * 1024);
        }
#pragma unroll
        for (int j = 0; j < XI; ++j) dma16_to_lds_s(pA + (size_t)t * 128, vx[j] - back, l + (WI + j) * 1024);
    };
    uint32_t off[2];
#pragma unroll
    for (int ks = 0; ks < 2; ++ks) off[ks] = (uint32_t)((r & 7) * 128 + (((ks * 4 + g) ^ (r & 7)) << 4));
    const uint32_t upper = (r >> 3) * 1024;                  // second 8-row group of a fragment
    i32x4 acc[TM][TN];
#pragma unroll
    for (int i = 0; i < TM; ++i)
#pragma unroll
        for (int j = 0; j < TN; ++j) acc[i][j] = i32x4{0, 0, 0, 0};
    auto multiply = [&](int t, int st) {
        const char* const s = smem + (wave * STAGES + st) * STAGE;
        i32x4 w[2][TN], x[2][TM];
#pragma unroll
        for (int ks = 0; ks < 2; ++ks) {
#pragma unroll
            for (int j = 0; j < TN; ++j) w[ks][j] = i8_fragment(s + off[ks] + upper + j * 2048);
#pragma unroll
            for (int i = 0; i < TM; ++i)
                x[ks][i] = i8_fragment(s + BN * 128 + off[ks] + (XR < 16 ? 0 : upper) + i * 2048);
        }
        if (t == nk - 1) {
#pragma unroll
            for (int ks = 0; ks < 2; ++ks)
                if (ks * 64 + g * 16 >= rest) {
#pragma unroll
                    for (int j = 0; j < TN; ++j) w[ks][j] = i32x4{0, 0, 0, 0};
                }
        }
#pragma unroll
        for (int ks = 0; ks < 2; ++ks)
#pragma unroll
            for (int i = 0; i < TM; ++i)
#pragma unroll
                for (int j = 0; j < TN; ++j)
                    acc[i][j] = __builtin_amdgcn_mfma_i32_16x16x64_i8(w[ks][j], x[ks][i], acc[i][j], 0, 0, 0);
    };
    // Tile w_begin + i sits in stage i % STAGES; the one STAGES - 1 further on goes
    // into the stage that the tile before it has left (wait_lds: it has been read).
#pragma unroll
    for (int i = 0; i < STAGES - 1; ++i)
        if (w_begin + i < w_end) dma(w_begin + i, i);
    for (int t = w_begin; t < w_end; t += STAGES) {
#pragma unroll
        for (int i = 0; i < STAGES; ++i) {
            if (t + i >= w_end) break;
            wait_lds();
            if (t + i + STAGES - 1 < w_end) dma(t + i + STAGES - 1, (i + STAGES - 1) % STAGES);
            wait_tiles<STAGES - 1, WI + XI>(w_end - 1 - t - i);
            multiply(t + i, i);
        }
    }
    // The outputs that this thread stores, four each, and what they need beside the
    // sums, asked for while these are exchanged.
    constexpr int UNITS = FR * 64, PER = (UNITS + 255) / 256;
    typename I8Epi<T>::Ahead ahead[PER];
    auto place = [&](int q, int& m, int& n) {
        const int f = q >> 6, l = q & 63;
        m = m0 + f / TN * 16 + (l & 15);
        n = n0 + f % TN * 16 + 4 * (l >> 4);
        return q < UNITS && m < M && n < N && (XR >= 16 || (l & 15) < XR);
    };
    if (splits == 1) {
#pragma unroll
        for (int u = 0; u < PER; ++u) {
            int m, n;
            if (place(tid + 256 * u, m, n)) ahead[u] = epi.ahead(m, n, M, N);
        }
    }
    // the waves' sums through LDS, once every wave is done
    __syncthreads();
    i32x4* const red = reinterpret_cast<i32x4*>(smem);
#pragma unroll
    for (int i = 0; i < TM; ++i)
#pragma unroll
        for (int j = 0; j < TN; ++j) red[(wave * FR + i * TN + j) * 64 + lane] = acc[i][j];
    __syncthreads();
#pragma unroll
    for (int u = 0; u < PER; ++u) {
        int m, n;
        const int q = tid + 256 * u;
        if (!place(q, m, n)) continue;
        i32x4 v = red[q];
#pragma unroll
        for (int w = 1; w < WAVES; ++w) v += red[w * UNITS + q];
        if (splits > 1) *reinterpret_cast<i32x4*>(ws + ((size_t)split * M + m) * ((N + 3) & ~3) + n) = v;
        else epi.store(m, n, M, N, v, ahead[u]);
    }
}

// Adds up the sums of several ranges of K: a thread four columns of a row.
template <typename T>
__global__ __launch_bounds__(256) void i8_join_kernel(const int* __restrict__ ws, int splits, int M, int N, I8Epi<T> epi)
{
    const int groups = (N + 3) >> 2;
    const int64_t at = (int64_t)blockIdx.x * 256 + threadIdx.x;
    if (at >= (int64_t)M * groups) return;
    const int m = (int)(at / groups), n = (int)(at % groups) * 4;
    const i32x4* p = reinterpret_cast<const i32x4*>(ws) + at;
    const auto cols = epi.cols(n, N);
    const float sa = epi.scale_a[m];
    i32x4 v = *p;
#pragma unroll 4
    for (int s = 1; s < splits; ++s) v += p[(int64_t)s * M * groups];
    epi.store(m, n, M, N, v, cols, sa);
}

// ------------------------------------------------------------- the checks --

static bool i8_dtype_ok(int dtype) { return dtype == EBRL_DTYPE_FP32 || dtype == EBRL_DTYPE_BF16; }
static int i8_size(int dtype) { return dtype == EBRL_DTYPE_FP32 ? 4 : 2; }
// Rows of `width` elements every `ld`, element-aligned.
static bool i8_rows_ok(const void* p, int64_t ld, int64_t width, int esz) {
    return p && (uintptr_t)p % esz == 0 && ld >= width && ld < ((int64_t)1 << 40);
}
static bool i8_codes_ok(const void* p, int64_t ld, int64_t width) {
    return p && (uintptr_t)p % 16 == 0 && ld >= width && ld % 16 == 0;
}

template <typename T, int OP> static void i8_quant_op(const ebrl_i8_quant_args& a, hipStream_t s) {
    const int cols = a.cols;
    // a launch has under 2^32 threads
    constexpr int MOST = 1 << 21;
    if (a.rows > MOST) {
        ebrl_i8_quant_args part = a;
        for (int64_t r = 0; r < a.rows; r += MOST) {
            part.rows = (int)std::min<int64_t>(MOST, a.rows - r);
            part.x = (const T*)a.x + r * a.ldx;
            if (OP == EBRL_I8_SWIGLU) part.up = (const T*)a.up + r * a.ldup;
            part.codes = a.codes + r * a.ldc;
            part.scales = a.scales + r;
            i8_quant_op<T, OP>(part, s);
        }
        return;
    }
    const unsigned rows = a.rows;
    auto go = [&](auto kern, unsigned groups, int threads) {
        hipLaunchKernelGGL(kern, dim3(groups), dim3(threads), 0, s, a);
    };
    if (cols <= 512) go(i8_quant_kernel<T, OP, 1, 1>, (rows + 3) / 4, 256);
    else if (cols <= 1024) go(i8_quant_kernel<T, OP, 1, 2>, (rows + 3) / 4, 256);
    else if (cols <= 2048) go(i8_quant_kernel<T, OP, 4, 1>, rows, 256);
    else if (cols <= 4096) go(i8_quant_kernel<T, OP, 4, 2>, rows, 256);
    else if (cols <= 8192) go(i8_quant_kernel<T, OP, 8, 2>, rows, 512);
    else if (cols <= 12288) go(i8_quant_kernel<T, OP, 12, 2>, rows, 768);
    else if (cols <= 16384) go(i8_quant_kernel<T, OP, 16, 2>, rows, 1024);
    else go(i8_quant_long_kernel<T, OP>, rows, 1024);
}
template <typename T> static void i8_quant_launch(const ebrl_i8_quant_args& a, hipStream_t s) {
    if (a.op == EBRL_I8_ROWS) i8_quant_op<T, EBRL_I8_ROWS>(a, s);
    else if (a.op == EBRL_I8_RMSNORM) i8_quant_op<T, EBRL_I8_RMSNORM>(a, s);
    else i8_quant_op<T, EBRL_I8_SWIGLU>(a, s);
}

static int i8_quant(const ebrl_i8_quant_args* args, hipStream_t s) {
    if (!args) return EBRL_E_INVALID;
    const ebrl_i8_quant_args& a = *args;
    if (!i8_dtype_ok(a.dtype) || a.op < EBRL_I8_ROWS || a.op > EBRL_I8_SWIGLU || a.rows < 0 || a.cols < 1 ||
        a.cols > I8_MAX_COLS || (a.op == EBRL_I8_RMSNORM && !(a.eps >= 0.f && a.eps < INFINITY)) || (a.op != EBRL_I8_SWIGLU && a.up) ||
        (a.op != EBRL_I8_RMSNORM && a.gain))
        return EBRL_E_INVALID;
    if (a.rows == 0) return EBRL_OK;
    const int esz = i8_size(a.dtype);
    if (!i8_rows_ok(a.x, a.ldx, a.cols, esz) || (a.op == EBRL_I8_SWIGLU && !i8_rows_ok(a.up, a.ldup, a.cols, esz)) ||
        (uintptr_t)a.gain % 4 || !i8_codes_ok(a.codes, a.ldc, (a.cols + 15) / 16 * 16) || a.ldc >= ((int64_t)1 << 40) ||
        !a.scales || (uintptr_t)a.scales % 4)
        return EBRL_E_INVALID;
    if (esz == 2) i8_quant_launch<bf16_t>(a, s);
    else i8_quant_launch<float>(a, s);
    return hipGetLastError() == hipSuccess ? EBRL_OK : EBRL_E_HIP;
}

static bool i8_shape_ok(const ebrl_i8_gemm_args* a) {
    return a && i8_dtype_ok(a->dtype) && a->M >= 0 && a->N >= 0 && a->K >= 16 && a->K % 16 == 0 && a->K <= I8_MAX_K &&
           (((int64_t)a->M + 31) / 32) * (((int64_t)a->N + 63) / 64) <= I8_MAX_TILES;
}

enum { I8_BIG, I8_RING, I8_DECODE };
struct I8Plan {
    int kind, bm, bn;                // tile (decode: rows loaded, columns)
    int grid;                        // workgroups
    int full, cut;                   // big: evenly dealt tiles, parts of each tile of the last round
    int splits, per_split, m_tiles;  // decode: ranges of K, their K tiles
};

constexpr int i8_decode_stages(int xr, int bn) {
    // as many K tiles in LDS as fit, at most four and those in 128 KB
    const int per = 4 * (bn + xr) * 128;
    return 4 * per <= 128 * 1024 ? 4 : 3 * per <= 150 * 1024 ? 3 : 2;
}

// The kernel and tile whose modelled time (us) is least.  The constants are a fit to
// all candidates on 385 products (M 1 to 9216, N 300 to 22016, K 1024 to 11008, bf16
// output, weights from HBM).  On 385 others of that range the candidate it picks is within 1 %
// of the best one on 287, on average 2.4 % and at worst 28 % slower (1 to 8 rows on 22016
// outputs, where slices of 96 columns make one round).  No choice changes a result.
static I8Plan i8_plan(int M, int N, int K) {
    constexpr int CUS = 256;
    const int nk = (K + 127) / 128;
    auto up = [](int64_t a, int64_t b) { return (a + b - 1) / b; };
    I8Plan best{};
    double least = 1e300;
    auto consider = [&](const I8Plan& p, double t) {
        if (t < least) {
            least = t;
            best = p;
        }
    };
    // 256 x 256 tiles: whole rounds, then the others whole or cut in two or four where
    // the pieces fit one round.  A K tile of a piece takes `alone` with the chip nearly
    // empty and `busy` with a piece on every CU.
    const int64_t tiles = up(M, 256) * up(N, 256);
    const int64_t rounds = tiles / CUS, full = rounds * CUS, rest = tiles - full;
    struct Cut { int cut; double c, alone, busy; };
    for (const Cut& v : {Cut{1, 10.3, 0.86, 1.32}, Cut{2, 6.8, 0.67, 0.92}, Cut{4, 5.1, 0.48, 0.635}}) {
        if (v.cut > 1 && (!rest || rest * v.cut > CUS)) continue;
        // (pieces past the last row or column have nothing to do)
        const int64_t pieces = full || v.cut == 1 ? rest * v.cut : up(M, 128) * up(N, v.cut == 2 ? 256 : 128);
        double t = v.c + rounds * (9.1 + 1.3 * nk);
        if (rest) t += nk * (v.alone + (v.busy - v.alone) * pieces / CUS);
        consider(I8Plan{I8_BIG, 256, 256, (int)(full ? CUS : rest * v.cut), (int)full, v.cut, 1, nk, 1}, t);
    }
    // Ring tiles: two workgroups share a CU, so they take rounds of one (`one` us a K
    // tile) or two (`two`) a CU; of that and the weights, streamed once for each
    // group of four row tiles, the shorter one shows by a seventh.
    struct Ring { int bm, bn; double epi, one, two; };
    for (const Ring& v : {Ring{64, 128, 3.3, 0.42, 0.70}, Ring{64, 64, 1.0, 0.30, 0.385}, Ring{32, 64, 0.76, 0.20, 0.30}}) {
        const int64_t wgs = up(M, v.bm) * up(N, v.bn), pairs = wgs / (2 * CUS);
        const double left = (double)(wgs - pairs * 2 * CUS) / CUS;   // workgroups a CU in the last round
        double t = 2.9 + pairs * (v.epi + nk * v.two);
        if (left > 1) t += v.epi + nk * (v.one + (v.two - v.one) * (0.6 + 0.4 * (left - 1)));
        else if (left > 0) t += v.epi / 2 + nk * v.one;
        const double w = (double)N * K * 1e-6 * (0.26 + 0.163 * (up(up(M, v.bm), 4) - 1));
        t = std::max(t, w) + 0.14 * std::min(t, w);
        consider(I8Plan{I8_RING, v.bm, v.bn, (int)wgs, 0, 0, 1, nk, 1}, t);
    }
    // Decode: a K tile of the four waves is (bn + xr) * 512 bytes through LDS, at 57 or
    // 69 KB/us a CU by how many are in flight (more where few CUs work); the weights
    // come at 10 TB/s at best, and the shorter time shows by two fifths.  Several ranges
    // of K cost a launch more, and their sums' way through memory.  More than 512 rows
    // come from memory too, and a K tile takes a third longer: where one round of
    // workgroups does, for few outputs (66 such products that would be the ring's: 22 %
    // less time on average, 1609 x 52 x 10944 19.3 -> 11.8 us; on 80 others the pick is 4 %
    // slower than the best on average, 29 % at worst).
    {
        const int xr = M <= 8 ? 8 : M <= 16 ? 16 : M <= 32 ? 32 : up(M, up(M, 64)) <= 48 ? 48 : 64;
        const int m_tiles = (int)up(M, xr);
        for (int bn : {16, 32, 48, 64, 96})
            for (int want : {1, 2, 4, 8, 16}) {
                const int per = (int)up(nk, want), splits = (int)up(nk, per);
                const int64_t wgs = up(N, bn) * m_tiles * splits;
                if (wgs > I8_MAX_TILES || ((want > 1 || M > 512) && wgs > CUS) || (want > 1 && nk < want * 8)) continue;
                const double step = (bn + xr) * 0.512 / (i8_decode_stages(xr, bn) == 2 ? 57 : 69) *
                                    (0.83 + 0.17 * std::min(1.0, wgs / 256.0)) * (M > 512 ? 1.33 : 1.0);
                const double cu = up(wgs, CUS) * (0.96 + up(per, 4) * step), hbm = ((double)N + (M > 512 ? M : 0)) * K / 9.83e6;
                double t = 2.55 + std::max(cu, hbm) + 0.39 * std::min(cu, hbm);
                if (splits > 1) t += 2.2 + 5.3e-6 * splits * M * N;
                consider(I8Plan{I8_DECODE, xr, bn, (int)wgs, 0, 0, splits, per, m_tiles}, t);
            }
    }
    return best;
}
static int64_t i8_plan_bytes(const I8Plan& p, int M, int N) {
    return p.kind == I8_DECODE && p.splits > 1 ? (int64_t)p.splits * M * ((N + 3) & ~3) * 4 : 0;
}

template <typename T, int XR, int BN> static void i8_decode_launch(const ebrl_i8_gemm_args& a, const I8Plan& p,
                                                                   const I8Epi<T>& epi, hipStream_t s) {
    constexpr int STAGES = i8_decode_stages(XR, BN);
    auto go = [&](auto kern) {
        hipLaunchKernelGGL(kern, dim3(p.grid), dim3(256), 0, s, a.a, (uint32_t)a.lda,
                           a.b, (uint32_t)a.ldb, a.M, a.N, a.K, p.per_split, p.splits, p.m_tiles, (int*)a.workspace, epi);
    };
    if constexpr (XR > 32) {
        if (p.m_tiles > 1) { go(i8_decode_kernel<T, XR, BN, STAGES, false>); return; }
    }
    go(i8_decode_kernel<T, XR, BN, STAGES, true>);
}
template <typename T, int XR> static void i8_decode_slices(const ebrl_i8_gemm_args& a, const I8Plan& p, const I8Epi<T>& epi,
                                                           hipStream_t s) {
    switch (p.bn) {
    case 16: i8_decode_launch<T, XR, 16>(a, p, epi, s); break;
    case 32: i8_decode_launch<T, XR, 32>(a, p, epi, s); break;
    case 48: i8_decode_launch<T, XR, 48>(a, p, epi, s); break;
    case 64: i8_decode_launch<T, XR, 64>(a, p, epi, s); break;
    default: i8_decode_launch<T, XR, 96>(a, p, epi, s); break;
    }
}

template <typename T> static void i8_gemm_launch(const ebrl_i8_gemm_args& a, const I8Plan& p, hipStream_t s) {
    const I8Epi<T> epi{a.scale_a, a.scale_b, a.bias, (const T*)a.residual, (T*)a.c, a.ldr, a.ldc};
    if (p.kind == I8_DECODE) {
        switch (p.bm) {
        case 8: i8_decode_slices<T, 8>(a, p, epi, s); break;
        case 16: i8_decode_slices<T, 16>(a, p, epi, s); break;
        case 32: i8_decode_slices<T, 32>(a, p, epi, s); break;
        case 48: i8_decode_slices<T, 48>(a, p, epi, s); break;
        default: i8_decode_slices<T, 64>(a, p, epi, s); break;
        }
        if (p.splits > 1)
            hipLaunchKernelGGL(i8_join_kernel<T>, dim3((unsigned)(((int64_t)a.M * ((a.N + 3) / 4) + 255) / 256)), dim3(256),
                               0, s, (const int*)a.workspace, p.splits, a.M, a.N, epi);
        return;
    }
    if (p.kind == I8_BIG) {
        auto big = [&](auto kern) {
            hipLaunchKernelGGL(kern, dim3(p.grid), dim3(512), 0, s, a.a, (uint32_t)a.lda, a.b, (uint32_t)a.ldb, a.M, a.N, a.K,
                               p.full, p.cut, epi);
        };
        // Results that the 256 MB cache will not hold beside the operands until they are read,
        // in whole cache lines, are stored past it: with two sets of operands in turn 9216 x
        // 12288 x 4096 343 -> 330 us (bf16), 383 -> 360 (fp32), with the rows' quantisation
        // behind it 423 -> 412.  Smaller ones are read from it (5476 x 8192 x 1024 and its gated
        // rows 78 us, 84 past it), as is a residual stream (9216 x 4096 x 4096 and its norm 194, 200).
        const int64_t esz = sizeof(T);
        const bool stream = a.M * (a.N * esz) >= 128 << 20 && (uintptr_t)a.c % 128 == 0 && a.ldc * esz % 128 == 0;
        if (a.residual) big(i8_big_kernel<T, true, false>);
        else if (stream) big(i8_big_kernel<T, false, true>);
        else big(i8_big_kernel<T, false, false>);
        return;
    }
    auto ring = [&](auto kern) {
        hipLaunchKernelGGL(kern, dim3(p.grid), dim3(256), 0, s, a.a, (uint32_t)a.lda, a.b, (uint32_t)a.ldb, a.M, a.N, a.K, epi);
    };
    if (p.bn == 128) ring(i8_ring_kernel<T, 64, 128, 3>);
    else if (p.bm == 64) ring(i8_ring_kernel<T, 64, 64, 3>);
    else ring(i8_ring_kernel<T, 32, 64, 4>);
}

static int64_t i8_gemm_workspace(const ebrl_i8_gemm_args* a) {
    if (!i8_shape_ok(a)) return EBRL_E_INVALID;
    return a->M == 0 || a->N == 0 ? 0 : i8_plan_bytes(i8_plan(a->M, a->N, a->K), a->M, a->N);
}

static int i8_gemm(const ebrl_i8_gemm_args* args, hipStream_t s) {
    if (!i8_shape_ok(args)) return EBRL_E_INVALID;
    const ebrl_i8_gemm_args& a = *args;
    if (a.M == 0 || a.N == 0) return EBRL_OK;
    const int esz = i8_size(a.dtype);
    if (!i8_codes_ok(a.a, a.lda, a.K) || !i8_codes_ok(a.b, a.ldb, a.K) || a.lda >= I8_MAX_LD || a.ldb >= I8_MAX_LD ||
        !a.scale_a || !a.scale_b || (uintptr_t)a.scale_a % 4 || (uintptr_t)a.scale_b % 4 || (uintptr_t)a.bias % 4 ||
        !i8_rows_ok(a.c, a.ldc, a.N, esz) || (a.residual && !i8_rows_ok(a.residual, a.ldr, a.N, esz)) ||
        (a.residual == a.c && a.ldr != a.ldc))
        return EBRL_E_INVALID;
    const I8Plan p = i8_plan(a.M, a.N, a.K);
    const int64_t need = i8_plan_bytes(p, a.M, a.N);
    if (need > 0 && (!a.workspace || a.workspace_bytes < need || (uintptr_t)a.workspace % 16)) return EBRL_E_INVALID;
    if (esz == 2) i8_gemm_launch<bf16_t>(a, p, s);
    else i8_gemm_launch<float>(a, p, s);
    return hipGetLastError() == hipSuccess ? EBRL_OK : EBRL_E_HIP;
}

}  // namespace ebrl

extern "C" {

int ebrl_op_i8_quant(const ebrl_i8_quant_args* args, void* stream) { return ebrl::i8_quant(args, (hipStream_t)stream); }

int64_t ebrl_op_i8_gemm_workspace(const ebrl_i8_gemm_args* args) { return ebrl::i8_gemm_workspace(args); }

int ebrl_op_i8_gemm_plan(int32_t M, int32_t N, int32_t K, int32_t plan[6]) {
    ebrl_i8_gemm_args a{};
    a.M = M;
    a.N = N;
    a.K = K;
    if (!plan || !ebrl::i8_shape_ok(&a) || M == 0 || N == 0) return EBRL_E_INVALID;
    const ebrl::I8Plan p = ebrl::i8_plan(M, N, K);
    const int32_t out[6] = {p.kind, p.bm, p.bn, p.splits, p.grid, p.cut};
    std::copy(out, out + 6, plan);
    return EBRL_OK;
}

int ebrl_op_i8_gemm(const ebrl_i8_gemm_args* args, void* stream) { return ebrl::i8_gemm(args, (hipStream_t)stream); }

}  // extern "C"

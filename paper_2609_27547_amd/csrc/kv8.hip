// The paged KV cache in 8 bits (include/ebrl_kv8.h): rotary positions and
// cache write, and attention over the cache.
//
// kv8_write_kernel: a wave takes the new tokens of one page and a run of
//   heads; all of a (page, head)'s values meet in one wave, which has their
//   maximum, and so the scale, in registers before it stores a code.
// Kv8Rows: a wave's 16 QT query rows (a row is a token and a head of the KV
//   head's group), which take the keys 32 (two pages) at a time.  Codes come to
//   the lanes in the order in which v_mfma_f32_16x16x32_bf16 takes them and
//   become bf16 by v_cvt_scalef32_pk_bf16_fp8, which applies the page's scale:
//   four significant bits and a power of two, so exact.
// kv8_decode_kernel, kv8_prompt_kernel: few and many rows; kv8_join_kernel:
//   parts of a row's keys put together.
#include <float.h>
#include <limits.h>
#include <math.h>

#include "../../include/ebrl.h"
#include "../../include/ebrl_kv8.h"
#include "kernels.h"

namespace ebrl {

typedef __bf16 bf16x2 __attribute__((ext_vector_type(2)));
typedef float f32x2 __attribute__((ext_vector_type(2)));
typedef int i32x8 __attribute__((ext_vector_type(8)));

constexpr int KV8_PAGE = EBRL_KV8_PAGE;
constexpr int KV8_EXP_MIN = -100, KV8_EXP_MAX = 120;   // 448 * 2^120 > FLT_MAX
constexpr int KV8_Q_EXP_MIN = -122;   // of a query row's scale: every bf16 number is whole in two terms
constexpr float KV8_SLACK = 10.f;     // log2 of the largest weight that a softmax keeps
constexpr float KV8_FAR = 0x1p24f;    // scores from here on are whole numbers, rounded before the maximum is taken off
constexpr int KV8_MAX_PARTS = 256;    // parts that a row's keys are cut into

// ----------------------------------------------------------------- write --

// A double as the float next to it with the last bit set where that is not
// exact: rounding it to eight bits or fewer then gives what rounding the
// double itself gives.
EBRL_DEV float kv8_odd(double d) {
    const float f = (float)d;
    const double b = (double)f;
    unsigned u = __float_as_uint(f);
    if (fabs(b) > fabs(d)) u -= 1;
    if (b != d) u |= 1;
    return __uint_as_float(u);
}
// What is stored of a value: itself, or NaN
EBRL_DEV float kv8_storable(float v) {
    return fabsf(v) < 0x1p127f ? v : __uint_as_float(0x7fc00000u);
}
// Least e >= `least` with a <= 448 * 2^e = 1.75 * 2^(8 + e); a >= 0, finite.
EBRL_DEV int kv8_exponent(float a, int least = KV8_EXP_MIN) {
    const unsigned u = __float_as_uint(a);
    return max((int)(u >> 23) - 127 - ((u & 0x7fffffu) <= 0x600000u ? 8 : 7), least);
}
EBRL_DEV float kv8_pow2(int e) { return __uint_as_float((unsigned)(max(e, -126) + 127) << 23); }
EBRL_DEV unsigned kv8_pack4(float a, float b, float c, float d) {
    int w = __builtin_amdgcn_cvt_pk_fp8_f32(a, b, 0, false);
    return (unsigned)__builtin_amdgcn_cvt_pk_fp8_f32(c, d, w, true);
}
// Four codes whose scale grows: values times `shift` (a power of two, <= 1).
EBRL_DEV unsigned kv8_shift4(unsigned w, float shift) {
    const f32x2 lo = __builtin_amdgcn_cvt_pk_f32_fp8(w, false), hi = __builtin_amdgcn_cvt_pk_f32_fp8(w, true);
    return kv8_pack4(lo[0] * shift, lo[1] * shift, hi[0] * shift, hi[1] * shift);
}

template <typename T, int N> EBRL_DEV void kv8_load(const T* p, float* o);
template <> EBRL_DEV void kv8_load<float, 4>(const float* p, float* o) {
    const float4 a = *reinterpret_cast<const float4*>(p);
    o[0] = a.x; o[1] = a.y; o[2] = a.z; o[3] = a.w;
}
template <> EBRL_DEV void kv8_load<float, 8>(const float* p, float* o) {
    kv8_load<float, 4>(p, o);
    kv8_load<float, 4>(p + 4, o + 4);
}
template <> EBRL_DEV void kv8_load<bf16_t, 4>(const bf16_t* p, float* o) {
    const uint2 u = *reinterpret_cast<const uint2*>(p);
    o[0] = __uint_as_float(u.x << 16); o[1] = __uint_as_float(u.x & 0xffff0000u);
    o[2] = __uint_as_float(u.y << 16); o[3] = __uint_as_float(u.y & 0xffff0000u);
}
template <> EBRL_DEV void kv8_load<bf16_t, 8>(const bf16_t* p, float* o) {
    const uint4 u = *reinterpret_cast<const uint4*>(p);
    const unsigned w[4] = {u.x, u.y, u.z, u.w};
#pragma unroll
    for (int i = 0; i < 4; ++i) {
        o[2 * i] = __uint_as_float(w[i] << 16);
        o[2 * i + 1] = __uint_as_float(w[i] & 0xffff0000u);
    }
}
EBRL_DEV void kv8_store8(float* p, const float* y) {
    *reinterpret_cast<float4*>(p) = make_float4(y[0], y[1], y[2], y[3]);
    *reinterpret_cast<float4*>(p + 4) = make_float4(y[4], y[5], y[6], y[7]);
}
EBRL_DEV void kv8_store8(bf16_t* p, const float* y) {
    bf16x8 o;
#pragma unroll
    for (int i = 0; i < 8; ++i) o[i] = (__bf16)y[i];
    *reinterpret_cast<bf16x8*>(p) = o;
}

// N elements as they lie in memory (N * sizeof(T) a multiple of 16 bytes).
template <typename T, int N> struct Kv8Raw {
    uint4 w[N * sizeof(T) / 16];
    EBRL_DEV void load(const T* p) {
#pragma unroll
        for (int i = 0; i < (int)(N * sizeof(T) / 16); ++i) w[i] = reinterpret_cast<const uint4*>(p)[i];
    }
    EBRL_DEV void get(float (&o)[N]) const {
#pragma unroll
        for (int q = 0; q < N; q += 8) kv8_load<T, 8>(reinterpret_cast<const T*>(w) + q, o + q);
    }
};

struct Kv8WriteKernelArgs {
    ebrl_kv8_cache c;
    ebrl_kv8_write_args a;
    int pages;        // most pages of a sequence that a call touches
    int per_wave;     // heads that a wave takes in turn
    int rot_units, v_units;   // waves of a (sequence, page): for the Q and K heads, for the V heads
};

// The new tokens of one page: slots s0 .. s1 - 1 of `page` (outside the pool:
// there is none), slot t's row row0 + t.
struct Kv8Span { int s0, s1, row0, pos0, page; };
EBRL_DEV bool kv8_span(const Kv8WriteKernelArgs& w, int i, int pg, Kv8Span& s) {
    const ebrl_kv8_write_args& a = w.a;
    const int trow = a.seq ? a.seq[i] : i;
    const int r0 = min(max(a.row_start[i], 0), a.rows);
    const int len = min(min(max(a.row_start[i + 1], 0), a.rows) - r0, a.max_len);
    const int p0 = a.pos0[i];
    if (trow < 0 || trow >= w.c.table_rows || len <= 0 || p0 < 0 || p0 >= w.c.table_stride * KV8_PAGE) return false;
    const int at = p0 / KV8_PAGE + pg;
    if (at >= w.c.table_stride) return false;
    const int first = at * KV8_PAGE - p0;             // token of slot 0, counted from the first new one
    s.s0 = max(-first, 0);
    s.s1 = min(KV8_PAGE, len - first);
    s.row0 = r0 + first;
    s.pos0 = at * KV8_PAGE;
    s.page = w.c.block_table[(size_t)trow * w.c.table_stride + at];
    return s.s1 > s.s0;
}

// The table row of a pair's axis.
EBRL_DEV int kv8_axis_row(int pair, int b1, int b2, int row0, int row1, int row2) {
    return pair < b1 ? row0 : pair < b2 ? row1 : row2;
}

// Cosines and sines of N pairs from pair `at` on (multiples of 4) for `row` at
// cache position `pos`: each from the table row of its axis's position.
template <int HALF, int N>
EBRL_DEV void kv8_angles(const ebrl_kv8_write_args& a, int row, int pos, int at, float (&cs)[N], float (&sn)[N]) {
    const int* ap = a.axis_pos ? a.axis_pos + (size_t)row * a.n_axes : nullptr;
    const int b1 = a.sections[0], b2 = b1 + (a.n_axes > 1 ? a.sections[1] : 0);
    const int most = a.tab_rows - 1;
    const int row0 = min(max(ap ? ap[0] : pos, 0), most), row1 = min(max(a.n_axes > 1 ? ap[1] : 0, 0), most);
    const int row2 = min(max(a.n_axes > 2 ? ap[2] : 0, 0), most);
    // four pairs of one axis at a time, unless axes change inside four
    const bool whole = (b1 & 3) == 0 && (b2 & 3) == 0;
#pragma unroll
    for (int q = 0; q < N; q += 4) {
        if (whole) {
            const size_t o = (size_t)kv8_axis_row(at + q, b1, b2, row0, row1, row2) * HALF + at + q;
            kv8_load<float, 4>(a.cos_tab + o, cs + q);
            kv8_load<float, 4>(a.sin_tab + o, sn + q);
        } else {
#pragma unroll
            for (int j = 0; j < 4; ++j) {
                const size_t o = (size_t)kv8_axis_row(at + q + j, b1, b2, row0, row1, row2) * HALF + at + q + j;
                cs[q + j] = a.cos_tab[o];
                sn[q + j] = a.sin_tab[o];
            }
        }
    }
}

// Pairs (x0, x1) turned, in 64 bits (the products are exact, so each result is
// rounded once there) and rounded to odd, so that the rounding that follows is
// that of the 64-bit value; `whole`: the results are the 32-bit values.
template <int N>
EBRL_DEV void kv8_turn(float (&x0)[N], float (&x1)[N], const float (&cs)[N], const float (&sn)[N], bool whole) {
#pragma unroll
    for (int q = 0; q < N; ++q) {
        const double c = cs[q], s = sn[q], u = x0[q], v = x1[q];
        const double y0 = fma(u, c, -(v * s)), y1 = fma(v, c, u * s);
        x0[q] = whole ? (float)y0 : kv8_odd(y0);
        x1[q] = whole ? (float)y1 : kv8_odd(y1);
    }
}

// Exponent of a group's stored scale.
EBRL_DEV int kv8_stored_exponent(float scale) {
    return min(max((int)(__float_as_uint(scale) >> 23 & 255) - 127, KV8_EXP_MIN), KV8_EXP_MAX);
}

// Largest magnitude that is stored of x; what is not stored becomes NaN.
template <int N> EBRL_DEV float kv8_amax(float (&x)[N]) {
    float am = 0.f;
#pragma unroll
    for (int q = 0; q < N; ++q) {
        x[q] = kv8_storable(x[q]);
        am = fmaxf(am, fabsf(x[q]));   // passes a NaN over
    }
    return am;
}

// A call of several tokens a sequence: a wave takes the new tokens of a page
// and a run of heads, Q and K heads or V heads.  Bound by bytes: nine sequences
// of 3001 to 4095 tokens, 32 Q and 8 + 8 KV heads of 128, take 141 us, 5.0 TB/s,
// the rate of a copy; 16 of 600 tokens 37 us, 3.7 TB/s.  Four heads a wave in
// turn share the cosines and sines; one head a wave where there are too few
// waves to fill the chip.
template <typename T, int HD>
__global__ __launch_bounds__(256) void kv8_write_kernel(Kv8WriteKernelArgs w)
{
    constexpr int HALF = HD / 2;
    constexpr int PL = HD / 8;           // pairs of a lane: four lanes share a token's head
    const ebrl_kv8_write_args& a = w.a;
    const int lane = threadIdx.x & 63;
    const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    const int per_page = w.rot_units + w.v_units;
    const unsigned id = blockIdx.x * 4u + wave;
    const int unit = id % per_page;
    const unsigned sp = id / per_page;
    const int pg = sp % w.pages, i = sp / w.pages;
    Kv8Span s;
    if (i >= a.n || !kv8_span(w, i, pg, s)) return;
    const int s0 = s.s0, s1 = s.s1;
    const bool there = s.page >= 0 && s.page < w.c.num_blocks;
    const int hkv = w.c.kv_heads;
    uint8_t* const codes = (uint8_t*)w.c.codes;

    if (unit < w.rot_units) {
        // Q and K heads: lane (t, g) has slot t's pairs PL g .. PL g + PL - 1
        const int t = lane >> 2, g = lane & 3;
        const bool mine = t >= s0 && t < s1;
        const int slot = mine ? t : s0, row = s.row0 + slot;
        const int h_lo = unit * w.per_wave, h_hi = min(h_lo + w.per_wave, a.q_heads + hkv);
        auto src = [&](int h) {
            return (h < a.q_heads ? (const T*)a.q + (size_t)row * a.ldq + h * HD
                                  : (const T*)a.k + (size_t)row * a.ldk + (h - a.q_heads) * HD) + PL * g;
        };
        Kv8Raw<T, PL> r0, r1;
        r0.load(src(h_lo));
        r1.load(src(h_lo) + HALF);
        float cs[PL], sn[PL];
        if (a.n_axes) kv8_angles<HALF, PL>(a, row, s.pos0 + slot, PL * g, cs, sn);
        for (int h = h_lo; h < h_hi; ++h) {
            const bool isq = h < a.q_heads;
            const int hh = isq ? h : h - a.q_heads;
            float x0[PL], x1[PL];
            r0.get(x0);
            r1.get(x1);
            const T* const next = src(min(h + 1, h_hi - 1));   // in flight while this head is worked on
            r0.load(next);
            r1.load(next + HALF);
            if (a.n_axes) kv8_turn<PL>(x0, x1, cs, sn, sizeof(T) == 4 && isq);
            if (isq) {
                if (mine) {
                    T* dst = (T*)a.q_out + (size_t)row * a.ldq_out + hh * HD + PL * g;
#pragma unroll
                    for (int q = 0; q < PL; q += 8) {
                        kv8_store8(dst + q, x0 + q);
                        kv8_store8(dst + HALF + q, x1 + q);
                    }
                }
                continue;
            }
            if (!there) continue;
            const float am = fmaxf(kv8_amax<PL>(x0), kv8_amax<PL>(x1));
            int e = kv8_exponent(wave_max(mine ? am : 0.f));
            const size_t grp = (size_t)s.page * 2 * hkv + hh;
            // lane's codes: pairs' first elements, and second ones HALF dims on
            uint8_t* const dst = codes + grp * (KV8_PAGE * HD) + t * 64 + PL * g;
            constexpr int HI = HD == 128 ? 1024 : 32;
            if (s0 > 0) {
                const int was = kv8_stored_exponent(w.c.scales[grp]);
                if (e > was && t < s0) {
                    const float sh = kv8_pow2(was - e);
#pragma unroll
                    for (int q = 0; q < PL; q += 4) {
                        unsigned* lo = reinterpret_cast<unsigned*>(dst + q);
                        unsigned* hi = reinterpret_cast<unsigned*>(dst + HI + q);
                        *lo = kv8_shift4(*lo, sh);
                        *hi = kv8_shift4(*hi, sh);
                    }
                }
                e = max(e, was);
            }
            if (mine) {
                const float inv = kv8_pow2(-e);
                unsigned lo[PL / 4], hi[PL / 4];
#pragma unroll
                for (int q = 0; q < PL; q += 4) {
                    lo[q / 4] = kv8_pack4(x0[q] * inv, x0[q + 1] * inv, x0[q + 2] * inv, x0[q + 3] * inv);
                    hi[q / 4] = kv8_pack4(x1[q] * inv, x1[q + 1] * inv, x1[q + 2] * inv, x1[q + 3] * inv);
                }
                if constexpr (PL == 16) {
                    *reinterpret_cast<uint4*>(dst) = make_uint4(lo[0], lo[1], lo[2], lo[3]);
                    *reinterpret_cast<uint4*>(dst + HI) = make_uint4(hi[0], hi[1], hi[2], hi[3]);
                } else {
                    *reinterpret_cast<uint2*>(dst) = make_uint2(lo[0], lo[1]);
                    *reinterpret_cast<uint2*>(dst + HI) = make_uint2(hi[0], hi[1]);
                }
            }
            if (lane == 0) w.c.scales[grp] = kv8_pow2(e);
        }
    } else {
        // V heads: lane (g, l) has slots 4 g .. 4 g + 3 of dims 64 c + 4 l .. + 3: the 16 bytes it stores
        if (!there) return;
        const int g = lane >> 4, l = lane & 15;
        constexpr int NC = HD / 64;
        const int u = unit - w.rot_units;
        const int h_lo = u * w.per_wave, h_hi = min(h_lo + w.per_wave, hkv);
        // bytes of a dword that hold slots before the new ones (their values
        // stay), and those or slots behind (their bytes stay)
        unsigned before = 0, keep = 0;
#pragma unroll
        for (int j = 0; j < 4; ++j) {
            if (4 * g + j < s0) before |= 0xffu << (8 * j);
            if (4 * g + j < s0 || 4 * g + j >= s1) keep |= 0xffu << (8 * j);
        }
        for (int h = h_lo; h < h_hi; ++h) {
            float x[4][4 * NC];
            float am = 0.f;
#pragma unroll
            for (int j = 0; j < 4; ++j) {
                const int t = 4 * g + j;
                const bool mine = t >= s0 && t < s1;
                const T* src = (const T*)a.v + (size_t)(s.row0 + (mine ? t : s0)) * a.ldv + h * HD + 4 * l;
#pragma unroll
                for (int c = 0; c < NC; ++c) kv8_load<T, 4>(src + 64 * c, x[j] + 4 * c);
                const float m = kv8_amax<4 * NC>(x[j]);
                if (mine) am = fmaxf(am, m);
            }
            int e = kv8_exponent(wave_max(am));
            const size_t grp = ((size_t)s.page * 2 + 1) * hkv + h;
            uint4* const dst = reinterpret_cast<uint4*>(codes + grp * (KV8_PAGE * HD)) + lane;
            float sh = 1.f;
            if (s0 > 0) {
                const int was = kv8_stored_exponent(w.c.scales[grp]);
                if (e > was) sh = kv8_pow2(was - e);
                e = max(e, was);
            }
            const float inv = kv8_pow2(-e);
            if (keep != ~0u || (before && sh != 1.f)) {
#pragma unroll
                for (int c = 0; c < NC; ++c) {
                    uint4 old = make_uint4(0, 0, 0, 0);
                    if (keep) old = dst[64 * c];
                    unsigned o[4] = {old.x, old.y, old.z, old.w};
#pragma unroll
                    for (int d = 0; d < 4; ++d) {
                        const int q = 4 * c + d;
                        const unsigned nw = kv8_pack4(x[0][q] * inv, x[1][q] * inv, x[2][q] * inv, x[3][q] * inv);
                        if (sh != 1.f) o[d] = (kv8_shift4(o[d], sh) & before) | (o[d] & ~before);
                        o[d] = (o[d] & keep) | (nw & ~keep);
                    }
                    dst[64 * c] = make_uint4(o[0], o[1], o[2], o[3]);
                }
            }
            if (lane == 0) w.c.scales[grp] = kv8_pow2(e);
        }
    }
}

// Largest over the LPH lanes (4 or 8) that share a head.
template <int LPH> EBRL_DEV float kv8_head_max(float v) {
    v = fmaxf(v, dpp_f<DPP_SWAP1>(v));
    v = fmaxf(v, dpp_f<DPP_SWAP2>(v));
    return LPH == 8 ? fmaxf(v, dpp_f<DPP_HALF_MIRROR>(v)) : v;
}

// One token a sequence: a wave takes 64 / LPH heads of a sequence's token,
// eight pairs (Q, K) or sixteen dims (V) a lane, so that every lane has work.
// Bound by latency: the chain is lengths, page, scale, codes (3.3 us for one
// sequence, 3.6 for 101).
template <typename T, int HD>
__global__ __launch_bounds__(256) void kv8_write_token_kernel(Kv8WriteKernelArgs w)
{
    constexpr int HALF = HD / 2, LPH = HD / 16, HPW = 64 / LPH;
    const ebrl_kv8_write_args& a = w.a;
    const int lane = threadIdx.x & 63;
    const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    const int per = w.rot_units + w.v_units;
    const unsigned id = blockIdx.x * 4u + wave;
    const int unit = id % per, i = id / per;
    Kv8Span s;
    if (i >= a.n || !kv8_span(w, i, 0, s)) return;
    const int t = s.s0, row = s.row0 + t;
    const bool there = s.page >= 0 && s.page < w.c.num_blocks;
    const int hkv = w.c.kv_heads;
    const int j = lane % LPH;
    if (unit < w.rot_units) {
        const int h = unit * HPW + lane / LPH, hs = min(h, a.q_heads + hkv - 1);
        const bool isq = hs < a.q_heads;
        const int hh = isq ? hs : hs - a.q_heads;
        const T* src = isq ? (const T*)a.q + (size_t)row * a.ldq : (const T*)a.k + (size_t)row * a.ldk;
        src += hh * HD + 8 * j;
        const size_t grp = (size_t)(there ? s.page : 0) * 2 * hkv + hh;
        const float stored = isq ? 0.f : w.c.scales[grp];
        float x0[8], x1[8], cs[8], sn[8];
        kv8_load<T, 8>(src, x0);
        kv8_load<T, 8>(src + HALF, x1);
        if (a.n_axes) {
            kv8_angles<HALF, 8>(a, row, s.pos0 + t, 8 * j, cs, sn);
            kv8_turn<8>(x0, x1, cs, sn, sizeof(T) == 4 && isq);
        }
        if (isq) {
            T* dst = (T*)a.q_out + (size_t)row * a.ldq_out + hh * HD + 8 * j;
            kv8_store8(dst, x0);
            kv8_store8(dst + HALF, x1);
        }
        int e = kv8_exponent(kv8_head_max<LPH>(fmaxf(kv8_amax<8>(x0), kv8_amax<8>(x1))));
        if (isq || !there || h != hs) return;
        uint8_t* const dst = (uint8_t*)w.c.codes + grp * (KV8_PAGE * HD) + 8 * j;
        constexpr int HI = HD == 128 ? 1024 : 32;
        if (t > 0) {
            const int was = kv8_stored_exponent(stored);
            if (e > was) {
                const float sh = kv8_pow2(was - e);
                for (int b = 0; b < t; ++b)
#pragma unroll
                    for (int x = 0; x < 2; ++x) {
                        uint2* const at = reinterpret_cast<uint2*>(dst + b * 64 + x * HI);
                        *at = make_uint2(kv8_shift4(at->x, sh), kv8_shift4(at->y, sh));
                    }
            }
            e = max(e, was);
        }
        const float inv = kv8_pow2(-e);
#pragma unroll
        for (int x = 0; x < 2; ++x) {
            const float* const y = x ? x1 : x0;
            *reinterpret_cast<uint2*>(dst + t * 64 + x * HI) =
                make_uint2(kv8_pack4(y[0] * inv, y[1] * inv, y[2] * inv, y[3] * inv),
                           kv8_pack4(y[4] * inv, y[5] * inv, y[6] * inv, y[7] * inv));
        }
        if (j == 0) w.c.scales[grp] = kv8_pow2(e);
    } else {
        const int h = (unit - w.rot_units) * HPW + lane / LPH, hh = min(h, hkv - 1);
        const T* src = (const T*)a.v + (size_t)row * a.ldv + hh * HD + 16 * j;
        float x[16];
        kv8_load<T, 8>(src, x);
        kv8_load<T, 8>(src + 8, x + 8);
        const size_t grp = ((size_t)(there ? s.page : 0) * 2 + 1) * hkv + hh;
        // the lane's 16 dims are 64 bytes of each four slots
        uint4* const dst = reinterpret_cast<uint4*>((uint8_t*)w.c.codes + grp * (KV8_PAGE * HD) + j / 4 * 1024) + j % 4 * 4;
        const float stored = w.c.scales[grp];
        uint4 old[4];
#pragma unroll
        for (int x4 = 0; x4 < 4; ++x4) old[x4] = dst[t / 4 * 16 + x4];
        int e = kv8_exponent(kv8_head_max<LPH>(kv8_amax<16>(x)));
        if (!there || h != hh) return;
        float sh = 1.f;
        if (t > 0) {
            const int was = kv8_stored_exponent(stored);
            if (e > was) sh = kv8_pow2(was - e);
            e = max(e, was);
        }
        const float inv = kv8_pow2(-e);
        if (sh != 1.f)
            for (int b = 0; b < t / 4; ++b)
#pragma unroll
                for (int x4 = 0; x4 < 4; ++x4) {
                    uint4* const at = dst + b * 16 + x4;
                    const uint4 o = *at;
                    *at = make_uint4(kv8_shift4(o.x, sh), kv8_shift4(o.y, sh), kv8_shift4(o.z, sh), kv8_shift4(o.w, sh));
                }
        const int bit = 8 * (t & 3);
        const unsigned before = (1u << bit) - 1, mine = 0xffu << bit;
#pragma unroll
        for (int x4 = 0; x4 < 4; ++x4) {
            unsigned o[4] = {old[x4].x, old[x4].y, old[x4].z, old[x4].w};
#pragma unroll
            for (int d = 0; d < 4; ++d) {
                const float v = x[4 * x4 + d] * inv;
                if (sh != 1.f) o[d] = (kv8_shift4(o[d], sh) & before) | (o[d] & ~before);
                o[d] = (o[d] & ~mine) | (kv8_pack4(v, v, v, v) & mine);
            }
            dst[t / 4 * 16 + x4] = make_uint4(o[0], o[1], o[2], o[3]);
        }
        if (j == 0) w.c.scales[grp] = kv8_pow2(e);
    }
}

// ------------------------------------------------------------- attention --

// How a call is cut into workgroups of four waves.
enum Kv8Kind {
    KV8_WAVE,     // decode: each wave has a (sequence, KV head)'s rows, up to 16, to itself
    KV8_GROUP,    // decode: the four waves share the rows and deal the keys
    KV8_PAIRS,    // prompt: two waves share 16 rows, 32 rows a workgroup
    KV8_ROWS,     // prompt: 16 rows a wave, 64 a workgroup
    KV8_TALL      // prompt, bf16: 32 rows a wave, 128 a workgroup
};
struct Kv8Plan {
    Kv8Kind kind = KV8_GROUP;
    int tile_rows = 16;   // query rows (token, head of the group) of a workgroup or, KV8_WAVE, a wave
    int tiles = 1;        // of them, that a (sequence, KV head)'s rows take
    int parts = 1;        // most parts that a tile's keys are cut into
    int part_keys = 0;    // keys of a part
};

struct Kv8AttnKernelArgs {
    ebrl_kv8_cache c;
    ebrl_kv8_attn_args a;
    int grp, tiles, tile_rows, parts, part_keys;
    int join_rows;    // rows of a tile, at most
    float scale_log2;
    float* part_o;    // [unit][part][tile_rows][head_dim], unit = (sequence, KV head, tile)
    float* part_ml;   // [unit][part][tile_rows][2]: maximum and sum
};

// What a tile of query rows has before it.
struct Kv8Tile {
    int r0, m;         // first row and rows of the sequence
    int rows, t0;      // its (token, head) rows, the tile's first
    int len;           // keys of the sequence
    int parts;         // parts that the keys seen by some row are cut into
    int end;           // those keys
    const int* table;  // the sequence's pages
};
// Sequence i's row of the block table, or -1.
EBRL_DEV int kv8_table_row(const Kv8AttnKernelArgs& w, int i) {
    const int row = w.a.seq ? w.a.seq[i] : i;
    return row < w.c.table_rows ? max(row, -1) : -1;
}
EBRL_DEV Kv8Tile kv8_tile(const Kv8AttnKernelArgs& w, int i, int tile) {
    const ebrl_kv8_attn_args& a = w.a;
    Kv8Tile t;
    const int trow = kv8_table_row(w, i);
    t.r0 = min(max(a.row_start[i], 0), a.rows);
    t.m = min(max(min(max(a.row_start[i + 1], 0), a.rows) - t.r0, 0), a.max_q_len);
    t.rows = t.m * w.grp;
    t.t0 = tile * w.tile_rows;
    t.len = trow >= 0 ? min(max(a.kv_len[i], 0), min(a.max_kv_len, w.c.table_stride * KV8_PAGE)) : 0;
    const int last = (min(t.t0 + w.tile_rows, t.rows) - 1) / w.grp;
    t.end = a.causal ? max(min(t.len, t.len - t.m + last + 1), 0) : t.len;
    t.parts = max(1, (t.end + w.part_keys - 1) / w.part_keys);
    t.table = w.c.block_table + (size_t)max(trow, 0) * w.c.table_stride;
    return t;
}

// First key of a part of a (sequence, KV head) that is there, or INT_MAX; by a
// whole wave, 64 pages at a time.
EBRL_DEV int kv8_first_key(const Kv8AttnKernelArgs& w, unsigned pair, int part) {
    asm volatile("" : "+s"(pair));   // the table's row is worked out again, not kept through the loop over keys
    const int trow = kv8_table_row(w, pair / w.c.kv_heads);
    if (trow < 0) return INT_MAX;
    const int* const table = w.c.block_table + (size_t)trow * w.c.table_stride;
    const int lo = part * (w.part_keys / KV8_PAGE), hi = min(lo + w.part_keys / KV8_PAGE, w.c.table_stride);
    const int lane = threadIdx.x & 63;
    for (int p = lo; p < hi; p += 64) {
        const int page = p + lane < hi ? table[p + lane] : -1;
        const uint64_t there = __ballot(page >= 0 && page < w.c.num_blocks);
        if (there) return (p + __builtin_ctzll(there)) * KV8_PAGE;
    }
    return INT_MAX;
}

// Eight codes (two dwords) as bf16, the scales applied.
EBRL_DEV bf16x8 kv8_bf16(unsigned lo, unsigned hi, float sl, float sh) {
    const bf16x2 a = __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(lo, sl, false);
    const bf16x2 b = __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(lo, sl, true);
    const bf16x2 c = __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(hi, sh, false);
    const bf16x2 d = __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(hi, sh, true);
    return bf16x8{a[0], a[1], b[0], b[1], c[0], c[1], d[0], d[1]};
}

// Bit 7 of each byte that is a NaN code.
EBRL_DEV unsigned kv8_nan_bytes(unsigned w) { return ((w & 0x7f7f7f7fu) + 0x01010101u) & 0x80808080u; }

// A float as NP bf16 terms that add up to it (three hold all 24 bits).
template <int NP> EBRL_DEV void kv8_split(float x, __bf16* o) {
#pragma unroll
    for (int p = 0; p < NP; ++p) {
        o[p] = (__bf16)x;
        x -= (float)o[p];
    }
}

// x - m with x = s scale rounded as a float.  The fused form takes the exact
// product, which from 2^24 on lies further than one from x: where m is the
// largest x, weights relative to it would be anything.
EBRL_DEV float kv8_scaled(float s, float scale, float m) {
#pragma clang fp contract(off)
    const float x = s * scale;
    return x - m;
}

// What a row's weighted sum is multiplied by: 0 where it sees no key.
EBRL_DEV float kv8_inverse(float mx, float sum) { return mx == -INFINITY ? 0.f : 1.f / sum; }

// The state of a wave's 16 QT query rows.  Lane (r, g) holds query r of each
// 16: its elements 64 c + 16 g .. + 15, its scores for keys 4 g .. 4 g + 3 of
// each page, and its results in dims 64 c + 16 g .. + 15.
template <typename T, int HD, int QT, bool MX, int WP> struct Kv8Rows {
    static constexpr int NP = sizeof(T) == 4 ? 3 : 1;   // bf16 terms of a query element
    // WP: bf16 terms of a weight.  Three hold all 24 bits (fp32 rows).  Two are
    // off by 2^-17 at most: decode, whose time is the cache's bytes (61 sequences
    // 97.4 us, with one term 97.0 to 99.3).  One is off by 2^-8: prompts, which a
    // second term would slow by a fifth to two fifths.  Their sum is of the
    // rounded weights, by a product with ones, so that a row's result is a mean
    // of its keys' values whatever the rounding (a key that outweighs all others
    // gives its value), and the vector adds fall away (727 us against 737 a long
    // prompt, 163 against 171 at head dim 64).
    static constexpr int NC = HD / 64;
    // MX: K's codes enter the first product as they are, in
    // v_mfma_scale_f32_16x16x128_f8f6f4 with the page's scale, and q as two
    // e4m3 terms with scales of their own.  A bf16 element has eight
    // significant bits and a term four: they are exact down to 2^-13 of the
    // row's largest element, and off by 2^-21 of that at most below.  The
    // products take the same time as the bf16 ones, and half the conversions
    // of codes fall away.  Head dim 128: a product for each term.  Head dim 64:
    // one for both.  Of a lane's 32 elements the first 16 are the product's
    // elements 16 g .. 16 g + 15 and the others 64 more; they hold the first
    // and the second term of the same dims, K's codes enter twice, and the
    // scales, which lane g gives for elements 32 g .. 32 g + 31, are the first
    // term's in lanes 0 and 1 and the second's in lanes 2 and 3.
    static_assert(!MX || NP == 1, "a bf16 element has two e4m3 terms");
    static constexpr int QP = MX && HD == 128 ? 2 : 1;  // products for q's terms
    bf16x8 q[QT][NP][MX ? 1 : HD / 32];
    i32x8 q8[QT][QP];
    int q8_scale[QT];         // exponent byte of q8[.][0]'s scale; a second term's is 4 less
    f32x4 acc[QT][HD / 16];   // acc[4 c + d][v]: dim 64 c + 16 g + 4 v + d
    float mx[QT], sum[QT];    // log2 of what the weights are relative to; WP > 1: this lane's share of their sum
    f32x4 ones[WP == 1 ? QT : 1];   // WP 1: the whole sum, four times
    int lim[QT];              // keys that the row sees
    int all, end;             // keys that every row, that some row of the wave sees
    bool far;                 // some row's mx is KV8_FAR and more

    EBRL_DEV void init(const Kv8AttnKernelArgs& w, const Kv8Tile& t, int kvh, int wr0, int k_hi, int lane) {
        const int r = lane & 15, g = lane >> 4;
#pragma unroll
        for (int qt = 0; qt < QT; ++qt) {
            const int row = min(wr0 + 16 * qt + r, t.rows - 1);
            const int tok = row / w.grp, h = kvh * w.grp + (row - tok * w.grp);
            lim[qt] = w.a.causal ? min(t.len, t.len - t.m + tok + 1) : t.len;
            const T* src = (const T*)w.a.q + (size_t)(t.r0 + tok) * w.a.ldq + h * HD;
            if constexpr (MX) {
                float x[NC][16];
                float am = 0.f;
#pragma unroll
                for (int c = 0; c < NC; ++c) {
                    kv8_load<T, 8>(src + 64 * c + 16 * g, x[c]);
                    kv8_load<T, 8>(src + 64 * c + 16 * g + 8, x[c] + 8);
#pragma unroll
                    for (int j = 0; j < 16; ++j) am = fmaxf(am, fabsf(x[c][j]));
                }
                // the terms' scale bytes, e + 127 and 4 less, stay above 0
                const int e = kv8_exponent(attn_max_xor16_32(am), KV8_Q_EXP_MIN);
                const float inv = kv8_pow2(-e);
                q8_scale[qt] = e + 127 - (QP == 1 && g >= 2 ? 4 : 0);
#pragma unroll
                for (int c = 0; c < NC; ++c)
#pragma unroll
                    for (int j = 0; j < 16; j += 4) {
                        float y[4];
#pragma unroll
                        for (int z = 0; z < 4; ++z) y[z] = x[c][j + z] * inv;
                        const unsigned w0 = kv8_pack4(y[0], y[1], y[2], y[3]);
                        const f32x2 lo = __builtin_amdgcn_cvt_pk_f32_fp8(w0, false);
                        const f32x2 hi = __builtin_amdgcn_cvt_pk_f32_fp8(w0, true);
                        const unsigned w1 = kv8_pack4((y[0] - lo[0]) * 16.f, (y[1] - lo[1]) * 16.f,
                                                      (y[2] - hi[0]) * 16.f, (y[3] - hi[1]) * 16.f);
                        q8[qt][0][4 * c + j / 4] = (int)w0;
                        q8[qt][QP - 1][4 * (QP == 2 ? c : 1) + j / 4] = (int)w1;
                    }
            } else {
#pragma unroll
                for (int s = 0; s < HD / 32; ++s) {
                    const T* const at = src + (s >> 1) * 64 + g * 16 + (s & 1) * 8;
                    if constexpr (NP == 1) {
                        q[qt][0][s] = *reinterpret_cast<const bf16x8*>(at);
                    } else {
                        float x[8];
                        kv8_load<T, 8>(at, x);
#pragma unroll
                        for (int j = 0; j < 8; ++j) {
                            __bf16 p[NP];
                            kv8_split<NP>(x[j], p);
#pragma unroll
                            for (int y = 0; y < NP; ++y) q[qt][y][s][j] = p[y];
                        }
                    }
                }
            }
            mx[qt] = -INFINITY;
            sum[qt] = 0.f;
            if constexpr (WP == 1) ones[qt] = f32x4{0.f, 0.f, 0.f, 0.f};
#pragma unroll
            for (int d = 0; d < HD / 16; ++d) acc[qt][d] = f32x4{0.f, 0.f, 0.f, 0.f};
        }
        far = false;
        all = end = k_hi;
        if (w.a.causal) {
            all = min(all, t.len - t.m + min(wr0, t.rows - 1) / w.grp + 1);
            end = min(end, t.len - t.m + (min(wr0 + 16 * QT, t.rows) - 1) / w.grp + 1);
        }
        if (wr0 >= t.rows) end = 0;
    }

    // After the last step: sum[] is the rows' whole sum.  A row that sees keys
    // of the (sequence, KV head)'s part but whose scores are all -infinity gets
    // a finite maximum: its result, 0 over a sum of 0, is NaN, and not that of
    // a row that sees no key.  k_first: the wave's first key.
    EBRL_DEV void finish(const Kv8AttnKernelArgs& w, unsigned pair, int part, int k_first) {
        bool none = false;
#pragma unroll
        for (int qt = 0; qt < QT; ++qt) none |= mx[qt] == -INFINITY && k_first < lim[qt];
        if (__any(none)) {
            const int first = kv8_first_key(w, pair, part);
#pragma unroll
            for (int qt = 0; qt < QT; ++qt)
                if (first < lim[qt]) mx[qt] = fmaxf(mx[qt], -FLT_MAX);
        }
#pragma unroll
        for (int qt = 0; qt < QT; ++qt) {
            if constexpr (WP == 1) sum[qt] = ones[qt][0];
            else sum[qt] = attn_sum_xor16_32(sum[qt]);
        }
    }

    // P pages (an even number; 16 P keys from k0 on) in the lanes' order: kc, vc
    // their codes, ks, vs their scales, there: whether each is one.
    template <int P>
    EBRL_DEV void step(uint4 (&kc)[P][NC], uint4 (&vc)[P][NC], const float (&ks)[P], const float (&vs)[P],
                       const bool (&there)[P], int k0, int len, float scale_log2, int lane)
    {
        const int g = lane >> 4;
        // S^T = K Q^T
        f32x4 s[QT][P];
#pragma unroll
        for (int t = 0; t < P; ++t) {
#pragma unroll
            for (int qt = 0; qt < QT; ++qt) s[qt][t] = f32x4{0.f, 0.f, 0.f, 0.f};
            if constexpr (MX) {
                const i32x8 ka = {(int)kc[t][0].x, (int)kc[t][0].y, (int)kc[t][0].z, (int)kc[t][0].w,
                                  (int)kc[t][NC - 1].x, (int)kc[t][NC - 1].y, (int)kc[t][NC - 1].z, (int)kc[t][NC - 1].w};
                const int sk = (int)(__float_as_uint(ks[t]) >> 23);
#pragma unroll
                for (int p = QP - 1; p >= 0; --p)
#pragma unroll
                    for (int qt = 0; qt < QT; ++qt)
                        s[qt][t] = __builtin_amdgcn_mfma_scale_f32_16x16x128_f8f6f4(ka, q8[qt][p], s[qt][t], 0, 0, 0, sk, 0,
                                                                                    q8_scale[qt] - 4 * p);
                continue;
            }
#pragma unroll
            for (int c = 0; c < NC; ++c) {
                const bf16x8 ka = kv8_bf16(kc[t][c].x, kc[t][c].y, ks[t], ks[t]);
                const bf16x8 kb = kv8_bf16(kc[t][c].z, kc[t][c].w, ks[t], ks[t]);
#pragma unroll
                for (int p = NP - 1; p >= 0; --p)
#pragma unroll
                    for (int qt = 0; qt < QT; ++qt)
                        s[qt][t] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(ka, q[qt][p][MX ? 0 : 2 * c], s[qt][t], 0, 0, 0);
#pragma unroll
                for (int p = NP - 1; p >= 0; --p)
#pragma unroll
                    for (int qt = 0; qt < QT; ++qt)
                        s[qt][t] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(kb, q[qt][p][MX ? 0 : 2 * c + 1], s[qt][t], 0, 0, 0);
            }
        }
        // Codes of V that are NaN where not every row sees every key: a bit
        // each, pairs of pages apart.
        uint64_t nan_v[P / 2];
        bool all_there = true;
#pragma unroll
        for (int t = 0; t < P; ++t) {
            all_there &= there[t];
            if (t % 2) nan_v[t / 2] = 0;
        }
        bool nans = false;
        if (k0 + 16 * P > all || !all_there) {
            // some row does not see some key.  Slots past the last key may
            // hold anything: their weights are zero, and so have their
            // values to be.
            unsigned bad = 0;
#pragma unroll
            for (int t = 0; t < P; ++t) {
                const int left = there[t] ? len - (k0 + 16 * t + 4 * g) : 0;
                const unsigned ok = left >= 4 ? ~0u : left <= 0 ? 0u : (1u << (8 * left)) - 1;
#pragma unroll
                for (int c = 0; c < NC; ++c) {
                    unsigned* const x = reinterpret_cast<unsigned*>(&vc[t][c]);
#pragma unroll
                    for (int d = 0; d < 4; ++d) {
                        x[d] &= ok;
                        bad |= kv8_nan_bytes(x[d]);
                    }
                }
#pragma unroll
                for (int qt = 0; qt < QT; ++qt)
#pragma unroll
                    for (int v = 0; v < 4; ++v)
                        s[qt][t][v] = there[t] && k0 + 16 * t + 4 * g + v < lim[qt] ? s[qt][t][v] : -INFINITY;
            }
            nans = __any(bad != 0);
            if (nans) {
                // a NaN counts for the rows that see its key alone: the
                // product takes it as zero
#pragma unroll
                for (int t = 0; t < P; ++t)
#pragma unroll
                    for (int c = 0; c < NC; ++c) {
                        unsigned* const x = reinterpret_cast<unsigned*>(&vc[t][c]);
#pragma unroll
                        for (int d = 0; d < 4; ++d) {
                            const unsigned z = kv8_nan_bytes(x[d]) >> 7;
                            x[d] &= ~(z * 0xffu);
                            nan_v[t / 2] |= (uint64_t)(z * 0x01020408u >> 24 & 15u) << (4 * ((t % 2 * NC + c) * 4 + d));
                        }
                    }
            }
        }
        // Weights are 2^(x - mx), x = score log2(e) / sqrt(hd).  mx is a whole
        // number that follows the row's maximum: it moves when a weight would
        // pass 2^KV8_SLACK, and rescaling by a power of two is exact, so a
        // weight's last 32-bit place is all that the moves and the cut into
        // steps can change.
        bool move = false;
        float tm[QT];
#pragma unroll
        for (int qt = 0; qt < QT; ++qt) {
            tm[qt] = -INFINITY;
#pragma unroll
            for (int t = 0; t < P; ++t)
#pragma unroll
                for (int v = 0; v < 4; ++v) tm[qt] = fmaxf(tm[qt], s[qt][t][v]);
            move |= kv8_scaled(tm[qt], scale_log2, mx[qt]) > KV8_SLACK;
        }
        if (__any(move)) {
            far = false;
#pragma unroll
            for (int qt = 0; qt < QT; ++qt) {
                const float nm = fmaxf(mx[qt], ceilf(attn_max_xor16_32(tm[qt]) * scale_log2));
                const float alpha = mx[qt] == nm ? 1.f : ldexpf(1.0f, (int)fmaxf(mx[qt] - nm, -300.f));
                mx[qt] = nm;
                far |= fabsf(nm) >= KV8_FAR && nm != -INFINITY;
                if constexpr (WP == 1) ones[qt] *= alpha;
                else sum[qt] *= alpha;
#pragma unroll
                for (int d = 0; d < HD / 16; ++d) acc[qt][d] *= alpha;
            }
            far = __any(far);
        }
        // x - mx, for rows whose mx is far; the others' are what the fused form
        // below gives, which then takes them as they are
        if (far) {
#pragma unroll
            for (int qt = 0; qt < QT; ++qt) {
                const bool row_far = fabsf(mx[qt]) >= KV8_FAR;
                const float use = mx[qt] == -INFINITY ? 0.f : mx[qt];
#pragma unroll
                for (int t = 0; t < P; ++t)
#pragma unroll
                    for (int v = 0; v < 4; ++v)
                        s[qt][t][v] = row_far ? kv8_scaled(s[qt][t][v], scale_log2, use) : fmaf(s[qt][t][v], scale_log2, -use);
            }
        }
        const float by = far ? 1.f : scale_log2;
        // O^T += V^T P^T for a pair of pages: row r of product 4 c + d is dim
        // 64 c + 4 r + d, a lane's eight keys those that its scores are of
#pragma unroll
        for (int u = 0; u < P; u += 2) {
            bf16x8 pb[QT][WP];
#pragma unroll
            for (int qt = 0; qt < QT; ++qt) {
                const float use = far || mx[qt] == -INFINITY ? 0.f : mx[qt];
                float ps = 0.f;
#pragma unroll
                for (int t = 0; t < 2; ++t)
#pragma unroll
                    for (int v = 0; v < 4; ++v) {
                        const float p = fast_exp2(fmaf(s[qt][u + t][v], by, -use));
                        ps += p;
                        __bf16 o[WP];
                        kv8_split<WP>(p, o);
#pragma unroll
                        for (int y = 0; y < WP; ++y) pb[qt][y][4 * t + v] = o[y];
                    }
                if constexpr (WP == 1) {
                    const __bf16 e = (__bf16)1.f;
                    ones[qt] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(bf16x8{e, e, e, e, e, e, e, e}, pb[qt][0], ones[qt],
                                                                      0, 0, 0);
                } else {
                    sum[qt] += ps;
                }
            }
#pragma unroll
            for (int c = 0; c < NC; ++c) {
                const unsigned x0[4] = {vc[u][c].x, vc[u][c].y, vc[u][c].z, vc[u][c].w};
                const unsigned x1[4] = {vc[u + 1][c].x, vc[u + 1][c].y, vc[u + 1][c].z, vc[u + 1][c].w};
#pragma unroll
                for (int d = 0; d < 4; ++d) {
                    const bf16x8 va = kv8_bf16(x0[d], x1[d], vs[u], vs[u + 1]);
#pragma unroll
                    for (int p = WP - 1; p >= 0; --p)
#pragma unroll
                        for (int qt = 0; qt < QT; ++qt)
                            acc[qt][4 * c + d] =
                                __builtin_amdgcn_mfma_f32_16x16x32_bf16(va, pb[qt][p], acc[qt][4 * c + d], 0, 0, 0);
                }
            }
        }
        if (nans) {
            // how many NaNs of a dim each row sees
#pragma unroll
            for (int u = 0; u < P; u += 2)
#pragma unroll
                for (int qt = 0; qt < QT; ++qt) {
                    int below = lim[qt];
                    asm volatile("" : "+v"(below));   // keeps what follows in this rare branch
                    bf16x8 sees;
#pragma unroll
                    for (int j = 0; j < 8; ++j)
                        sees[j] = (__bf16)(k0 + 16 * (u + (j >> 2)) + 4 * g + (j & 3) < below ? 1.f : 0.f);
#pragma unroll
                    for (int x = 0; x < 4 * NC; ++x) {
                        bf16x8 isnan;
#pragma unroll
                        for (int j = 0; j < 8; ++j)
                            isnan[j] = (__bf16)((nan_v[u / 2] >> (4 * ((j >> 2) * NC * 4 + x) + (j & 3)) & 1) ? 1.f : 0.f);
                        const f32x4 n =
                            __builtin_amdgcn_mfma_f32_16x16x32_bf16(isnan, sees, f32x4{0.f, 0.f, 0.f, 0.f}, 0, 0, 0);
#pragma unroll
                        for (int v = 0; v < 4; ++v)
                            if (n[v] > 0.f) acc[qt][x][v] = __uint_as_float(0x7fc00000u);
                    }
                }
        }
    }
};

// Where (token, head) row `row` of a sequence's output lies.
template <typename T, int HD>
EBRL_DEV T* kv8_out(const Kv8AttnKernelArgs& w, const Kv8Tile& t, int kvh, int row) {
    const int tok = row / w.grp;
    return (T*)w.a.out + (size_t)(t.r0 + tok) * w.a.ldo + (size_t)(kvh * w.grp + (row - tok * w.grp)) * HD;
}

// A row's state: the result if its keys are in one part, else that part (the
// `to`-th of the workspace).  Lane group g has dims 64 c + 16 g .. + 15.
template <typename T, int HD>
EBRL_DEV void kv8_store(const Kv8AttnKernelArgs& w, const f32x4 (&acc)[HD / 16], float mx, float sum, int parts, T* out,
                        size_t to, int g)
{
    const float inv = parts > 1 ? 1.f : kv8_inverse(mx, sum);
#pragma unroll
    for (int c = 0; c < HD / 64; ++c)
#pragma unroll
        for (int v = 0; v < 4; ++v) {
            const int d = 64 * c + 16 * g + 4 * v;
            const f32x4 o = {acc[4 * c][v] * inv, acc[4 * c + 1][v] * inv, acc[4 * c + 2][v] * inv, acc[4 * c + 3][v] * inv};
            if (parts == 1) st4<T>(out + d, o[0], o[1], o[2], o[3]);
            else *reinterpret_cast<f32x4*>(w.part_o + to * HD + d) = o;
        }
    if (parts > 1 && g == 0) { w.part_ml[2 * to] = mx; w.part_ml[2 * to + 1] = sum; }
}

// 16 bytes that are read once: marked non-temporal.
EBRL_DEV uint4 kv8_stream16(const uint8_t* p) {
    return __builtin_bit_cast(uint4, __builtin_nontemporal_load(reinterpret_cast<const u32x4*>(p)));
}

// One query row a sequence, or few: KW waves share a (sequence, KV head)'s
// rows, at most 16, and deal the pairs of pages of a part of the keys.  Bound
// by the bytes of the cache: codes go straight to registers, and a step's
// registers are loaded again as soon as it is done, so that each wave keeps
// 8 to 16 KB in flight (head dim 128).  95 us, 5.6 TB/s, on 61 sequences of 500
// to 8000 keys (8 KV heads of 128), where a streaming read reaches 7.1; one
// sequence of 291 keys 6 us, the latency of lengths, pages and codes in turn.
template <typename T, int HD, int KW>
__global__ __launch_bounds__(256, 2) void kv8_decode_kernel(Kv8AttnKernelArgs w)
{
    constexpr int NC = HD / 64;
    constexpr int STEP = 32 * KW;              // keys that the waves take at a time
    __shared__ __attribute__((aligned(16))) float s_o[KW > 1 ? KW : 1][KW > 1 ? 16 : 1][KW > 1 ? HD + 4 : 4];
    __shared__ float s_m[KW][16], s_l[KW][16];

    const int hkv = w.c.kv_heads;
    const int tid = threadIdx.x, lane = tid & 63;
    const int wave = __builtin_amdgcn_readfirstlane(tid >> 6);
    const int r = lane & 15, g = lane >> 4;
    const int kw = KW > 1 ? wave : 0;
    const unsigned units = (unsigned)w.a.n * hkv, id = KW > 1 ? blockIdx.x : blockIdx.x * 4 + wave;
    const int part = id / units;
    const unsigned unit = id % units;
    if (part >= w.parts) return;
    const int kvh = unit % hkv, i = unit / hkv;
    // 32 steps of this wave at a time: lane 2 s + t has page t of step s.  The
    // first pages are asked for before the lengths are known.
    constexpr int BATCH = 32;
    const int k_lo = part * w.part_keys;
    const int p_at = (lane >> 1) * (STEP / KV8_PAGE) + kw * 2 + (lane & 1);
    const int trow = kv8_table_row(w, i);
    const int* const table = w.c.block_table + (size_t)max(trow, 0) * w.c.table_stride;
    int page = k_lo / KV8_PAGE + p_at < w.c.table_stride ? table[k_lo / KV8_PAGE + p_at] : -1;
    const Kv8Tile t = kv8_tile(w, i, 0);
    if (t.rows == 0 || part >= t.parts) return;
    const int k_hi = min(t.end, k_lo + w.part_keys);

    const size_t gb = (size_t)KV8_PAGE * HD;   // bytes of a (page, K or V, head) group
    const uint8_t* const codes = (const uint8_t*)w.c.codes + kvh * gb;
    const int k_at = r * 64 + g * 16, v_at = lane * 16;
    Kv8Rows<T, HD, 1, false, sizeof(T) == 4 ? 3 : 2> rows;
    const int p_hi = (k_hi + KV8_PAGE - 1) / KV8_PAGE;
    rows.init(w, t, kvh, 0, k_hi, lane);
    for (int kb = k_lo; kb < k_hi; kb += BATCH * STEP) {
        const int at = kb / KV8_PAGE + p_at;
        if (kb > k_lo) page = at < p_hi ? table[at] : -1;
        if (at >= p_hi || page >= w.c.num_blocks) page = -1;
        float ksv = 1.f, vsv = 1.f;
        if (page >= 0) {
            ksv = w.c.scales[(size_t)page * 2 * hkv + kvh];
            vsv = w.c.scales[((size_t)page * 2 + 1) * hkv + kvh];
        }
        const int n = (k_hi - kb - kw * 32 + STEP - 1) / STEP;
        const int steps = min(max(n, 0), BATCH);
        auto load = [&](int s, uint4 (&kc)[2][NC], uint4 (&vc)[2][NC]) {
#pragma unroll
            for (int x = 0; x < 2; ++x) {
                // a page that is none: page 0's codes, not used
                const int pg = max(2 * s + x < 64 ? __builtin_amdgcn_readlane(page, 2 * s + x) : 0, 0);
                const uint8_t* kp = codes + (size_t)pg * 2 * hkv * gb;
                const uint8_t* vp = kp + (size_t)hkv * gb;
#pragma unroll
                for (int c = 0; c < NC; ++c) {
                    kc[x][c] = kv8_stream16(kp + 1024 * c + k_at);
                    vc[x][c] = kv8_stream16(vp + 1024 * c + v_at);
                }
            }
        };
        auto work = [&](int s, uint4 (&kc)[2][NC], uint4 (&vc)[2][NC]) {
            float ks[2], vs[2];
            bool there[2];
#pragma unroll
            for (int x = 0; x < 2; ++x) {
                there[x] = __builtin_amdgcn_readlane(page, 2 * s + x) >= 0;
                ks[x] = readlane_f(ksv, 2 * s + x);
                vs[x] = readlane_f(vsv, 2 * s + x);
            }
            rows.step(kc, vc, ks, vs, there, kb + s * STEP + kw * 32, t.len, w.scale_log2, lane);
        };
        if (steps <= 0) continue;
        uint4 ka[2][NC], va[2][NC], kn[2][NC], vn[2][NC];
        load(0, ka, va);
        load(1, kn, vn);
        asm volatile("" :: "v"(ksv), "v"(vsv));   // waited for here, not on every turn of the loop
        // the loads are issued on every path, so that the waits leave the
        // other step's in flight
        for (int s = 0; s < steps; s += 2) {
            work(s, ka, va);
            load(s + 2, ka, va);
            if (s + 1 < steps) work(s + 1, kn, vn);
            load(s + 3, kn, vn);
        }
    }
    rows.finish(w, unit, part, k_lo + kw * 32);

    const size_t to0 = ((size_t)unit * w.parts + part) * 16;
    if constexpr (KW == 1) {
        if (r >= t.rows) return;
        kv8_store<T, HD>(w, rows.acc[0], rows.mx[0], rows.sum[0], t.parts, kv8_out<T, HD>(w, t, kvh, r), to0 + r, g);
    } else {
        // the waves join in their order
#pragma unroll
        for (int c = 0; c < NC; ++c)
#pragma unroll
            for (int v = 0; v < 4; ++v) {
                const f32x4 o = {rows.acc[0][4 * c][v], rows.acc[0][4 * c + 1][v], rows.acc[0][4 * c + 2][v],
                                 rows.acc[0][4 * c + 3][v]};
                *reinterpret_cast<f32x4*>(&s_o[wave][r][64 * c + 16 * g + 4 * v]) = o;
            }
        if (g == 0) { s_m[wave][r] = rows.mx[0]; s_l[wave][r] = rows.sum[0]; }
        __syncthreads();
        for (int x = tid; x < t.rows * (HD / 4); x += 256) {
            const int row = x / (HD / 4), d = x % (HD / 4) * 4;
            float M = -INFINITY, L = 0.f;
            f32x4 o = {0.f, 0.f, 0.f, 0.f};
#pragma unroll
            for (int y = 0; y < KW; ++y) M = fmaxf(M, s_m[y][row]);
#pragma unroll
            for (int y = 0; y < KW; ++y) {
                const float my = s_m[y][row];
                const float wt = my == -INFINITY ? 0.f : fast_exp2(my - M);
                L += wt * s_l[y][row];
                o += wt * *reinterpret_cast<const f32x4*>(&s_o[y][row][d]);
            }
            if (t.parts == 1) {
                const float inv = kv8_inverse(M, L);
                st4<T>(kv8_out<T, HD>(w, t, kvh, row) + d, o[0] * inv, o[1] * inv, o[2] * inv, o[3] * inv);
            } else {
                *reinterpret_cast<f32x4*>(w.part_o + (to0 + row) * HD + d) = o;
                if (d == 0) { w.part_ml[2 * (to0 + row)] = M; w.part_ml[2 * (to0 + row) + 1] = L; }
            }
        }
    }
}

// Many rows: the keys go through two LDS buffers, 64 at a time, that DMA fills
// with raw codes (16 KB a step at head dim 128) in the order in which a lane
// reads them back: 16 bytes a lane, one after the other.  A wave has 16 QT rows
// and takes P pages at a time; with KG 1 the four waves of a workgroup have
// rows of their own and take all keys, with KG 2 two waves share rows and take
// 32 keys of each step.  Bound by issue: with 32 rows a wave (QT 2, head dim 128,
// 2 x 4096 rows of 32 heads on 8 k keys) 710 to 760 us by card and clock, 1.06
// to 1.13 PFLOP/s; matrix instructions take 44 to 49 % of a SIMD's cycles and
// vector instructions 54 to 61 %, and they hardly overlap.  148 rows of 37 sequences on 730 keys 34 us, 480 TFLOP/s.
// At head dim 64 K's codes go to the scaled product with 32 rows a wave, held to
// 128 registers (2048 rows of 32 heads on 8 k keys, 168 us now, 172 against 179 with
// conversions; without the bound 167, but 4 x 2048 rows on themselves 93 against
// 90); with 16 rows preparing q and two registers more cost what it saves (24
// prompts of 200 to 424 tokens 20.8 us against 19.1).
template <typename T, int HD, int QT, int KG, int P>
__global__ __launch_bounds__(256, HD == 64 && QT == 2 ? 4 : 2) void kv8_prompt_kernel(Kv8AttnKernelArgs w)
{
    constexpr int NC = HD / 64;
    constexpr int RW = 16 * QT;
    constexpr int TR = RW * (4 / KG);
    constexpr int SEG = 256;                   // pages whose ids and scales LDS holds
    constexpr int GB = KV8_PAGE * HD;
    __shared__ __attribute__((aligned(1024))) uint8_t s_kv[2][4][2][GB];
    __shared__ __attribute__((aligned(16))) int s_page[SEG];
    __shared__ __attribute__((aligned(16))) float s_ks[SEG], s_vs[SEG];

    const int hkv = w.c.kv_heads;
    const int tid = threadIdx.x, lane = tid & 63;
    const int wave = __builtin_amdgcn_readfirstlane(tid >> 6);
    const int r = lane & 15, g = lane >> 4;
    // Workgroups go round-robin to the eight XCDs: a (sequence, KV head) keeps
    // to one, whose L2 then serves its tiles.  Tiles with the most work start
    // first: causal ones at the end of a sequence, others at its start.
    const unsigned heads = (unsigned)w.a.n * hkv;
    unsigned u, rest;
    if (heads % 8 == 0) {
        const unsigned per = heads / 8, j = blockIdx.x >> 3;
        u = (blockIdx.x & 7) * per + j % per;
        rest = j / per;
    } else {
        u = blockIdx.x % heads;
        rest = blockIdx.x / heads;
    }
    const int part = rest % w.parts;
    const int tile = w.a.causal ? w.tiles - 1 - (int)(rest / w.parts) : rest / w.parts;
    const int kvh = u % hkv, i = u / hkv;
    const unsigned unit = u * w.tiles + tile;
    const Kv8Tile t = kv8_tile(w, i, tile);
    if (t.t0 >= t.rows || part >= t.parts) return;
    const int k_lo = part * w.part_keys, k_hi = min(t.end, k_lo + w.part_keys);

    const int kg = KG == 1 ? 0 : wave & 1;
    const int wr0 = t.t0 + wave / KG * RW;
    Kv8Rows<T, HD, QT, sizeof(T) == 2 && (HD == 128 || QT == 2), sizeof(T) == 4 ? 3 : 1> rows;
    rows.init(w, t, kvh, wr0, k_hi, lane);

    const uint8_t* const codes = (const uint8_t*)w.c.codes + (size_t)kvh * GB;
    const uint32_t lds = (uint32_t)(uintptr_t)(attn_lds_ptr_t)&s_kv[0][0][0][0];
    const int k_at = r * 64 + g * 16, v_at = lane * 16;
    for (int seg = k_lo; seg < k_hi; seg += SEG * KV8_PAGE) {
        const int seg_hi = min(k_hi, seg + SEG * KV8_PAGE);
        const int n_pages = (seg_hi - seg + KV8_PAGE - 1) / KV8_PAGE, steps = (n_pages + 3) / 4;
        __syncthreads();                       // the segment before is done with the lists
        for (int x = tid; x < steps * 4; x += 256) {
            int page = x < n_pages ? t.table[seg / KV8_PAGE + x] : -1;
            if (page >= w.c.num_blocks) page = -1;
            s_page[x] = max(page, -1);
            s_ks[x] = page >= 0 ? w.c.scales[(size_t)page * 2 * hkv + kvh] : 1.f;
            s_vs[x] = page >= 0 ? w.c.scales[((size_t)page * 2 + 1) * hkv + kvh] : 1.f;
        }
        __syncthreads();
        auto dma = [&](int it, int buf) {
            // a page that is none: page 0's codes, not used
            const int pg = max(__builtin_amdgcn_readfirstlane(s_page[4 * it + wave]), 0);
            const uint8_t* kp = codes + (size_t)pg * 2 * hkv * GB;
            const uint8_t* vp = kp + (size_t)hkv * GB;
            const uint32_t to = __builtin_amdgcn_readfirstlane(lds + (buf * 4 + wave) * 2 * GB);
#pragma unroll
            for (int c = 0; c < NC; ++c) {
                attn_dma16(kp + 1024 * c + k_at, to + 1024 * c);
                attn_dma16(vp + 1024 * c + v_at, to + GB + 1024 * c);
            }
        };
        dma(0, 0);
        for (int it = 0; it < steps; ++it) {
            const int buf = it & 1;
            // this wave's part of step `it` has landed, then every wave's has
            // and every wave is done with the buffer that is filled next
            attn_wait_vmcnt<0>();
            __syncthreads();
            if (it + 1 < steps) dma(it + 1, buf ^ 1);
#pragma unroll
            for (int x = 0; x < 4 / KG; x += P) {
                const int p0 = kg * (4 / KG) + x, k0 = seg + it * 64 + 16 * p0;
                if (k0 >= rows.end) break;     // nothing that a row of this wave sees
                uint4 kc[P][NC], vc[P][NC];
                float ks[P], vs[P];
                bool there[P];
#pragma unroll
                for (int y = 0; y < P; ++y) {
#pragma unroll
                    for (int c = 0; c < NC; ++c) {
                        kc[y][c] = *reinterpret_cast<const uint4*>(&s_kv[buf][p0 + y][0][1024 * c + lane * 16]);
                        vc[y][c] = *reinterpret_cast<const uint4*>(&s_kv[buf][p0 + y][1][1024 * c + lane * 16]);
                    }
                    there[y] = __builtin_amdgcn_readfirstlane(s_page[4 * it + p0 + y]) >= 0;
                    ks[y] = s_ks[4 * it + p0 + y];
                    vs[y] = s_vs[4 * it + p0 + y];
                }
                rows.step(kc, vc, ks, vs, there, k0, t.len, w.scale_log2, lane);
            }
        }
    }
    rows.finish(w, u, part, k_lo + kg * 32);
    if constexpr (KG == 2) {
        // the second wave of a pair hands its state to the first, in the buffers
        constexpr int LD = HD + 4;
        static_assert(TR * (LD + 2) * 4 <= 2 * 4 * 2 * GB, "the states fit the buffers");
        float* const s_o = reinterpret_cast<float*>(&s_kv[0][0][0][0]);
        float* const s_ml = s_o + TR * LD;
        __syncthreads();
#pragma unroll
        for (int qt = 0; qt < QT; ++qt) {
            const int row = wave / 2 * RW + 16 * qt + r;
            if (kg == 1) {
#pragma unroll
                for (int c = 0; c < NC; ++c)
#pragma unroll
                    for (int v = 0; v < 4; ++v) {
                        const f32x4 o = {rows.acc[qt][4 * c][v], rows.acc[qt][4 * c + 1][v], rows.acc[qt][4 * c + 2][v],
                                         rows.acc[qt][4 * c + 3][v]};
                        *reinterpret_cast<f32x4*>(s_o + row * LD + 64 * c + 16 * g + 4 * v) = o;
                    }
                if (g == 0) { s_ml[2 * row] = rows.mx[qt]; s_ml[2 * row + 1] = rows.sum[qt]; }
            }
        }
        __syncthreads();
        if (kg == 1) return;
#pragma unroll
        for (int qt = 0; qt < QT; ++qt) {
            const int row = wave / 2 * RW + 16 * qt + r;
            const float m1 = s_ml[2 * row], M = fmaxf(rows.mx[qt], m1);
            const float w0 = rows.mx[qt] == -INFINITY ? 0.f : fast_exp2(rows.mx[qt] - M);
            const float w1 = m1 == -INFINITY ? 0.f : fast_exp2(m1 - M);
            rows.mx[qt] = M;
            rows.sum[qt] = w0 * rows.sum[qt] + w1 * s_ml[2 * row + 1];
#pragma unroll
            for (int c = 0; c < NC; ++c)
#pragma unroll
                for (int v = 0; v < 4; ++v) {
                    const f32x4 o = *reinterpret_cast<const f32x4*>(s_o + row * LD + 64 * c + 16 * g + 4 * v);
#pragma unroll
                    for (int d = 0; d < 4; ++d)
                        rows.acc[qt][4 * c + d][v] = w0 * rows.acc[qt][4 * c + d][v] + w1 * o[d];
                }
        }
    }
#pragma unroll
    for (int qt = 0; qt < QT; ++qt) {
        const int row = wr0 + 16 * qt + r;
        if (row >= t.rows) continue;
        kv8_store<T, HD>(w, rows.acc[qt], rows.mx[qt], rows.sum[qt], t.parts, kv8_out<T, HD>(w, t, kvh, row),
                         ((size_t)unit * w.parts + part) * TR + (row - t.t0), g);
    }
}

// Joins the parts of a row's keys, in their order: a wave a row, HD / 4 lanes
// across it and the others taking further parts.  Bound by latency: what it
// needs of the workspace is asked for before the sequence's lengths, which say
// how many parts there are, have come.  5 us for 61 x 8 pairs of two parts.
template <typename T, int HD>
__global__ __launch_bounds__(256) void kv8_join_kernel(Kv8AttnKernelArgs w)
{
    constexpr int LPR = HD / 4, PG = 64 / LPR, AHEAD = 2;
    __shared__ float s_w[4][KV8_MAX_PARTS];
    const int lane = threadIdx.x & 63;
    const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    const unsigned per = (w.join_rows + 3) / 4;
    const unsigned unit = blockIdx.x / per;
    const int row = (blockIdx.x % per) * 4 + wave;
    if (row >= w.join_rows) return;
    const size_t base = (size_t)unit * w.parts * w.tile_rows + row;
    auto ml = [&](int p) { return *reinterpret_cast<const float2*>(w.part_ml + 2 * (base + (size_t)p * w.tile_rows)); };
    const int d = lane % LPR * 4, p0 = lane / LPR;
    auto part = [&](int p) { return *reinterpret_cast<const f32x4*>(w.part_o + (base + (size_t)p * w.tile_rows) * HD + d); };
    const float2 first = ml(min(lane, w.parts - 1));
    f32x4 ahead[AHEAD];
#pragma unroll
    for (int k = 0; k < AHEAD; ++k) ahead[k] = part(min(p0 + k * PG, w.parts - 1));
    unsigned id = unit;
    const int tile = id % w.tiles;
    id /= w.tiles;
    const int kvh = id % w.c.kv_heads, i = id / w.c.kv_heads;
    const Kv8Tile t = kv8_tile(w, i, tile);
    if (t.parts == 1 || t.t0 + row >= t.rows) return;
    float m = lane < t.parts ? first.x : -INFINITY;
    for (int p = lane + 64; p < t.parts; p += 64) m = fmaxf(m, ml(p).x);
    const float M = wave_max(m);
    float l = 0.f;
    for (int p = lane; p < t.parts; p += 64) {
        const float2 y = p == lane ? first : ml(p);
        const float wt = y.x == -INFINITY ? 0.f : fast_exp2(y.x - M);
        s_w[wave][p] = wt;
        l += wt * y.y;
    }
    const float L = wave_sum(l);
    asm volatile("s_waitcnt lgkmcnt(0)" ::: "memory");   // the wave's own s_w
    f32x4 o = {0.f, 0.f, 0.f, 0.f};
#pragma unroll
    for (int k = 0; k < AHEAD; ++k)
        if (p0 + k * PG < t.parts) o += s_w[wave][p0 + k * PG] * ahead[k];
#pragma unroll 4
    for (int p = p0 + AHEAD * PG; p < t.parts; p += PG) o += s_w[wave][p] * part(p);
#pragma unroll
    for (int v = 0; v < 4; ++v) {
        if (PG == 4) o[v] += swz_xor16_f(o[v]);
        o[v] += __shfl_xor(o[v], 32, 64);
    }
    const float inv = kv8_inverse(M, L);
    if (lane < LPR) st4<T>(kv8_out<T, HD>(w, t, kvh, t.t0 + row) + d, o[0] * inv, o[1] * inv, o[2] * inv, o[3] * inv);
}

// ------------------------------------------------------- plans, launches --

// `n`: the sequences that the cut is made for (a policy's calls take its
// largest batch, so that a sequence's bits do not depend on the call's).
static Kv8Plan kv8_plan(const ebrl_kv8_cache& c, const ebrl_kv8_attn_args& a, int n) {
    Kv8Plan p;
    const int64_t rows = (int64_t)a.max_q_len * (a.q_heads / c.kv_heads), pairs = (int64_t)n * c.kv_heads;
    auto groups = [&](int tile_rows) { return pairs * ((rows + tile_rows - 1) / tile_rows); };
    if (rows <= 16) {
        // A wave of its own for each (sequence, KV head) saves the joining of
        // four, and pays where keys are few and waves many: 1024 pairs of
        // 300 keys 20 us against 25, 4096 of 600 99.5 against 104.5; 256 of
        // 600 16.6 against 15.0, 512 of up to 2048 43 against 31.
        p.kind = pairs >= 1024 && a.max_kv_len <= 1024 ? KV8_WAVE : KV8_GROUP;
        p.tile_rows = 16;
    } else if (a.dtype == EBRL_DTYPE_BF16 && groups(128) >= 512 && a.max_kv_len >= 1024) {
        // 32 rows a wave halve the conversions of codes, and pay once they
        // fill the chip twice over and keys are many: 2 x 4 k rows of 32 heads
        // on 8 k keys 726 us against 811 with 16 rows a wave, 2048 rows on
        // 8 k keys 232 against 258, 4 x 2048 rows on themselves 156 against
        // 168; as good where 4 x 1024 rows meet 1024 keys (51 against 50) or
        // 32 x 37 rows 2037 (72 against 71); 128 x 37 rows on 748 keys 118
        // against 115, 96 x 48 on 288 keys 56 against 48.
        p.kind = KV8_TALL;
        p.tile_rows = 128;
    } else if (groups(64) >= 512) {
        p.kind = KV8_ROWS;
        p.tile_rows = 64;
    } else {
        // few workgroups: twice as many of half the rows, two waves sharing
        // them (600 rows of 32 heads on 600 keys 17 us against 29, 512 rows
        // of 4 heads each on 1512 keys 22.4 against 33; 37 sequences of 148
        // rows on 730 keys, 888 workgroups of 64 rows, 37 against 34; 64
        // sequences of them 75 against 58)
        p.kind = KV8_PAIRS;
        p.tile_rows = 32;
    }
    p.tiles = (int)((rows + p.tile_rows - 1) / p.tile_rows);
    // Keys are cut where that brings the workgroups to the 768 that the chip
    // holds at a time (three a CU), but not below 512 keys a part: three
    // sequences of 50000 to 131000 keys, 24 pairs, in 32 parts 108 us, in 42
    // 109, in 96 113; 512 pairs of 4096 keys in one part 87, in two 94.
    const int64_t units = pairs * p.tiles;
    int64_t want = p.kind == KV8_WAVE ? 1 : (768 + units / 2 - 1) / units;
    want = std::max<int64_t>(1, std::min<int64_t>({want, KV8_MAX_PARTS, ((int64_t)a.max_kv_len + 511) / 512}));
    const int step = p.kind == KV8_GROUP ? 128 : 64;   // keys that a workgroup takes at a time
    const int64_t keys = ((int64_t)a.max_kv_len + want - 1) / want;
    p.part_keys = (int)std::max<int64_t>(step, (keys + step - 1) / step * step);
    p.parts = (int)std::max<int64_t>(1, ((int64_t)a.max_kv_len + p.part_keys - 1) / p.part_keys);
    return p;
}

constexpr int64_t KV8_MAX_GROUPS = 1 << 23;   // workgroups of 256 threads in a launch: under 2^32 threads
constexpr int KV8_MAX_HEADS = 1 << 20;        // a row's elements are counted in 32 bits

static bool kv8_cache_ok(const ebrl_kv8_cache* c) {
    return c && c->num_blocks >= 1 && c->table_rows >= 1 && c->table_stride >= 1 && c->table_stride < (1 << 27) &&
           c->kv_heads >= 1 && c->kv_heads <= KV8_MAX_HEADS && (c->head_dim == 64 || c->head_dim == 128);
}
static bool kv8_pointers_ok(const ebrl_kv8_cache* c) {
    return c->codes && c->scales && c->block_table && (uintptr_t)c->codes % 16 == 0 && (uintptr_t)c->scales % 4 == 0 &&
           (uintptr_t)c->block_table % 4 == 0;
}
// Rows of `width` elements every `ld`, 16-byte aligned.
static bool kv8_rows_ok(const void* p, int64_t ld, int64_t width, int esz) {
    return p && (uintptr_t)p % 16 == 0 && ld >= width && ld * esz % 16 == 0 && ld < ((int64_t)1 << 40);
}

static bool kv8_attn_shape_ok(const ebrl_kv8_cache* c, const ebrl_kv8_attn_args* a) {
    return kv8_cache_ok(c) && a && (a->dtype == EBRL_DTYPE_BF16 || a->dtype == EBRL_DTYPE_FP32) && a->n >= 0 &&
           a->rows >= 0 && a->max_q_len >= 0 && a->max_kv_len >= 0 &&
           a->max_kv_len <= (1 << 30) && a->q_heads >= 1 && a->q_heads <= KV8_MAX_HEADS &&
           a->q_heads % c->kv_heads == 0 &&
           (int64_t)a->max_q_len * (a->q_heads / c->kv_heads) < (1 << 30);
}

// Whether a cut for n sequences can be counted: a workgroup, at least, for each
// (sequence, KV head), in 64 bits with their tiles and parts.
static bool kv8_pairs_ok(const ebrl_kv8_cache& c, int n) { return (int64_t)n * c.kv_heads <= KV8_MAX_GROUPS; }

template <typename T, int HD>
static void kv8_write_launch(bool token, const Kv8WriteKernelArgs& w, unsigned groups, hipStream_t s) {
    if (token) hipLaunchKernelGGL((kv8_write_token_kernel<T, HD>), dim3(groups), dim3(256), 0, s, w);
    else hipLaunchKernelGGL((kv8_write_kernel<T, HD>), dim3(groups), dim3(256), 0, s, w);
}

template <typename T, int HD>
static void kv8_attn_launch(const Kv8Plan& p, const Kv8AttnKernelArgs& w, int64_t units, hipStream_t s) {
    const dim3 grid((unsigned)(units * p.parts)), wg(256);
    switch (p.kind) {
    case KV8_WAVE:
        hipLaunchKernelGGL((kv8_decode_kernel<T, HD, 1>), dim3((unsigned)((units + 3) / 4)), wg, 0, s, w);
        break;
    case KV8_GROUP: hipLaunchKernelGGL((kv8_decode_kernel<T, HD, 4>), grid, wg, 0, s, w); break;
    case KV8_PAIRS: hipLaunchKernelGGL((kv8_prompt_kernel<T, HD, 1, 2, 2>), grid, wg, 0, s, w); break;
    case KV8_ROWS: hipLaunchKernelGGL((kv8_prompt_kernel<T, HD, 1, 1, 2>), grid, wg, 0, s, w); break;
    case KV8_TALL:
        if constexpr (sizeof(T) == 2)
            hipLaunchKernelGGL((kv8_prompt_kernel<T, HD, 2, 1, HD / 32>), grid, wg, 0, s, w);
        break;
    }
    if (p.parts > 1)
        hipLaunchKernelGGL((kv8_join_kernel<T, HD>), dim3((unsigned)(units * ((w.join_rows + 3) / 4))), wg, 0, s, w);
}

int kv8_write(const ebrl_kv8_cache* cache, const ebrl_kv8_write_args* args, hipStream_t s) {
    if (!kv8_cache_ok(cache) || !args) return EBRL_E_INVALID;
    const ebrl_kv8_write_args& a = *args;
    const int hd = cache->head_dim, hkv = cache->kv_heads;
    if ((a.dtype != EBRL_DTYPE_BF16 && a.dtype != EBRL_DTYPE_FP32) || a.n < 0 || a.rows < 0 || a.max_len < 0 ||
        a.q_heads < 0 || a.q_heads > KV8_MAX_HEADS || a.n_axes < 0 || a.n_axes > 3 || (a.q_heads > 0 && a.n_axes == 0))
        return EBRL_E_INVALID;
    int sum = 0;
    for (int x = 0; x < a.n_axes; ++x) {
        if (a.sections[x] < 1 || a.sections[x] > hd / 2) return EBRL_E_INVALID;
        sum += a.sections[x];
    }
    if (a.n_axes && (sum != hd / 2 || a.tab_rows < 1 || !a.cos_tab || !a.sin_tab || (uintptr_t)a.cos_tab % 16 ||
                     (uintptr_t)a.sin_tab % 16 || (a.n_axes > 1 && !a.axis_pos)))
        return EBRL_E_INVALID;
    if (a.n == 0 || a.rows == 0 || a.max_len == 0) return EBRL_OK;
    const int esz = a.dtype == EBRL_DTYPE_FP32 ? 4 : 2;
    if (!kv8_pointers_ok(cache) || !a.row_start || !a.pos0 || !kv8_rows_ok(a.k, a.ldk, (int64_t)hkv * hd, esz) ||
        !kv8_rows_ok(a.v, a.ldv, (int64_t)hkv * hd, esz))
        return EBRL_E_INVALID;
    if (a.q_heads && (!kv8_rows_ok(a.q, a.ldq, (int64_t)a.q_heads * hd, esz) ||
                      !kv8_rows_ok(a.q_out, a.ldq_out, (int64_t)a.q_heads * hd, esz) ||
                      (a.q == a.q_out && a.ldq != a.ldq_out)))
        return EBRL_E_INVALID;
    Kv8WriteKernelArgs w;
    w.c = *cache;
    w.a = a;
    const bool token = a.max_len == 1;
    const int64_t len = std::min<int64_t>(a.max_len, a.rows);
    w.pages = token ? 1 : (int)((len + 2 * KV8_PAGE - 2) / KV8_PAGE);
    const int64_t sp = (int64_t)a.n * w.pages;
    if (sp > 4 * KV8_MAX_GROUPS) return EBRL_E_INVALID;   // a wave each, at least
    // one head a wave up to some 16 waves a SIMD; from there on, four heads a
    // wave share their cosines and sines (9 sequences of 3001 to 4095 tokens,
    // 40 + 8 heads of 128: 182 us with one, 148 with two, 141 with four, 145
    // with eight; 16 of 600 tokens, 24 + 8 heads: 43, 36.5, 37, 36.5)
    w.per_wave = token ? 1024 / hd : sp * (a.q_heads + 2 * hkv) > 16384 ? 4 : 1;
    w.rot_units = (a.q_heads + hkv + w.per_wave - 1) / w.per_wave;
    w.v_units = (hkv + w.per_wave - 1) / w.per_wave;
    const int64_t groups = (sp * (w.rot_units + w.v_units) + 3) / 4;
    if (groups > KV8_MAX_GROUPS) return EBRL_E_INVALID;
    if (esz == 2) {
        if (hd == 64) kv8_write_launch<bf16_t, 64>(token, w, (unsigned)groups, s);
        else kv8_write_launch<bf16_t, 128>(token, w, (unsigned)groups, s);
    } else {
        if (hd == 64) kv8_write_launch<float, 64>(token, w, (unsigned)groups, s);
        else kv8_write_launch<float, 128>(token, w, (unsigned)groups, s);
    }
    return hipGetLastError() == hipSuccess ? EBRL_OK : EBRL_E_HIP;
}

static int64_t kv8_plan_bytes(const Kv8Plan& p, const ebrl_kv8_cache& c, int n) {
    return p.parts == 1 ? 0 : (int64_t)n * c.kv_heads * p.tiles * p.parts * p.tile_rows * (c.head_dim + 2) * 4;
}

int64_t kv8_attn_workspace(const ebrl_kv8_cache* cache, const ebrl_kv8_attn_args* args, int plan_n) {
    if (!kv8_attn_shape_ok(cache, args)) return EBRL_E_INVALID;
    if (args->n == 0 || args->max_q_len == 0) return 0;
    if (!kv8_pairs_ok(*cache, std::max(args->n, plan_n))) return EBRL_E_INVALID;
    return kv8_plan_bytes(kv8_plan(*cache, *args, plan_n), *cache, args->n);
}

int kv8_attn(const ebrl_kv8_cache* cache, const ebrl_kv8_attn_args* args, int plan_n, hipStream_t s) {
    if (!kv8_attn_shape_ok(cache, args) || !(args->scale > 0.f) || !isfinite(args->scale * 1.4426950408889634f))
        return EBRL_E_INVALID;
    const ebrl_kv8_attn_args& a = *args;
    if (a.n == 0 || a.rows == 0 || a.max_q_len == 0) return EBRL_OK;
    const int hd = cache->head_dim, esz = a.dtype == EBRL_DTYPE_FP32 ? 4 : 2;
    const int64_t width = (int64_t)a.q_heads * hd;
    if (!kv8_pointers_ok(cache) || !a.row_start || !a.kv_len || !kv8_rows_ok(a.q, a.ldq, width, esz) ||
        !kv8_rows_ok(a.out, a.ldo, width, esz) || a.q == a.out)
        return EBRL_E_INVALID;
    if (!kv8_pairs_ok(*cache, std::max(a.n, plan_n))) return EBRL_E_INVALID;
    const Kv8Plan p = kv8_plan(*cache, a, plan_n);
    const int64_t need = kv8_plan_bytes(p, *cache, a.n);
    if (need > 0 && (!a.workspace || a.workspace_bytes < need || (uintptr_t)a.workspace % 16)) return EBRL_E_INVALID;
    const int64_t units = (int64_t)a.n * cache->kv_heads * p.tiles;
    // (the join's are fewer: there is one only below some 768 units)
    if (units * p.parts > KV8_MAX_GROUPS) return EBRL_E_INVALID;
    Kv8AttnKernelArgs w;
    w.c = *cache;
    w.a = a;
    w.grp = a.q_heads / cache->kv_heads;
    w.tiles = p.tiles;
    w.tile_rows = p.tile_rows;
    w.parts = p.parts;
    w.part_keys = p.part_keys;
    w.join_rows = (int)std::min<int64_t>(p.tile_rows, (int64_t)a.max_q_len * w.grp);
    w.scale_log2 = a.scale * 1.4426950408889634f;
    w.part_o = (float*)a.workspace;
    w.part_ml = need ? w.part_o + units * p.parts * p.tile_rows * hd : nullptr;
    if (esz == 2) {
        if (hd == 64) kv8_attn_launch<bf16_t, 64>(p, w, units, s);
        else kv8_attn_launch<bf16_t, 128>(p, w, units, s);
    } else {
        if (hd == 64) kv8_attn_launch<float, 64>(p, w, units, s);
        else kv8_attn_launch<float, 128>(p, w, units, s);
    }
    return hipGetLastError() == hipSuccess ? EBRL_OK : EBRL_E_HIP;
}

// Pages of one layer after another: the codes and scales of page pairs[i].x
// go to page pairs[i].y (negative: nothing is copied).  A workgroup a (K or V,
// head) group: a denoise call copies before each step, with few environments
// too (4 layers of 8 heads of 128: 4 environments 4.8 us, 64 6.4 us; with a
// workgroup a page 5.6 and 7.6).
__global__ __launch_bounds__(128) void kv8_copy_kernel(uint8_t* codes, float* scales, int num_blocks, int groups,
                                                       int group_bytes, const int2* pairs)
{
    const int2 p = pairs[blockIdx.x / groups];
    if (p.x < 0 || p.y < 0 || p.x >= num_blocks || p.y >= num_blocks) return;
    const size_t layer = (size_t)blockIdx.y * num_blocks, group = blockIdx.x % groups;
    const size_t from = (layer + p.x) * groups + group, to = (layer + p.y) * groups + group;
    const uint4* src = reinterpret_cast<const uint4*>(codes + from * group_bytes);
    uint4* dst = reinterpret_cast<uint4*>(codes + to * group_bytes);
    for (int i = threadIdx.x; i < group_bytes / 16; i += 128) dst[i] = src[i];
    if (threadIdx.x == 0) scales[to] = scales[from];
}
void kv8_copy_pages(const ebrl_kv8_cache& c, int layers, const int2* pairs, int n, hipStream_t s) {
    if (n <= 0) return;
    const int groups = 2 * c.kv_heads;
    hipLaunchKernelGGL(kv8_copy_kernel, dim3((unsigned)n * groups, layers), dim3(128), 0, s, (uint8_t*)c.codes, c.scales,
                       c.num_blocks, groups, KV8_PAGE * c.head_dim, pairs);
}

// Value of an e4m3 code, on the host.
static float kv8_code_value(unsigned c) {
    const int e = c >> 3 & 15, m = c & 7;
    const float v = e == 15 && m == 7 ? NAN : e ? ldexpf(1.f + m / 8.f, e - 7) : ldexpf(m / 8.f, -6);
    return c & 128 ? -v : v;
}
void kv8_group_values(const uint8_t* codes, float scale, bool value, int head_dim, int slot, float* out) {
    for (int d = 0; d < head_dim; ++d) {
        const int at = 1024 * (d / 64) + (value ? 256 * (slot / 4) + 16 * (d % 64 / 4) + 4 * (d % 4) + slot % 4
                                                : 64 * slot + d % 64);
        out[d] = kv8_code_value(codes[at]) * scale;
    }
}

}  // namespace ebrl

extern "C" {

int ebrl_op_kv8_write(const ebrl_kv8_cache* cache, const ebrl_kv8_write_args* args, void* stream) {
    return ebrl::kv8_write(cache, args, (hipStream_t)stream);
}

int64_t ebrl_op_kv8_attn_workspace(const ebrl_kv8_cache* cache, const ebrl_kv8_attn_args* args) {
    return args ? ebrl::kv8_attn_workspace(cache, args, args->n) : EBRL_E_INVALID;
}

int ebrl_op_kv8_attn(const ebrl_kv8_cache* cache, const ebrl_kv8_attn_args* args, void* stream) {
    return args ? ebrl::kv8_attn(cache, args, args->n, (hipStream_t)stream) : EBRL_E_INVALID;
}

}  // extern "C"

// The paged KV cache in 8 bits (include/ebrl_kv8.h): rotary positions and
// cache write, and attention over the cache.
//
// kv8_write_kernel: a wave takes the new tokens of one page and a run of
//   heads; all of a (page, head)'s values meet in one wave, which has their
//   maximum, and so the scale, in registers before it stores a code.
// kv8_attn_kernel: a wave holds 16 QT query rows (a row is a token and a head
//   of the KV head's group) and walks the keys 32 (two pages) at a time.
//   Codes go from memory to the lanes in the order in which
//   v_mfma_f32_16x16x32_bf16 takes them and become bf16 by
//   v_cvt_scalef32_pk_bf16_fp8, which applies the page's scale: four
//   significant bits and a power of two, so exact.
#include <math.h>

#include "../../include/ebrl.h"
#include "../../include/ebrl_kv8.h"
#include "kernels.h"

namespace ebrl {

typedef __bf16 bf16x2 __attribute__((ext_vector_type(2)));
typedef float f32x2 __attribute__((ext_vector_type(2)));

constexpr int KV8_PAGE = EBRL_KV8_PAGE;
constexpr int KV8_EXP_MIN = -100, KV8_EXP_MAX = 120;   // 448 * 2^120 > FLT_MAX

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
// Least e >= KV8_EXP_MIN with a <= 448 * 2^e = 1.75 * 2^(8 + e); a >= 0, finite.
EBRL_DEV int kv8_exponent(float a) {
    const unsigned u = __float_as_uint(a);
    return max((int)(u >> 23) - 127 - ((u & 0x7fffffu) <= 0x600000u ? 8 : 7), KV8_EXP_MIN);
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
// Eight results of 64 bits, each rounded once.
EBRL_DEV void kv8_store8(float* p, const double* y) {
    *reinterpret_cast<float4*>(p) = make_float4((float)y[0], (float)y[1], (float)y[2], (float)y[3]);
    *reinterpret_cast<float4*>(p + 4) = make_float4((float)y[4], (float)y[5], (float)y[6], (float)y[7]);
}
EBRL_DEV void kv8_store8(bf16_t* p, const double* y) {
    bf16x8 o;
#pragma unroll
    for (int i = 0; i < 8; ++i) o[i] = (__bf16)kv8_odd(y[i]);
    *reinterpret_cast<bf16x8*>(p) = o;
}

struct Kv8WriteKernelArgs {
    ebrl_kv8_cache c;
    ebrl_kv8_write_args a;
    int pages;        // most pages of a sequence that a call touches
    int per_wave;     // heads that a wave takes in turn
    int rot_units, v_units;   // waves of a (sequence, page): for the Q and K heads, for the V heads
};

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
    if (i >= a.n) return;

    // the new tokens of this page: slots s0 .. s1 - 1, rows row0 ..
    const int trow = a.seq ? a.seq[i] : i;
    const int r0 = min(max(a.row_start[i], 0), a.rows);
    const int len = min(min(a.row_start[i + 1], a.rows) - r0, a.max_len);
    const int p0 = a.pos0[i];
    if (trow < 0 || trow >= w.c.table_rows || len <= 0 || p0 < 0 || p0 >= w.c.table_stride * KV8_PAGE) return;
    const int page_at = p0 / KV8_PAGE + pg;
    if (page_at >= w.c.table_stride) return;
    const int first = page_at * KV8_PAGE - p0;             // token of slot 0, counted from the first new one
    const int s0 = max(-first, 0), s1 = min(KV8_PAGE, len - first);
    if (s1 <= s0) return;
    const int page = w.c.block_table[(size_t)trow * w.c.table_stride + page_at];
    const bool there = page >= 0 && page < w.c.num_blocks;
    const int hkv = w.c.kv_heads;
    uint8_t* const codes = (uint8_t*)w.c.codes;

    if (unit < w.rot_units) {
        // Q and K heads: lane (t, g) has slot t's pairs PL g .. PL g + PL - 1
        const int t = lane >> 2, g = lane & 3;
        const bool mine = t >= s0 && t < s1;
        const int row = r0 + first + (mine ? t : s0);
        float cs[PL], sn[PL];
        if (a.n_axes) {
            const int* ap = a.axis_pos ? a.axis_pos + (size_t)row * a.n_axes : nullptr;
            const int b1 = a.sections[0], b2 = b1 + (a.n_axes > 1 ? a.sections[1] : 0);
            int pos[3];
            pos[0] = ap ? ap[0] : p0 + (row - r0);
            pos[1] = a.n_axes > 1 ? ap[1] : 0;
            pos[2] = a.n_axes > 2 ? ap[2] : 0;
            size_t base[3];
#pragma unroll
            for (int x = 0; x < 3; ++x) base[x] = (size_t)min(max(pos[x], 0), a.tab_rows - 1) * HALF;
#pragma unroll
            for (int q = 0; q < PL; q += 4) {
                const int at = PL * g + q;
                auto axis = [&](int pair) { return pair < b1 ? 0 : pair < b2 ? 1 : 2; };
                if (axis(at) == axis(at + 3)) {
                    const int x = axis(at);
                    const size_t o = (x == 0 ? base[0] : x == 1 ? base[1] : base[2]) + at;
                    kv8_load<float, 4>(a.cos_tab + o, cs + q);
                    kv8_load<float, 4>(a.sin_tab + o, sn + q);
                } else {
#pragma unroll
                    for (int j = 0; j < 4; ++j) {
                        const int x = axis(at + j);
                        const size_t o = (x == 0 ? base[0] : x == 1 ? base[1] : base[2]) + at + j;
                        cs[q + j] = a.cos_tab[o];
                        sn[q + j] = a.sin_tab[o];
                    }
                }
            }
        }
        const int h_lo = unit * w.per_wave, h_hi = min(h_lo + w.per_wave, a.q_heads + hkv);
        for (int h = h_lo; h < h_hi; ++h) {
            const bool isq = h < a.q_heads;
            const int hh = isq ? h : h - a.q_heads;
            const T* src = isq ? (const T*)a.q + (size_t)row * a.ldq : (const T*)a.k + (size_t)row * a.ldk;
            src += hh * HD + PL * g;
            float x0[PL], x1[PL];
#pragma unroll
            for (int q = 0; q < PL; q += 8) {
                kv8_load<T, 8>(src + q, x0 + q);
                kv8_load<T, 8>(src + HALF + q, x1 + q);
            }
            double y0[PL], y1[PL];
#pragma unroll
            for (int q = 0; q < PL; ++q) {
                y0[q] = x0[q];
                y1[q] = x1[q];
                if (a.n_axes) {
                    y0[q] = (double)x0[q] * cs[q] - (double)x1[q] * sn[q];
                    y1[q] = (double)x1[q] * cs[q] + (double)x0[q] * sn[q];
                }
            }
            if (isq) {
                if (mine) {
                    T* dst = (T*)a.q_out + (size_t)row * a.ldq_out + hh * HD + PL * g;
#pragma unroll
                    for (int q = 0; q < PL; q += 8) {
                        kv8_store8(dst + q, y0 + q);
                        kv8_store8(dst + HALF + q, y1 + q);
                    }
                }
                continue;
            }
            if (!there) continue;
            float am = 0.f;
#pragma unroll
            for (int q = 0; q < PL; ++q) {
                x0[q] = kv8_storable(kv8_odd(y0[q]));
                x1[q] = kv8_storable(kv8_odd(y1[q]));
                am = fmaxf(am, fmaxf(fabsf(x0[q]), fabsf(x1[q])));   // fmax passes a NaN over
            }
            am = wave_max(mine ? am : 0.f);
            int e = kv8_exponent(am);
            const size_t grp = ((size_t)page * 2) * hkv + hh;
            // lane's codes: pairs' first elements, and second ones HALF dims on
            uint8_t* const dst = codes + grp * (KV8_PAGE * HD) + t * 64 + PL * g;
            constexpr int HI = HD == 128 ? 1024 : 32;
            if (s0 > 0) {
                const int was = min(max((int)(__float_as_uint(w.c.scales[grp]) >> 23 & 255) - 127, KV8_EXP_MIN), KV8_EXP_MAX);
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
        unsigned keep = 0;               // bytes of a dword that are not new
#pragma unroll
        for (int j = 0; j < 4; ++j)
            if (4 * g + j < s0 || 4 * g + j >= s1) keep |= 0xffu << (8 * j);
        for (int h = h_lo; h < h_hi; ++h) {
            float x[NC][4][4];
            float am = 0.f;
#pragma unroll
            for (int j = 0; j < 4; ++j) {
                const int t = 4 * g + j;
                const bool mine = t >= s0 && t < s1;
                const T* src = (const T*)a.v + (size_t)(r0 + first + (mine ? t : s0)) * a.ldv + h * HD + 4 * l;
#pragma unroll
                for (int c = 0; c < NC; ++c) {
                    kv8_load<T, 4>(src + 64 * c, x[c][j]);
#pragma unroll
                    for (int d = 0; d < 4; ++d) {
                        x[c][j][d] = kv8_storable(x[c][j][d]);
                        if (mine) am = fmaxf(am, fabsf(x[c][j][d]));
                    }
                }
            }
            am = wave_max(am);
            int e = kv8_exponent(am);
            const size_t grp = ((size_t)page * 2 + 1) * hkv + h;
            uint4* const dst = reinterpret_cast<uint4*>(codes + grp * (KV8_PAGE * HD)) + lane;
            float sh = 1.f;
            if (s0 > 0) {
                const int was = min(max((int)(__float_as_uint(w.c.scales[grp]) >> 23 & 255) - 127, KV8_EXP_MIN), KV8_EXP_MAX);
                if (e > was) sh = kv8_pow2(was - e);
                e = max(e, was);
            }
            const float inv = kv8_pow2(-e);
            // slots before s0 keep their values, slots behind s1 their bytes
            unsigned before = 0;
#pragma unroll
            for (int j = 0; j < 4; ++j)
                if (4 * g + j < s0) before |= 0xffu << (8 * j);
            if (keep != ~0u || (before && sh != 1.f)) {
#pragma unroll
                for (int c = 0; c < NC; ++c) {
                    unsigned o[4], n[4] = {0, 0, 0, 0};
                    if (keep) {
                        const uint4 old = dst[64 * c];
                        n[0] = old.x; n[1] = old.y; n[2] = old.z; n[3] = old.w;
                    }
#pragma unroll
                    for (int d = 0; d < 4; ++d) {
                        const unsigned nw = kv8_pack4(x[c][0][d] * inv, x[c][1][d] * inv, x[c][2][d] * inv, x[c][3][d] * inv);
                        unsigned od = n[d];
                        if (sh != 1.f) od = (kv8_shift4(od, sh) & before) | (od & ~before);
                        o[d] = (od & keep) | (nw & ~keep);
                    }
                    dst[64 * c] = make_uint4(o[0], o[1], o[2], o[3]);
                }
            }
            if (lane == 0) w.c.scales[grp] = kv8_pow2(e);
        }
    }
}

// ------------------------------------------------------------- attention --

struct Kv8Plan {
    int kw = 4;         // waves of a workgroup that share its rows and split its keys
    int tile_rows = 16; // query rows (token, head of the group) of a workgroup
    int tiles = 1;      // workgroups that a (sequence, KV head)'s rows take
    int parts = 1;      // most parts that a tile's keys are cut into
    int part_keys = 0;  // keys of a part
};

struct Kv8AttnKernelArgs {
    ebrl_kv8_cache c;
    ebrl_kv8_attn_args a;
    int grp, tiles, parts, part_keys;
    float scale_log2;
    unsigned* counters;
    float* part;
};

// Lanes l, l ^ 16, l ^ 32, l ^ 48 hold one query's keys.
EBRL_DEV float kv8_max_groups(float v) {
    const unsigned u = __float_as_uint(v);
    const auto a = __builtin_amdgcn_permlane16_swap(u, u, false, false);
    v = fmaxf(__uint_as_float((unsigned)a[0]), __uint_as_float((unsigned)a[1]));
    const unsigned w = __float_as_uint(v);
    const auto b = __builtin_amdgcn_permlane32_swap(w, w, false, false);
    return fmaxf(__uint_as_float((unsigned)b[0]), __uint_as_float((unsigned)b[1]));
}
EBRL_DEV float kv8_sum_groups(float v) {
    const unsigned u = __float_as_uint(v);
    const auto a = __builtin_amdgcn_permlane16_swap(u, u, false, false);
    v = __uint_as_float((unsigned)a[0]) + __uint_as_float((unsigned)a[1]);
    const unsigned w = __float_as_uint(v);
    const auto b = __builtin_amdgcn_permlane32_swap(w, w, false, false);
    return __uint_as_float((unsigned)b[0]) + __uint_as_float((unsigned)b[1]);
}

// Eight codes (two dwords) as bf16, the scale applied.
EBRL_DEV bf16x8 kv8_bf16(unsigned lo, unsigned hi, float sl, float sh) {
    const bf16x2 a = __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(lo, sl, false);
    const bf16x2 b = __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(lo, sl, true);
    const bf16x2 c = __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(hi, sh, false);
    const bf16x2 d = __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(hi, sh, true);
    return bf16x8{a[0], a[1], b[0], b[1], c[0], c[1], d[0], d[1]};
}

// A float as NP bf16 terms that add up to it (three hold all 24 bits).
template <int NP> EBRL_DEV void kv8_split(float x, __bf16* o, int stride) {
#pragma unroll
    for (int p = 0; p < NP; ++p) {
        o[p * stride] = (__bf16)x;
        x -= (float)o[p * stride];
    }
}

template <typename T, int HD, int QT, int KW>
__global__ __launch_bounds__(256) void kv8_attn_kernel(Kv8AttnKernelArgs w)
{
    constexpr int NP = sizeof(T) == 4 ? 3 : 1;   // bf16 terms of a query element and of a weight
    constexpr int NC = HD / 64;
    constexpr int RW = 16 * QT;                  // rows of a wave
    constexpr int TR = RW * (4 / KW);            // rows of a workgroup
    __shared__ __attribute__((aligned(16))) float s_o[KW > 1 ? 4 : 1][KW > 1 ? RW : 1][KW > 1 ? HD + 4 : 1];
    __shared__ float s_m[4][RW], s_l[4][RW];
    __shared__ int s_last;

    const ebrl_kv8_attn_args& a = w.a;
    const int hkv = w.c.kv_heads, grp = w.grp;
    const int tid = threadIdx.x, lane = tid & 63;
    const int wave = __builtin_amdgcn_readfirstlane(tid >> 6);
    const int r = lane & 15, g = lane >> 4;

    // part, then tile, then KV head, then sequence
    unsigned id = blockIdx.x;
    const int part = id % w.parts;
    id /= w.parts;
    const int unit = id;
    const int tile = id % w.tiles;
    id /= w.tiles;
    const int kvh = id % hkv, i = id / hkv;

    const int trow = a.seq ? a.seq[i] : i;
    const int r0 = min(max(a.row_start[i], 0), a.rows);
    const int m = min(max(min(a.row_start[i + 1], a.rows) - r0, 0), a.max_q_len);
    const int rows = m * grp, t0 = tile * TR;
    if (t0 >= rows) return;
    const bool known = trow >= 0 && trow < w.c.table_rows;
    const int len = known ? min(max(a.kv_len[i], 0), min(a.max_kv_len, w.c.table_stride * KV8_PAGE)) : 0;
    // keys that some row of this workgroup sees
    const int last_tok = (min(t0 + TR, rows) - 1) / grp;
    const int end = a.causal ? max(min(len, len - m + last_tok + 1), 0) : len;
    const int parts = max(1, (end + w.part_keys - 1) / w.part_keys);
    if (part >= parts) return;
    const int k_lo = part * w.part_keys, k_hi = min(end, k_lo + w.part_keys);

    // this wave's rows and what they see
    const int wr0 = t0 + (wave / KW) * RW;
    int tok[QT], lim[QT];
    bf16x8 qb[QT][NP][HD / 32];
    int see_all = k_hi, wave_end = k_hi;   // keys that every row, that some row of the wave sees
#pragma unroll
    for (int qt = 0; qt < QT; ++qt) {
        const int row = min(wr0 + 16 * qt + r, rows - 1);
        tok[qt] = row / grp;
        const int h = kvh * grp + (row - tok[qt] * grp);
        lim[qt] = a.causal ? min(len, len - m + tok[qt] + 1) : len;
        const T* q = (const T*)a.q + (size_t)(r0 + tok[qt]) * a.ldq + h * HD;
#pragma unroll
        for (int s = 0; s < HD / 32; ++s) {
            float x[8];
            kv8_load<T, 8>(q + (s >> 1) * 64 + g * 16 + (s & 1) * 8, x);
#pragma unroll
            for (int j = 0; j < 8; ++j) {
                __bf16 p[NP];
                kv8_split<NP>(x[j], p, 1);
#pragma unroll
                for (int y = 0; y < NP; ++y) qb[qt][y][s][j] = p[y];
            }
        }
    }
    if (a.causal) {
        see_all = min(see_all, len - m + min(wr0, rows - 1) / grp + 1);
        wave_end = min(wave_end, len - m + (min(wr0 + RW, rows) - 1) / grp + 1);
    }
    if (wr0 >= rows) wave_end = k_lo;

    f32x4 acc[QT][HD / 16];
    float mx[QT], sum[QT];
#pragma unroll
    for (int qt = 0; qt < QT; ++qt) {
        mx[qt] = -INFINITY;
        sum[qt] = 0.f;
#pragma unroll
        for (int d = 0; d < HD / 16; ++d) acc[qt][d] = f32x4{0.f, 0.f, 0.f, 0.f};
    }

    const int* table = w.c.block_table + (size_t)(known ? trow : 0) * w.c.table_stride;
    const size_t group_bytes = (size_t)KV8_PAGE * HD;
    for (int k0 = k_lo + 32 * (wave % KW); k0 < wave_end; k0 += 32 * KW) {
        uint4 kc[2][NC], vc[2][NC];
        float ks[2], vs[2];
        bool there[2];
#pragma unroll
        for (int t = 0; t < 2; ++t) {
            const int at = k0 + 16 * t;
            int page = at < k_hi ? table[at / KV8_PAGE] : -1;
            page = __builtin_amdgcn_readfirstlane(page);
            there[t] = page >= 0 && page < w.c.num_blocks;
            if (there[t]) {
                const size_t kg = (size_t)page * 2 * hkv + kvh, vg = kg + hkv;
                const uint8_t* kp = (const uint8_t*)w.c.codes + kg * group_bytes + r * 64 + g * 16;
                const uint8_t* vp = (const uint8_t*)w.c.codes + vg * group_bytes + lane * 16;
                ks[t] = w.c.scales[kg];
                vs[t] = w.c.scales[vg];
#pragma unroll
                for (int c = 0; c < NC; ++c) {
                    kc[t][c] = *reinterpret_cast<const uint4*>(kp + 1024 * c);
                    vc[t][c] = *reinterpret_cast<const uint4*>(vp + 1024 * c);
                }
            } else {
                ks[t] = vs[t] = 1.f;
#pragma unroll
                for (int c = 0; c < NC; ++c) kc[t][c] = vc[t][c] = make_uint4(0, 0, 0, 0);
            }
        }
        // S^T: lane (r, g) gets query r's keys 16 t + 4 g + v
        f32x4 s[QT][2];
#pragma unroll
        for (int t = 0; t < 2; ++t) {
#pragma unroll
            for (int qt = 0; qt < QT; ++qt) s[qt][t] = f32x4{0.f, 0.f, 0.f, 0.f};
#pragma unroll
            for (int c = 0; c < NC; ++c) {
                const bf16x8 ka = kv8_bf16(kc[t][c].x, kc[t][c].y, ks[t], ks[t]);
                const bf16x8 kb = kv8_bf16(kc[t][c].z, kc[t][c].w, ks[t], ks[t]);
#pragma unroll
                for (int qt = 0; qt < QT; ++qt)
#pragma unroll
                    for (int p = NP - 1; p >= 0; --p) {
                        s[qt][t] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(ka, qb[qt][p][2 * c], s[qt][t], 0, 0, 0);
                        s[qt][t] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(kb, qb[qt][p][2 * c + 1], s[qt][t], 0, 0, 0);
                    }
            }
        }
        const bool masked = k0 + 32 > see_all || !there[0] || !there[1];
        unsigned nan_v = 0;               // this lane holds V codes that are NaN
        if (masked) {
            // slots past the last key may hold anything: their weights are
            // zero, and so have their values to be
#pragma unroll
            for (int t = 0; t < 2; ++t) {
                const int left = len - (k0 + 16 * t + 4 * g);
                const unsigned ok = left >= 4 ? ~0u : left <= 0 ? 0u : (1u << (8 * left)) - 1;
#pragma unroll
                for (int c = 0; c < NC; ++c) {
                    vc[t][c].x &= ok; vc[t][c].y &= ok; vc[t][c].z &= ok; vc[t][c].w &= ok;
                    const unsigned x[4] = {vc[t][c].x, vc[t][c].y, vc[t][c].z, vc[t][c].w};
#pragma unroll
                    for (int d = 0; d < 4; ++d) nan_v |= ((x[d] & 0x7f7f7f7fu) + 0x01010101u) & 0x80808080u;
                }
#pragma unroll
                for (int qt = 0; qt < QT; ++qt)
#pragma unroll
                    for (int v = 0; v < 4; ++v)
                        s[qt][t][v] = there[t] && k0 + 16 * t + 4 * g + v < lim[qt] ? s[qt][t][v] : -INFINITY;
            }
        }
        const bool nans = masked && __any(nan_v != 0);
        bf16x8 pb[QT][NP];
#pragma unroll
        for (int qt = 0; qt < QT; ++qt) {
            float tm = -INFINITY;
#pragma unroll
            for (int t = 0; t < 2; ++t)
#pragma unroll
                for (int v = 0; v < 4; ++v) tm = fmaxf(tm, s[qt][t][v]);
            tm = kv8_max_groups(tm);
            // the running maximum is a whole number of log2 units: rescaling
            // is by a power of two, exact
            const float nm = fmaxf(mx[qt], ceilf(tm * w.scale_log2));
            const float use = nm == -INFINITY ? 0.f : nm;
            const float alpha = mx[qt] == -INFINITY ? 0.f : ldexpf(1.0f, (int)(mx[qt] - use));
            float ps = 0.f;
#pragma unroll
            for (int t = 0; t < 2; ++t)
#pragma unroll
                for (int v = 0; v < 4; ++v) {
                    const float p = fast_exp2(fmaf(s[qt][t][v], w.scale_log2, -use));
                    ps += p;
                    __bf16 o[NP];
                    kv8_split<NP>(p, o, 1);
#pragma unroll
                    for (int y = 0; y < NP; ++y) pb[qt][y][4 * t + v] = o[y];
                }
            sum[qt] = sum[qt] * alpha + ps;
            mx[qt] = nm;
#pragma unroll
            for (int d = 0; d < HD / 16; ++d) acc[qt][d] *= alpha;
        }
        // O^T += V^T P^T: row r of tile 4 c + dt is dim 64 c + 4 r + dt, the
        // lane's eight keys those its scores are of
        if (!nans) {
#pragma unroll
            for (int c = 0; c < NC; ++c) {
                const unsigned x0[4] = {vc[0][c].x, vc[0][c].y, vc[0][c].z, vc[0][c].w};
                const unsigned x1[4] = {vc[1][c].x, vc[1][c].y, vc[1][c].z, vc[1][c].w};
#pragma unroll
                for (int d = 0; d < 4; ++d) {
                    const bf16x8 va = kv8_bf16(x0[d], x1[d], vs[0], vs[1]);
#pragma unroll
                    for (int qt = 0; qt < QT; ++qt)
#pragma unroll
                        for (int p = NP - 1; p >= 0; --p)
                            acc[qt][4 * c + d] =
                                __builtin_amdgcn_mfma_f32_16x16x32_bf16(va, pb[qt][p], acc[qt][4 * c + d], 0, 0, 0);
                }
            }
        } else {
            // a value is NaN in a tile that not every row sees whole: it
            // counts for the rows that see its key alone.  Products with the
            // NaNs taken as zero, then a count of those each row sees.
#pragma unroll
            for (int c = 0; c < NC; ++c) {
                const unsigned x0[4] = {vc[0][c].x, vc[0][c].y, vc[0][c].z, vc[0][c].w};
                const unsigned x1[4] = {vc[1][c].x, vc[1][c].y, vc[1][c].z, vc[1][c].w};
#pragma unroll
                for (int d = 0; d < 4; ++d) {
                    bf16x8 va = kv8_bf16(x0[d], x1[d], vs[0], vs[1]), bad;
#pragma unroll
                    for (int j = 0; j < 8; ++j) {
                        const unsigned b = (j < 4 ? x0[d] : x1[d]) >> (8 * (j & 3)) & 0x7f;
                        bad[j] = (__bf16)(b == 0x7f ? 1.f : 0.f);
                        if (b == 0x7f) va[j] = (__bf16)0.f;
                    }
#pragma unroll
                    for (int qt = 0; qt < QT; ++qt) {
                        bf16x8 seen;
#pragma unroll
                        for (int j = 0; j < 8; ++j) {
                            const int key = k0 + 16 * (j >> 2) + 4 * g + (j & 3);
                            seen[j] = (__bf16)(there[j >> 2] && key < lim[qt] ? 1.f : 0.f);
                        }
#pragma unroll
                        for (int p = NP - 1; p >= 0; --p)
                            acc[qt][4 * c + d] =
                                __builtin_amdgcn_mfma_f32_16x16x32_bf16(va, pb[qt][p], acc[qt][4 * c + d], 0, 0, 0);
                        const f32x4 cnt =
                            __builtin_amdgcn_mfma_f32_16x16x32_bf16(bad, seen, f32x4{0.f, 0.f, 0.f, 0.f}, 0, 0, 0);
#pragma unroll
                        for (int v = 0; v < 4; ++v)
                            if (cnt[v] > 0.f) acc[qt][4 * c + d][v] = __uint_as_float(0x7fc00000u);
                    }
                }
            }
        }
    }
#pragma unroll
    for (int qt = 0; qt < QT; ++qt) sum[qt] = kv8_sum_groups(sum[qt]);

    // the waves that share rows join in wave order
    if constexpr (KW > 1) {
#pragma unroll
        for (int qt = 0; qt < QT; ++qt) {
#pragma unroll
            for (int d = 0; d < HD / 16; ++d)
#pragma unroll
                for (int v = 0; v < 4; ++v)
                    s_o[wave][16 * qt + r][64 * (d >> 2) + 16 * g + 4 * v + (d & 3)] = acc[qt][d][v];
            if (g == 0) { s_m[wave][16 * qt + r] = mx[qt]; s_l[wave][16 * qt + r] = sum[qt]; }
        }
        __syncthreads();
    }
    const int here = min(TR, rows - t0);            // rows of this workgroup
    const int n_parts = w.parts;
    auto out_at = [&](int row) {
        const int t = row / grp;
        return (T*)a.out + (size_t)(r0 + t) * a.ldo + (size_t)(kvh * grp + (row - t * grp)) * HD;
    };
    const __amdgpu_buffer_rsrc_t pr = coherent_rsrc(w.part + (size_t)unit * n_parts * TR * (HD + 2));
    if constexpr (KW > 1) {
        for (int x = tid; x < here * (HD / 4); x += 256) {
            const int row = x / (HD / 4), d = x % (HD / 4) * 4;
            const int w0 = row / RW * KW, rr = row % RW;
            float M = -INFINITY, L = 0.f;
            f32x4 o = f32x4{0.f, 0.f, 0.f, 0.f};
#pragma unroll
            for (int y = 0; y < KW; ++y) M = fmaxf(M, s_m[w0 + y][rr]);
#pragma unroll
            for (int y = 0; y < KW; ++y) {
                const float my = s_m[w0 + y][rr];
                const float wt = my == -INFINITY ? 0.f : fast_exp2(my - M);
                L += wt * s_l[w0 + y][rr];
                o += wt * *reinterpret_cast<const f32x4*>(&s_o[w0 + y][rr][d]);
            }
            if (parts == 1) {
                const float inv = L == 0.f ? 0.f : 1.f / L;
                st4<T>(out_at(t0 + row) + d, o[0] * inv, o[1] * inv, o[2] * inv, o[3] * inv);
            } else {
                const int at = (part * TR + row) * (HD + 2);
                st_coherent1(pr, (at + d) * 4, o[0]);
                st_coherent1(pr, (at + d + 1) * 4, o[1]);
                st_coherent1(pr, (at + d + 2) * 4, o[2]);
                st_coherent1(pr, (at + d + 3) * 4, o[3]);
                if (d == 0) { st_coherent1(pr, (at + HD) * 4, M); st_coherent1(pr, (at + HD + 1) * 4, L); }
            }
        }
    } else {
#pragma unroll
        for (int qt = 0; qt < QT; ++qt) {
            const int row = wr0 + 16 * qt + r - t0;
            if (row >= here) continue;
            const float inv = parts > 1 ? 1.f : sum[qt] == 0.f ? 0.f : 1.f / sum[qt];
            const int at = (part * TR + row) * (HD + 2);
#pragma unroll
            for (int c = 0; c < NC; ++c)
#pragma unroll
                for (int v = 0; v < 4; ++v) {
                    const int d = 64 * c + 16 * g + 4 * v;
                    const float o0 = acc[qt][4 * c][v] * inv, o1 = acc[qt][4 * c + 1][v] * inv;
                    const float o2 = acc[qt][4 * c + 2][v] * inv, o3 = acc[qt][4 * c + 3][v] * inv;
                    if (parts == 1) {
                        st4<T>(out_at(t0 + row) + d, o0, o1, o2, o3);
                    } else {
                        st_coherent1(pr, (at + d) * 4, o0);
                        st_coherent1(pr, (at + d + 1) * 4, o1);
                        st_coherent1(pr, (at + d + 2) * 4, o2);
                        st_coherent1(pr, (at + d + 3) * 4, o3);
                    }
                }
            if (parts > 1 && g == 0) { st_coherent1(pr, (at + HD) * 4, mx[qt]); st_coherent1(pr, (at + HD + 1) * 4, sum[qt]); }
        }
    }
    if (parts == 1) return;
    // the workgroup that finishes its tile's last part joins all of them, in their order
    asm volatile("s_waitcnt vmcnt(0)" ::: "memory");
    __syncthreads();
    if (tid == 0)
        s_last = __hip_atomic_fetch_add(w.counters + unit, 1u, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT) ==
                 (unsigned)(parts - 1);
    __syncthreads();
    if (!s_last) return;
    for (int x = tid; x < here * HD; x += 256) {
        const int row = x / HD, d = x % HD;
        float M = -INFINITY, L = 0.f, o = 0.f;
        for (int y = 0; y < parts; ++y) M = fmaxf(M, ld_coherent1(pr, ((y * TR + row) * (HD + 2) + HD) * 4));
        for (int y = 0; y < parts; ++y) {
            const int at = (y * TR + row) * (HD + 2);
            const float my = ld_coherent1(pr, (at + HD) * 4);
            const float wt = my == -INFINITY ? 0.f : fast_exp2(my - M);
            L += wt * ld_coherent1(pr, (at + HD + 1) * 4);
            o += wt * ld_coherent1(pr, (at + d) * 4);
        }
        st_elem<T>(out_at(t0 + row) + d, L == 0.f ? 0.f : o / L);
    }
    if (tid == 0) __hip_atomic_store(w.counters + unit, 0u, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT);
}

// ------------------------------------------------------- plans, launches --

static Kv8Plan kv8_plan(const ebrl_kv8_cache& c, const ebrl_kv8_attn_args& a) {
    Kv8Plan p;
    const int64_t rows = (int64_t)a.max_q_len * (a.q_heads / c.kv_heads);
    if (rows <= 16) {
        p.kw = 4;
        p.tile_rows = 16;
    } else {
        p.kw = 1;
        p.tile_rows = a.dtype == EBRL_DTYPE_FP32 ? 64 : 128;
    }
    p.tiles = (int)((rows + p.tile_rows - 1) / p.tile_rows);
    const int64_t units = (int64_t)a.n * c.kv_heads * p.tiles;
    const int step = 32 * p.kw;                       // keys that a workgroup takes at a time
    const int64_t most = std::max<int64_t>(1, ((int64_t)a.max_kv_len + 255) / 256);
    const int64_t want = std::min(most, std::max<int64_t>(1, 1024 / units));
    const int64_t keys = ((int64_t)a.max_kv_len + want - 1) / want;
    p.part_keys = (int)std::max<int64_t>(step, (keys + step - 1) / step * step);
    p.parts = (int)std::max<int64_t>(1, ((int64_t)a.max_kv_len + p.part_keys - 1) / p.part_keys);
    return p;
}

static int64_t kv8_counter_bytes(int64_t units) { return (units * 4 + 255) / 256 * 256; }

static bool kv8_cache_ok(const ebrl_kv8_cache* c) {
    return c && c->num_blocks >= 1 && c->table_rows >= 1 && c->table_stride >= 1 && c->table_stride < (1 << 27) &&
           c->kv_heads >= 1 && (c->head_dim == 64 || c->head_dim == 128);
}
static bool kv8_pointers_ok(const ebrl_kv8_cache* c) {
    return c->codes && c->scales && c->block_table && (uintptr_t)c->codes % 16 == 0 && (uintptr_t)c->scales % 4 == 0 &&
           (uintptr_t)c->block_table % 4 == 0;
}
// Rows of `width` elements every `ld`, 16-byte aligned.
static bool kv8_rows_ok(const void* p, int64_t ld, int64_t width, int esz) {
    return p && (uintptr_t)p % 16 == 0 && ld >= width && ld * esz % 16 == 0 && ld < ((int64_t)1 << 40);
}
constexpr int64_t KV8_MAX_GROUPS = 1 << 23;   // workgroups of 256 threads in a launch: under 2^32 threads

static bool kv8_attn_shape_ok(const ebrl_kv8_cache* c, const ebrl_kv8_attn_args* a) {
    return kv8_cache_ok(c) && a && (a->dtype == EBRL_DTYPE_BF16 || a->dtype == EBRL_DTYPE_FP32) && a->n >= 0 &&
           a->rows >= 0 && a->max_q_len >= 0 && a->max_kv_len >= 0 &&
           a->max_kv_len <= (1 << 30) && a->q_heads >= 1 && a->q_heads % c->kv_heads == 0 &&
           (int64_t)a->max_q_len * (a->q_heads / c->kv_heads) < (1 << 30);
}

template <typename T, int HD>
static void kv8_attn_launch(const Kv8Plan& p, const Kv8AttnKernelArgs& w, unsigned groups, hipStream_t s) {
    constexpr int QT = sizeof(T) == 4 ? 1 : 2;
    if (p.kw == 4) hipLaunchKernelGGL((kv8_attn_kernel<T, HD, 1, 4>), dim3(groups), dim3(256), 0, s, w);
    else hipLaunchKernelGGL((kv8_attn_kernel<T, HD, QT, 1>), dim3(groups), dim3(256), 0, s, w);
}

}  // namespace ebrl

using namespace ebrl;

extern "C" {

int ebrl_op_kv8_write(const ebrl_kv8_cache* cache, const ebrl_kv8_write_args* args, void* stream) {
    if (!kv8_cache_ok(cache) || !args) return EBRL_E_INVALID;
    const ebrl_kv8_write_args& a = *args;
    const int hd = cache->head_dim, hkv = cache->kv_heads;
    if ((a.dtype != EBRL_DTYPE_BF16 && a.dtype != EBRL_DTYPE_FP32) || a.n < 0 || a.rows < 0 || a.max_len < 0 ||
        a.q_heads < 0 || a.n_axes < 0 || a.n_axes > 3 || (a.q_heads > 0 && a.n_axes == 0))
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
    const int64_t len = std::min<int64_t>(a.max_len, a.rows);
    w.pages = (int)((len + 2 * KV8_PAGE - 2) / KV8_PAGE);
    const int64_t sp = (int64_t)a.n * w.pages;
    w.per_wave = sp * (a.q_heads + 2 * hkv) > 16384 ? 4 : 1;
    w.rot_units = (a.q_heads + hkv + w.per_wave - 1) / w.per_wave;
    w.v_units = (hkv + w.per_wave - 1) / w.per_wave;
    const int64_t groups = (sp * (w.rot_units + w.v_units) + 3) / 4;
    if (groups > KV8_MAX_GROUPS) return EBRL_E_INVALID;
    const dim3 grid((unsigned)groups);
    hipStream_t s = (hipStream_t)stream;
    if (esz == 2) {
        if (hd == 64) hipLaunchKernelGGL((kv8_write_kernel<bf16_t, 64>), grid, dim3(256), 0, s, w);
        else hipLaunchKernelGGL((kv8_write_kernel<bf16_t, 128>), grid, dim3(256), 0, s, w);
    } else {
        if (hd == 64) hipLaunchKernelGGL((kv8_write_kernel<float, 64>), grid, dim3(256), 0, s, w);
        else hipLaunchKernelGGL((kv8_write_kernel<float, 128>), grid, dim3(256), 0, s, w);
    }
    return hipGetLastError() == hipSuccess ? EBRL_OK : EBRL_E_HIP;
}

int64_t ebrl_op_kv8_attn_workspace(const ebrl_kv8_cache* cache, const ebrl_kv8_attn_args* args) {
    if (!kv8_attn_shape_ok(cache, args)) return EBRL_E_INVALID;
    if (args->n == 0 || args->max_q_len == 0) return 0;
    const Kv8Plan p = kv8_plan(*cache, *args);
    if (p.parts == 1) return 0;
    const int64_t units = (int64_t)args->n * cache->kv_heads * p.tiles;
    return kv8_counter_bytes(units) + units * p.parts * p.tile_rows * (cache->head_dim + 2) * 4;
}

int ebrl_op_kv8_attn(const ebrl_kv8_cache* cache, const ebrl_kv8_attn_args* args, void* stream) {
    if (!kv8_attn_shape_ok(cache, args) || !(args->scale > 0.f) || !isfinite(args->scale)) return EBRL_E_INVALID;
    const ebrl_kv8_attn_args& a = *args;
    if (a.n == 0 || a.rows == 0 || a.max_q_len == 0) return EBRL_OK;
    const int hd = cache->head_dim, esz = a.dtype == EBRL_DTYPE_FP32 ? 4 : 2;
    const int64_t width = (int64_t)a.q_heads * hd;
    if (!kv8_pointers_ok(cache) || !a.row_start || !a.kv_len || !kv8_rows_ok(a.q, a.ldq, width, esz) ||
        !kv8_rows_ok(a.out, a.ldo, width, esz) || a.q == a.out)
        return EBRL_E_INVALID;
    const int64_t need = ebrl_op_kv8_attn_workspace(cache, args);
    if (need > 0 && (!a.workspace || a.workspace_bytes < need || (uintptr_t)a.workspace % 16)) return EBRL_E_INVALID;
    const Kv8Plan p = kv8_plan(*cache, a);
    const int64_t units = (int64_t)a.n * cache->kv_heads * p.tiles, groups = units * p.parts;
    if (groups > KV8_MAX_GROUPS) return EBRL_E_INVALID;
    Kv8AttnKernelArgs w;
    w.c = *cache;
    w.a = a;
    w.grp = a.q_heads / cache->kv_heads;
    w.tiles = p.tiles;
    w.parts = p.parts;
    w.part_keys = p.part_keys;
    w.scale_log2 = a.scale * 1.4426950408889634f;
    w.counters = (unsigned*)a.workspace;
    w.part = need ? (float*)((char*)a.workspace + kv8_counter_bytes(units)) : nullptr;
    hipStream_t s = (hipStream_t)stream;
    if (esz == 2) {
        if (hd == 64) kv8_attn_launch<bf16_t, 64>(p, w, (unsigned)groups, s);
        else kv8_attn_launch<bf16_t, 128>(p, w, (unsigned)groups, s);
    } else {
        if (hd == 64) kv8_attn_launch<float, 64>(p, w, (unsigned)groups, s);
        else kv8_attn_launch<float, 128>(p, w, (unsigned)groups, s);
    }
    return hipGetLastError() == hipSuccess ? EBRL_OK : EBRL_E_HIP;
}

}  // extern "C"

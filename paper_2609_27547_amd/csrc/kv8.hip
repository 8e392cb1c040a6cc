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
#include <math.h>

#include "../../include/ebrl.h"
#include "../../include/ebrl_kv8.h"
#include "kernels.h"

namespace ebrl {

typedef __bf16 bf16x2 __attribute__((ext_vector_type(2)));
typedef float f32x2 __attribute__((ext_vector_type(2)));

constexpr int KV8_PAGE = EBRL_KV8_PAGE;
constexpr int KV8_EXP_MIN = -100, KV8_EXP_MAX = 120;   // 448 * 2^120 > FLT_MAX
constexpr float KV8_SLACK = 10.f;     // log2 of the largest weight that a softmax keeps
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

// How a call is cut into workgroups of four waves.
struct Kv8Plan {
    bool decode = true;   // the waves share 16 rows and deal the keys, or share the keys and have 32 rows each
    int tile_rows = 16;   // query rows (token, head of the group) of a workgroup
    int tiles = 1;        // workgroups that a (sequence, KV head)'s rows take
    int parts = 1;        // most parts that a tile's keys are cut into
    int part_keys = 0;    // keys of a part
};

struct Kv8AttnKernelArgs {
    ebrl_kv8_cache c;
    ebrl_kv8_attn_args a;
    int grp, tiles, tile_rows, parts, part_keys;
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
EBRL_DEV Kv8Tile kv8_tile(const Kv8AttnKernelArgs& w, int i, int tile) {
    const ebrl_kv8_attn_args& a = w.a;
    Kv8Tile t;
    const int trow = a.seq ? a.seq[i] : i;
    t.r0 = min(max(a.row_start[i], 0), a.rows);
    t.m = min(max(min(a.row_start[i + 1], a.rows) - t.r0, 0), a.max_q_len);
    t.rows = t.m * w.grp;
    t.t0 = tile * w.tile_rows;
    const bool known = trow >= 0 && trow < w.c.table_rows;
    t.len = known ? min(max(a.kv_len[i], 0), min(a.max_kv_len, w.c.table_stride * KV8_PAGE)) : 0;
    const int last = (min(t.t0 + w.tile_rows, t.rows) - 1) / w.grp;
    t.end = a.causal ? max(min(t.len, t.len - t.m + last + 1), 0) : t.len;
    t.parts = max(1, (t.end + w.part_keys - 1) / w.part_keys);
    t.table = w.c.block_table + (size_t)(known ? trow : 0) * w.c.table_stride;
    return t;
}

// Eight codes (two dwords) as bf16, the scales applied.
EBRL_DEV bf16x8 kv8_bf16(unsigned lo, unsigned hi, float sl, float sh) {
    const bf16x2 a = __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(lo, sl, false);
    const bf16x2 b = __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(lo, sl, true);
    const bf16x2 c = __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(hi, sh, false);
    const bf16x2 d = __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(hi, sh, true);
    return bf16x8{a[0], a[1], b[0], b[1], c[0], c[1], d[0], d[1]};
}

// A float as NP bf16 terms that add up to it (three hold all 24 bits).
template <int NP> EBRL_DEV void kv8_split(float x, __bf16* o) {
#pragma unroll
    for (int p = 0; p < NP; ++p) {
        o[p] = (__bf16)x;
        x -= (float)o[p];
    }
}

// The state of a wave's 16 QT query rows.  Lane (r, g) holds query r of each
// 16: its elements 64 c + 16 g .. + 15, its scores for keys 4 g .. 4 g + 3 of
// each page, and its results in dims 64 c + 16 g .. + 15.
template <typename T, int HD, int QT> struct Kv8Rows {
    static constexpr int NP = sizeof(T) == 4 ? 3 : 1;   // bf16 terms of a query element and of a weight
    static constexpr int NC = HD / 64;
    bf16x8 q[QT][NP][HD / 32];
    f32x4 acc[QT][HD / 16];   // acc[4 c + d][v]: dim 64 c + 16 g + 4 v + d
    float mx[QT], sum[QT];    // log2 of what the weights are relative to; this lane's share of their sum
    int lim[QT];              // keys that the row sees
    int all, end;             // keys that every row, that some row of the wave sees

    EBRL_DEV void init(const Kv8AttnKernelArgs& w, const Kv8Tile& t, int kvh, int wr0, int k_hi, int lane) {
        const int r = lane & 15, g = lane >> 4;
#pragma unroll
        for (int qt = 0; qt < QT; ++qt) {
            const int row = min(wr0 + 16 * qt + r, t.rows - 1);
            const int tok = row / w.grp, h = kvh * w.grp + (row - tok * w.grp);
            lim[qt] = w.a.causal ? min(t.len, t.len - t.m + tok + 1) : t.len;
            const T* src = (const T*)w.a.q + (size_t)(t.r0 + tok) * w.a.ldq + h * HD;
#pragma unroll
            for (int s = 0; s < HD / 32; ++s) {
                float x[8];
                kv8_load<T, 8>(src + (s >> 1) * 64 + g * 16 + (s & 1) * 8, x);
#pragma unroll
                for (int j = 0; j < 8; ++j) {
                    __bf16 p[NP];
                    kv8_split<NP>(x[j], p);
#pragma unroll
                    for (int y = 0; y < NP; ++y) q[qt][y][s][j] = p[y];
                }
            }
            mx[qt] = -INFINITY;
            sum[qt] = 0.f;
#pragma unroll
            for (int d = 0; d < HD / 16; ++d) acc[qt][d] = f32x4{0.f, 0.f, 0.f, 0.f};
        }
        all = end = k_hi;
        if (w.a.causal) {
            all = min(all, t.len - t.m + min(wr0, t.rows - 1) / w.grp + 1);
            end = min(end, t.len - t.m + (min(wr0 + 16 * QT, t.rows) - 1) / w.grp + 1);
        }
        if (wr0 >= t.rows) end = 0;
    }

    // Two pages (32 keys from k0 on) in the lanes' order: kc, vc their codes,
    // ks, vs their scales, there: whether each is one.
    EBRL_DEV void step(uint4 (&kc)[2][NC], uint4 (&vc)[2][NC], const float (&ks)[2], const float (&vs)[2],
                       const bool (&there)[2], int k0, int len, float scale_log2, int lane)
    {
        const int g = lane >> 4;
        // S^T = K Q^T
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
                for (int p = NP - 1; p >= 0; --p)
#pragma unroll
                    for (int qt = 0; qt < QT; ++qt)
                        s[qt][t] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(ka, q[qt][p][2 * c], s[qt][t], 0, 0, 0);
#pragma unroll
                for (int p = NP - 1; p >= 0; --p)
#pragma unroll
                    for (int qt = 0; qt < QT; ++qt)
                        s[qt][t] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(kb, q[qt][p][2 * c + 1], s[qt][t], 0, 0, 0);
            }
        }
        bool nans = false;
        if (k0 + 32 > all || !there[0] || !there[1]) {
            // some row does not see some key.  Slots past the last key may
            // hold anything: their weights are zero, and so have their
            // values to be.
            unsigned bad = 0;
#pragma unroll
            for (int t = 0; t < 2; ++t) {
                const int left = there[t] ? len - (k0 + 16 * t + 4 * g) : 0;
                const unsigned ok = left >= 4 ? ~0u : left <= 0 ? 0u : (1u << (8 * left)) - 1;
#pragma unroll
                for (int c = 0; c < NC; ++c) {
                    vc[t][c].x &= ok; vc[t][c].y &= ok; vc[t][c].z &= ok; vc[t][c].w &= ok;
                    const unsigned x[4] = {vc[t][c].x, vc[t][c].y, vc[t][c].z, vc[t][c].w};
#pragma unroll
                    for (int d = 0; d < 4; ++d) bad |= ((x[d] & 0x7f7f7f7fu) + 0x01010101u) & 0x80808080u;
                }
#pragma unroll
                for (int qt = 0; qt < QT; ++qt)
#pragma unroll
                    for (int v = 0; v < 4; ++v)
                        s[qt][t][v] = there[t] && k0 + 16 * t + 4 * g + v < lim[qt] ? s[qt][t][v] : -INFINITY;
            }
            nans = __any(bad != 0);
        }
        // Weights are 2^(x - mx), x = score log2(e) / sqrt(hd).  mx is a whole
        // number that follows the row's maximum: it moves when a weight would
        // pass 2^KV8_SLACK, and rescaling by a power of two is exact, so
        // neither the moves nor the cut into steps changes a weight's
        // rounding to bf16.
        bool move = false;
        float tm[QT];
#pragma unroll
        for (int qt = 0; qt < QT; ++qt) {
            tm[qt] = -INFINITY;
#pragma unroll
            for (int t = 0; t < 2; ++t)
#pragma unroll
                for (int v = 0; v < 4; ++v) tm[qt] = fmaxf(tm[qt], s[qt][t][v]);
            move |= tm[qt] * scale_log2 > mx[qt] + KV8_SLACK;
        }
        if (__any(move)) {
#pragma unroll
            for (int qt = 0; qt < QT; ++qt) {
                const float nm = fmaxf(mx[qt], ceilf(attn_max_xor16_32(tm[qt]) * scale_log2));
                const float alpha = mx[qt] == nm ? 1.f : ldexpf(1.0f, (int)fmaxf(mx[qt] - nm, -300.f));
                mx[qt] = nm;
                sum[qt] *= alpha;
#pragma unroll
                for (int d = 0; d < HD / 16; ++d) acc[qt][d] *= alpha;
            }
        }
        bf16x8 pb[QT][NP];
#pragma unroll
        for (int qt = 0; qt < QT; ++qt) {
            const float use = mx[qt] == -INFINITY ? 0.f : mx[qt];
#pragma unroll
            for (int t = 0; t < 2; ++t)
#pragma unroll
                for (int v = 0; v < 4; ++v) {
                    const float p = fast_exp2(fmaf(s[qt][t][v], scale_log2, -use));
                    sum[qt] += p;
                    __bf16 o[NP];
                    kv8_split<NP>(p, o);
#pragma unroll
                    for (int y = 0; y < NP; ++y) pb[qt][y][4 * t + v] = o[y];
                }
        }
        // O^T += V^T P^T: row r of product 4 c + d is dim 64 c + 4 r + d, a
        // lane's eight keys those that its scores are of
#pragma unroll
        for (int c = 0; c < NC; ++c) {
            const unsigned x0[4] = {vc[0][c].x, vc[0][c].y, vc[0][c].z, vc[0][c].w};
            const unsigned x1[4] = {vc[1][c].x, vc[1][c].y, vc[1][c].z, vc[1][c].w};
            if (!nans) {
#pragma unroll
                for (int d = 0; d < 4; ++d) {
                    const bf16x8 va = kv8_bf16(x0[d], x1[d], vs[0], vs[1]);
#pragma unroll
                    for (int p = NP - 1; p >= 0; --p)
#pragma unroll
                        for (int qt = 0; qt < QT; ++qt)
                            acc[qt][4 * c + d] =
                                __builtin_amdgcn_mfma_f32_16x16x32_bf16(va, pb[qt][p], acc[qt][4 * c + d], 0, 0, 0);
                }
            } else {
                // a value is NaN, and not every row sees its key: products
                // with NaNs taken as zero, then a count of those each row sees
#pragma unroll
                for (int d = 0; d < 4; ++d) {
                    bf16x8 va = kv8_bf16(x0[d], x1[d], vs[0], vs[1]), isnan;
#pragma unroll
                    for (int j = 0; j < 8; ++j) {
                        const unsigned b = (j < 4 ? x0[d] : x1[d]) >> (8 * (j & 3)) & 0x7f;
                        isnan[j] = (__bf16)(b == 0x7f ? 1.f : 0.f);
                        if (b == 0x7f) va[j] = (__bf16)0.f;
                    }
#pragma unroll
                    for (int qt = 0; qt < QT; ++qt) {
                        bf16x8 sees;
#pragma unroll
                        for (int j = 0; j < 8; ++j) {
                            const int key = k0 + 16 * (j >> 2) + 4 * g + (j & 3);
                            sees[j] = (__bf16)(there[j >> 2] && key < lim[qt] ? 1.f : 0.f);
                        }
#pragma unroll
                        for (int p = NP - 1; p >= 0; --p)
                            acc[qt][4 * c + d] =
                                __builtin_amdgcn_mfma_f32_16x16x32_bf16(va, pb[qt][p], acc[qt][4 * c + d], 0, 0, 0);
                        const f32x4 n =
                            __builtin_amdgcn_mfma_f32_16x16x32_bf16(isnan, sees, f32x4{0.f, 0.f, 0.f, 0.f}, 0, 0, 0);
#pragma unroll
                        for (int v = 0; v < 4; ++v)
                            if (n[v] > 0.f) acc[qt][4 * c + d][v] = __uint_as_float(0x7fc00000u);
                    }
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

// One query row a sequence, or few: the four waves of a workgroup share 16
// rows and deal the pairs of pages of its part of the keys.  Bound by the
// bytes of the cache: codes go straight to registers, the next two pages' in
// flight while two are worked on.
template <typename T, int HD>
__global__ __launch_bounds__(256, 2) void kv8_decode_kernel(Kv8AttnKernelArgs w)
{
    constexpr int NC = HD / 64;
    __shared__ __attribute__((aligned(16))) float s_o[4][16][HD + 4];
    __shared__ float s_m[4][16], s_l[4][16];

    const int hkv = w.c.kv_heads;
    const int tid = threadIdx.x, lane = tid & 63;
    const int wave = __builtin_amdgcn_readfirstlane(tid >> 6);
    const int r = lane & 15, g = lane >> 4;
    unsigned id = blockIdx.x;
    const int part = id % w.parts;
    const unsigned unit = id / w.parts;
    id = unit;
    const int tile = id % w.tiles;
    id /= w.tiles;
    const int kvh = id % hkv, i = id / hkv;
    const Kv8Tile t = kv8_tile(w, i, tile);
    if (t.t0 >= t.rows || part >= t.parts) return;
    const int k_lo = part * w.part_keys, k_hi = min(t.end, k_lo + w.part_keys);

    const size_t gb = (size_t)KV8_PAGE * HD;   // bytes of a (page, K or V, head) group
    const uint8_t* const codes = (const uint8_t*)w.c.codes + kvh * gb;
    const int k_at = r * 64 + g * 16, v_at = lane * 16;
    Kv8Rows<T, HD, 1> rows;
    const int p_hi = (k_hi + KV8_PAGE - 1) / KV8_PAGE;
    // 32 steps of this wave at a time: lane 2 s + t has page t of step s
    constexpr int BATCH = 32;
    bool first = true;
    for (int kb = k_lo; kb < k_hi || first; kb += BATCH * 128) {
        const int at = kb / KV8_PAGE + (lane >> 1) * 8 + wave * 2 + (lane & 1);
        int page = at < p_hi ? t.table[at] : -1;
        if (page >= w.c.num_blocks) page = -1;
        float ksv = 1.f, vsv = 1.f;
        if (page >= 0) {
            ksv = w.c.scales[(size_t)page * 2 * hkv + kvh];
            vsv = w.c.scales[((size_t)page * 2 + 1) * hkv + kvh];
        }
        const int n = (k_hi - kb - wave * 32 + 127) / 128;
        const int steps = min(max(n, 0), BATCH);
        auto load = [&](int s, uint4 (&kc)[2][NC], uint4 (&vc)[2][NC]) {
#pragma unroll
            for (int x = 0; x < 2; ++x) {
                // a page that is none: another's codes, not used
                const int pg = max(__builtin_amdgcn_readlane(page, 2 * s + x), 0);
                const uint8_t* kp = codes + (size_t)pg * 2 * hkv * gb;
                const uint8_t* vp = kp + (size_t)hkv * gb;
#pragma unroll
                for (int c = 0; c < NC; ++c) {
                    kc[x][c] = *reinterpret_cast<const uint4*>(kp + 1024 * c + k_at);
                    vc[x][c] = *reinterpret_cast<const uint4*>(vp + 1024 * c + v_at);
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
            rows.step(kc, vc, ks, vs, there, kb + s * 128 + wave * 32, t.len, w.scale_log2, lane);
        };
        uint4 ka[2][NC], va[2][NC], kn[2][NC], vn[2][NC];
        if (steps > 0) load(0, ka, va);
        if (first) rows.init(w, t, kvh, t.t0, k_hi, lane);
        first = false;
        for (int s = 0; s < steps; s += 2) {
            if (s + 1 < steps) load(s + 1, kn, vn);
            work(s, ka, va);
            if (s + 1 < steps) {
                if (s + 2 < steps) load(s + 2, ka, va);
                work(s + 1, kn, vn);
            }
        }
    }
    rows.sum[0] = attn_sum_xor16_32(rows.sum[0]);

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
    const int here = min(16, t.rows - t.t0);
    for (int x = tid; x < here * (HD / 4); x += 256) {
        const int row = x / (HD / 4), d = x % (HD / 4) * 4;
        float M = -INFINITY, L = 0.f;
        f32x4 o = {0.f, 0.f, 0.f, 0.f};
#pragma unroll
        for (int y = 0; y < 4; ++y) M = fmaxf(M, s_m[y][row]);
#pragma unroll
        for (int y = 0; y < 4; ++y) {
            const float my = s_m[y][row];
            const float wt = my == -INFINITY ? 0.f : fast_exp2(my - M);
            L += wt * s_l[y][row];
            o += wt * *reinterpret_cast<const f32x4*>(&s_o[y][row][d]);
        }
        if (t.parts == 1) {
            const float inv = L == 0.f ? 0.f : 1.f / L;
            st4<T>(kv8_out<T, HD>(w, t, kvh, t.t0 + row) + d, o[0] * inv, o[1] * inv, o[2] * inv, o[3] * inv);
        } else {
            const size_t to = ((size_t)unit * w.parts + part) * 16 + row;
            *reinterpret_cast<f32x4*>(w.part_o + to * HD + d) = o;
            if (d == 0) { w.part_ml[2 * to] = M; w.part_ml[2 * to + 1] = L; }
        }
    }
}

// Many rows: the four waves of a workgroup have 16 QT rows each and share
// the keys, 64 at a time, through a ring of LDS buffers that DMA fills with
// raw codes (16 KB a step at head dim 128), in the order in which a lane
// reads them back: 16 bytes a lane, one after the other.
template <typename T, int HD, int QT>
__global__ __launch_bounds__(256, 2) void kv8_prompt_kernel(Kv8AttnKernelArgs w)
{
    constexpr int NC = HD / 64;
    constexpr int RW = 16 * QT;
    constexpr int S = 3;                       // ring depth
    constexpr int SEG = 512;                   // pages whose ids and scales LDS holds
    constexpr int GB = KV8_PAGE * HD;
    constexpr int IPT = 2 * NC;                // DMA instructions of a wave a step: its page's K and V
    __shared__ __attribute__((aligned(1024))) uint8_t s_kv[S][4][2][GB];
    __shared__ __attribute__((aligned(16))) int s_page[SEG];
    __shared__ __attribute__((aligned(16))) float s_ks[SEG], s_vs[SEG];

    const int hkv = w.c.kv_heads;
    const int tid = threadIdx.x, lane = tid & 63;
    const int wave = __builtin_amdgcn_readfirstlane(tid >> 6);
    const int r = lane & 15, g = lane >> 4;
    // Workgroups go round-robin to the eight XCDs: a (sequence, KV head) keeps
    // to one, whose L2 then serves its tiles.  Tiles that see the most keys
    // start first.
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
    const int part = rest % w.parts, tile = w.tiles - 1 - (int)(rest / w.parts);
    const int kvh = u % hkv, i = u / hkv;
    const unsigned unit = u * w.tiles + tile;
    const Kv8Tile t = kv8_tile(w, i, tile);
    if (t.t0 >= t.rows || part >= t.parts) return;
    const int k_lo = part * w.part_keys, k_hi = min(t.end, k_lo + w.part_keys);

    const int wr0 = t.t0 + wave * RW;
    Kv8Rows<T, HD, QT> rows;
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
            // a page that is none: another's codes, not used
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
        for (int p = 0; p < S - 1 && p < steps; ++p) dma(p, p);
        int buf = 0;
        for (int it = 0; it < steps; ++it) {
            // this wave's part of step `it` has landed, then every wave's has
            // and every wave is done with the buffer that is filled next
            if (steps - 1 - it >= 1) attn_wait_vmcnt<IPT>();
            else attn_wait_vmcnt<0>();
            __syncthreads();
            if (it + S - 1 < steps) dma(it + S - 1, buf == 0 ? S - 1 : buf - 1);
            const int k0 = seg + it * 64;
#pragma unroll
            for (int half = 0; half < 2; ++half) {
                if (k0 + 32 * half >= rows.end) break;    // nothing that a row of this wave sees
                uint4 kc[2][NC], vc[2][NC];
                float ks[2], vs[2];
                bool there[2];
#pragma unroll
                for (int x = 0; x < 2; ++x) {
                    const int pg = 2 * half + x;
#pragma unroll
                    for (int c = 0; c < NC; ++c) {
                        kc[x][c] = *reinterpret_cast<const uint4*>(&s_kv[buf][pg][0][1024 * c + lane * 16]);
                        vc[x][c] = *reinterpret_cast<const uint4*>(&s_kv[buf][pg][1][1024 * c + lane * 16]);
                    }
                    there[x] = __builtin_amdgcn_readfirstlane(s_page[4 * it + pg]) >= 0;
                    ks[x] = s_ks[4 * it + pg];
                    vs[x] = s_vs[4 * it + pg];
                }
                rows.step(kc, vc, ks, vs, there, k0 + 32 * half, t.len, w.scale_log2, lane);
            }
            buf = buf == S - 1 ? 0 : buf + 1;
        }
    }
#pragma unroll
    for (int qt = 0; qt < QT; ++qt) {
        const float sum = attn_sum_xor16_32(rows.sum[qt]);
        const int row = wr0 + 16 * qt + r;
        if (row >= t.rows) continue;
        const float inv = t.parts > 1 ? 1.f : sum == 0.f ? 0.f : 1.f / sum;
        const size_t to = ((size_t)unit * w.parts + part) * (4 * RW) + (row - t.t0);
        T* const out = kv8_out<T, HD>(w, t, kvh, row);
#pragma unroll
        for (int c = 0; c < NC; ++c)
#pragma unroll
            for (int v = 0; v < 4; ++v) {
                const int d = 64 * c + 16 * g + 4 * v;
                const f32x4 o = {rows.acc[qt][4 * c][v] * inv, rows.acc[qt][4 * c + 1][v] * inv,
                                 rows.acc[qt][4 * c + 2][v] * inv, rows.acc[qt][4 * c + 3][v] * inv};
                if (t.parts == 1) st4<T>(out + d, o[0], o[1], o[2], o[3]);
                else *reinterpret_cast<f32x4*>(w.part_o + to * HD + d) = o;
            }
        if (t.parts > 1 && g == 0) { w.part_ml[2 * to] = rows.mx[qt]; w.part_ml[2 * to + 1] = sum; }
    }
}

// Joins the parts of a row's keys, in their order: a wave a row, HD / 4 lanes
// across it and the others taking further parts.
template <typename T, int HD>
__global__ __launch_bounds__(256) void kv8_join_kernel(Kv8AttnKernelArgs w)
{
    constexpr int LPR = HD / 4, PG = 64 / LPR;
    __shared__ float s_w[4][KV8_MAX_PARTS];
    const int lane = threadIdx.x & 63;
    const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    const unsigned per = (w.tile_rows + 3) / 4;
    const unsigned unit = blockIdx.x / per;
    const int row = (blockIdx.x % per) * 4 + wave;
    unsigned id = unit;
    const int tile = id % w.tiles;
    id /= w.tiles;
    const int kvh = id % w.c.kv_heads, i = id / w.c.kv_heads;
    const Kv8Tile t = kv8_tile(w, i, tile);
    if (t.parts == 1 || row >= w.tile_rows || t.t0 + row >= t.rows) return;
    const size_t base = (size_t)unit * w.parts * w.tile_rows + row;
    float m = -INFINITY;
    for (int p = lane; p < t.parts; p += 64) m = fmaxf(m, w.part_ml[2 * (base + (size_t)p * w.tile_rows)]);
    const float M = wave_max(m);
    float l = 0.f;
    for (int p = lane; p < t.parts; p += 64) {
        const float* ml = w.part_ml + 2 * (base + (size_t)p * w.tile_rows);
        const float wt = ml[0] == -INFINITY ? 0.f : fast_exp2(ml[0] - M);
        s_w[wave][p] = wt;
        l += wt * ml[1];
    }
    const float L = wave_sum(l);
    asm volatile("s_waitcnt lgkmcnt(0)" ::: "memory");   // the wave's own s_w
    const int d = lane % LPR * 4;
    f32x4 o = {0.f, 0.f, 0.f, 0.f};
#pragma unroll 4
    for (int p = lane / LPR; p < t.parts; p += PG)
        o += s_w[wave][p] * *reinterpret_cast<const f32x4*>(w.part_o + (base + (size_t)p * w.tile_rows) * HD + d);
#pragma unroll
    for (int v = 0; v < 4; ++v) {
        if (PG == 4) o[v] += swz_xor16_f(o[v]);
        o[v] += __shfl_xor(o[v], 32, 64);
    }
    const float inv = L == 0.f ? 0.f : 1.f / L;
    if (lane < LPR) st4<T>(kv8_out<T, HD>(w, t, kvh, t.t0 + row) + d, o[0] * inv, o[1] * inv, o[2] * inv, o[3] * inv);
}

// ------------------------------------------------------- plans, launches --

static Kv8Plan kv8_plan(const ebrl_kv8_cache& c, const ebrl_kv8_attn_args& a) {
    Kv8Plan p;
    const int64_t rows = (int64_t)a.max_q_len * (a.q_heads / c.kv_heads);
    p.decode = rows <= 16;
    p.tile_rows = p.decode ? 16 : a.dtype == EBRL_DTYPE_FP32 ? 64 : 128;
    p.tiles = (int)((rows + p.tile_rows - 1) / p.tile_rows);
    const int64_t units = (int64_t)a.n * c.kv_heads * p.tiles;
    const int least = p.decode ? 512 : 512, step = p.decode ? 128 : 64;
    int64_t want = p.decode ? (1024 + units - 1) / units : 512 / units;
    want = std::min<int64_t>(std::min<int64_t>(want, KV8_MAX_PARTS), (a.max_kv_len + least - 1) / least);
    want = std::max<int64_t>(want, 1);
    const int64_t keys = ((int64_t)a.max_kv_len + want - 1) / want;
    p.part_keys = (int)std::max<int64_t>(step, (keys + step - 1) / step * step);
    p.parts = (int)std::max<int64_t>(1, ((int64_t)a.max_kv_len + p.part_keys - 1) / p.part_keys);
    return p;
}

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
static void kv8_attn_launch(const Kv8Plan& p, const Kv8AttnKernelArgs& w, int64_t units, hipStream_t s) {
    constexpr int QT = sizeof(T) == 4 ? 1 : 2;
    const dim3 grid((unsigned)(units * p.parts)), wg(256);
    if (p.decode) hipLaunchKernelGGL((kv8_decode_kernel<T, HD>), grid, wg, 0, s, w);
    else hipLaunchKernelGGL((kv8_prompt_kernel<T, HD, QT>), grid, wg, 0, s, w);
    if (p.parts > 1)
        hipLaunchKernelGGL((kv8_join_kernel<T, HD>), dim3((unsigned)(units * ((p.tile_rows + 3) / 4))), wg, 0, s, w);
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
    return units * p.parts * p.tile_rows * (cache->head_dim + 2) * 4;
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
    const int64_t units = (int64_t)a.n * cache->kv_heads * p.tiles;
    if (units * std::max(p.parts, (p.tile_rows + 3) / 4) > KV8_MAX_GROUPS) return EBRL_E_INVALID;
    Kv8AttnKernelArgs w;
    w.c = *cache;
    w.a = a;
    w.grp = a.q_heads / cache->kv_heads;
    w.tiles = p.tiles;
    w.tile_rows = p.tile_rows;
    w.parts = p.parts;
    w.part_keys = p.part_keys;
    w.scale_log2 = a.scale * 1.4426950408889634f;
    w.part_o = (float*)a.workspace;
    w.part_ml = need ? w.part_o + units * p.parts * p.tile_rows * hd : nullptr;
    hipStream_t s = (hipStream_t)stream;
    if (esz == 2) {
        if (hd == 64) kv8_attn_launch<bf16_t, 64>(p, w, units, s);
        else kv8_attn_launch<bf16_t, 128>(p, w, units, s);
    } else {
        if (hd == 64) kv8_attn_launch<float, 64>(p, w, units, s);
        else kv8_attn_launch<float, 128>(p, w, units, s);
    }
    return hipGetLastError() == hipSuccess ? EBRL_OK : EBRL_E_HIP;
}

}  // extern "C"

// Projections in 8-bit integers (include/ebrl_i8.h): rows to codes, and the
// product of two operands of codes.
#include <hip/hip_runtime.h>

#include <type_traits>

#include "../../include/ebrl.h"
#include "../../include/ebrl_i8.h"
#include "kernels.h"

namespace ebrl {

typedef int i32x4 __attribute__((ext_vector_type(4)));

constexpr int I8_MAX_COLS = 1 << 20;
constexpr int I8_MAX_K = 131056;            // 2^14 K < 2^31, K a multiple of 16
constexpr int64_t I8_MAX_LD = 1 << 23;      // a tile's byte offsets are 32-bit numbers
constexpr int64_t I8_MAX_TILES = 1 << 23;

// ------------------------------------------------------- rows to codes --
// y in 64 bits: a code is off by one where y / s is nearer to a border than its
// error, and one such code moves a product by about 1e-4 of its size.  With 32-bit
// y that is a code in 1e5, with 64-bit ones none.

EBRL_DEV double i8_value(int op, float x, float up, double factor, float gain) {
    if (op == EBRL_I8_RMSNORM) return (double)x * factor * (double)gain;
    if (op == EBRL_I8_SWIGLU) return (double)x / (1.0 + exp(-(double)x)) * (double)up;
    return (double)x;
}
EBRL_DEV double i8_wave_max(double v) {
#pragma unroll
    for (int m = 1; m < 64; m <<= 1) v = fmax(v, __shfl_xor(v, m, 64));
    return v;
}
EBRL_DEV double i8_wave_sum(double v) {
#pragma unroll
    for (int m = 1; m < 64; m <<= 1) v += __shfl_xor(v, m, 64);
    return v;
}

template <typename T>
__global__ __launch_bounds__(256) void i8_quant_kernel(ebrl_i8_quant_args a)
{
    __shared__ double red[4];
    const int row = blockIdx.x, tid = threadIdx.x, wave = tid >> 6;
    const T* x = (const T*)a.x + (size_t)row * a.ldx;
    const T* up = a.op == EBRL_I8_SWIGLU ? (const T*)a.up + (size_t)row * a.ldup : nullptr;
    auto value = [&](int j, double factor) {
        return i8_value(a.op, ld_elem<T>(x + j), up ? ld_elem<T>(up + j) : 0.f, factor, a.gain ? a.gain[j] : 1.f);
    };
    double factor = 1.0;
    if (a.op == EBRL_I8_RMSNORM) {
        double ss = 0.0;
        for (int j = tid; j < a.cols; j += 256) {
            const double v = ld_elem<T>(x + j);
            ss += v * v;
        }
        ss = i8_wave_sum(ss);
        if ((tid & 63) == 0) red[wave] = ss;
        __syncthreads();
        factor = 1.0 / sqrt((red[0] + red[1] + red[2] + red[3]) / a.cols + (double)a.eps);
        __syncthreads();
    }
    double top = 0.0;
    bool bad = false;
    for (int j = tid; j < a.cols; j += 256) {
        const double v = fabs(value(j, factor));
        bad |= !(v <= 1.7976931348623157e308);
        top = fmax(top, v);
    }
    top = i8_wave_max(top);
    if ((tid & 63) == 0) red[wave] = top;
    bad = __syncthreads_or(bad);
    top = fmax(fmax(red[0], red[1]), fmax(red[2], red[3]));
    const float s = fmaxf((float)(top / 127.0), 0x1p-100f);
    bad |= !(s <= 3.40282347e38f);
    if (tid == 0) a.scales[row] = bad ? __builtin_nanf("") : s;
    int8_t* out = a.codes + (size_t)row * a.ldc;
    for (int j = tid; j < (a.cols + 15) / 16 * 16; j += 256)
        out[j] = j < a.cols && !bad ? (int8_t)(int)rint(value(j, factor) / (double)s) : (int8_t)0;
}

// -------------------------------------------------------------- product --

// One element's epilogue and its store; `m`, `n` inside.
template <typename T> struct I8Epi {
    const float *scale_a, *scale_b, *bias;
    const T* residual;
    T* c;
    int64_t ldr, ldc;
    EBRL_DEV void operator()(int m, int n, int sum) const {
#pragma clang fp contract(off)
        float v = (float)sum * scale_b[n] * scale_a[m];
        if (bias) v += bias[n];
        if (residual) v += ld_elem<T>(residual + (size_t)m * ldr + n);
        st_elem<T>(c + (size_t)m * ldc + n, v);
    }
};

// 64 x 64 tiles on four waves of 32 x 32, K 64 at a time through LDS.  The
// weights' rows are the first operand: a lane (r, g) of
// v_mfma_i32_16x16x64_i8 gives bytes 16 g .. of row r, and gets outputs n = 4 g ..
// of row m = r.
template <typename T>
__global__ __launch_bounds__(256) void i8_gemm_kernel(const int8_t* __restrict__ A, int64_t lda,
                                                      const int8_t* __restrict__ B, int64_t ldb, int M, int N, int K,
                                                      I8Epi<T> epi)
{
    __shared__ __attribute__((aligned(16))) int8_t sA[64 * 80], sB[64 * 80];
    const int tid = threadIdx.x, lane = tid & 63, wave = tid >> 6;
    const int tiles_n = (N + 63) / 64;
    const int m0 = blockIdx.x / tiles_n * 64, n0 = blockIdx.x % tiles_n * 64;
    const int wm = wave >> 1, wn = wave & 1, r = lane & 15, g = lane >> 4;
    const int row = tid >> 2, ch = tid & 3;
    const int8_t* pa = A + (size_t)min(m0 + row, M - 1) * lda + ch * 16;
    const int8_t* pb = B + (size_t)min(n0 + row, N - 1) * ldb + ch * 16;
    i32x4 acc[2][2] = {};
    for (int k = 0; k < K; k += 64) {
        i32x4 va = {}, vb = {};
        if (k + ch * 16 < K) {
            va = *reinterpret_cast<const i32x4*>(pa + k);
            vb = *reinterpret_cast<const i32x4*>(pb + k);
        }
        __syncthreads();
        *reinterpret_cast<i32x4*>(sA + row * 80 + ch * 16) = va;
        *reinterpret_cast<i32x4*>(sB + row * 80 + ch * 16) = vb;
        __syncthreads();
        i32x4 fa[2], fb[2];
#pragma unroll
        for (int i = 0; i < 2; ++i) {
            fa[i] = *reinterpret_cast<const i32x4*>(sA + (wm * 32 + i * 16 + r) * 80 + g * 16);
            fb[i] = *reinterpret_cast<const i32x4*>(sB + (wn * 32 + i * 16 + r) * 80 + g * 16);
        }
#pragma unroll
        for (int i = 0; i < 2; ++i)
#pragma unroll
            for (int j = 0; j < 2; ++j)
                acc[i][j] = __builtin_amdgcn_mfma_i32_16x16x64_i8(fb[j], fa[i], acc[i][j], 0, 0, 0);
    }
#pragma unroll
    for (int i = 0; i < 2; ++i)
#pragma unroll
        for (int j = 0; j < 2; ++j)
#pragma unroll
            for (int e = 0; e < 4; ++e) {
                const int m = m0 + wm * 32 + i * 16 + r, n = n0 + wn * 32 + j * 16 + 4 * g + e;
                if (m < M && n < N) epi(m, n, acc[i][j][e]);
            }
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

static int i8_quant(const ebrl_i8_quant_args* args, hipStream_t s) {
    if (!args) return EBRL_E_INVALID;
    const ebrl_i8_quant_args& a = *args;
    if (!i8_dtype_ok(a.dtype) || a.op < EBRL_I8_ROWS || a.op > EBRL_I8_SWIGLU || a.rows < 0 || a.cols < 1 ||
        a.cols > I8_MAX_COLS || (a.op == EBRL_I8_RMSNORM && !(a.eps >= 0.f)) || (a.op != EBRL_I8_SWIGLU && a.up) ||
        (a.op != EBRL_I8_RMSNORM && a.gain))
        return EBRL_E_INVALID;
    if (a.rows == 0) return EBRL_OK;
    const int esz = i8_size(a.dtype);
    if (!i8_rows_ok(a.x, a.ldx, a.cols, esz) || (a.op == EBRL_I8_SWIGLU && !i8_rows_ok(a.up, a.ldup, a.cols, esz)) ||
        (uintptr_t)a.gain % 4 || !i8_codes_ok(a.codes, a.ldc, (a.cols + 15) / 16 * 16) || a.ldc >= ((int64_t)1 << 40) ||
        !a.scales || (uintptr_t)a.scales % 4)
        return EBRL_E_INVALID;
    if (esz == 2) hipLaunchKernelGGL(i8_quant_kernel<bf16_t>, dim3(a.rows), dim3(256), 0, s, a);
    else hipLaunchKernelGGL(i8_quant_kernel<float>, dim3(a.rows), dim3(256), 0, s, a);
    return hipGetLastError() == hipSuccess ? EBRL_OK : EBRL_E_HIP;
}

static bool i8_shape_ok(const ebrl_i8_gemm_args* a) {
    return a && i8_dtype_ok(a->dtype) && a->M >= 0 && a->N >= 0 && a->K >= 16 && a->K % 16 == 0 && a->K <= I8_MAX_K &&
           (((int64_t)a->M + 31) / 32) * (((int64_t)a->N + 63) / 64) <= I8_MAX_TILES;
}

template <typename T> static void i8_gemm_launch(const ebrl_i8_gemm_args& a, hipStream_t s) {
    const I8Epi<T> epi{a.scale_a, a.scale_b, a.bias, (const T*)a.residual, (T*)a.c, a.ldr, a.ldc};
    const unsigned tiles = (unsigned)((((int64_t)a.M + 63) / 64) * (((int64_t)a.N + 63) / 64));
    hipLaunchKernelGGL(i8_gemm_kernel<T>, dim3(tiles), dim3(256), 0, s, a.a, a.lda, a.b, a.ldb, a.M, a.N, a.K, epi);
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
    if (esz == 2) i8_gemm_launch<bf16_t>(a, s);
    else i8_gemm_launch<float>(a, s);
    return hipGetLastError() == hipSuccess ? EBRL_OK : EBRL_E_HIP;
}

}  // namespace ebrl

extern "C" {

int ebrl_op_i8_quant(const ebrl_i8_quant_args* args, void* stream) { return ebrl::i8_quant(args, (hipStream_t)stream); }

int64_t ebrl_op_i8_gemm_workspace(const ebrl_i8_gemm_args* args) { return ebrl::i8_shape_ok(args) ? 0 : EBRL_E_INVALID; }

int ebrl_op_i8_gemm(const ebrl_i8_gemm_args* args, void* stream) { return ebrl::i8_gemm(args, (hipStream_t)stream); }

}  // extern "C"

/*
 * ebrl_i8.h -- projections in 8-bit integers: rows quantised to codes with a
 * scale for each, and the matrix product of two such operands.
 *
 * Paper: the generation stage's projections (Section 2.1's backbone and action
 * heads) at half the weight bytes and twice the matrix rate of bf16.  Same
 * conventions as ebrl.h: device pointers, stream-ordered calls, status codes; a
 * call allocates nothing, synchronises nothing and may be captured into a HIP
 * graph.
 *
 * An operand is rows of K codes, int8, and a float scale for each row: the value
 * is code * scale.  Activations have a row a token; weights, stored [out, in] as
 * everywhere in this library, a row an output channel (ebrl_op_i8_quant makes
 * both).  K is a multiple of 16: a width that is none is filled up with zeros.
 */
#ifndef EBRL_I8_H
#define EBRL_I8_H

#include <stdint.h>

#ifdef __cplusplus
extern "C" {
#endif

/* What is quantised: rows y of `cols` values */
enum {
    EBRL_I8_ROWS = 0,      /* y = x */
    EBRL_I8_RMSNORM = 1,   /* y = gain x / sqrt(mean x^2 + eps), the pre-norm of a block */
    EBRL_I8_SWIGLU = 2     /* y = x / (1 + exp(-x)) up: x the gate's rows */
};

typedef struct ebrl_i8_quant_args {
    int32_t dtype;           /* EBRL_DTYPE_FP32 or _BF16: type of x and up */
    int32_t op;              /* EBRL_I8_* */
    int32_t rows, cols;      /* cols 1 to 2^20 */
    float eps;               /* EBRL_I8_RMSNORM: >= 0, finite */
    const void *x, *up;      /* device rows; up: EBRL_I8_SWIGLU alone */
    int64_t ldx, ldup;       /* row strides in elements, >= cols */
    const float* gain;       /* device [cols] (EBRL_I8_RMSNORM), or NULL: ones */
    int8_t* codes;           /* device rows, 16-byte aligned */
    int64_t ldc;             /* row stride in bytes, a multiple of 16, >= cols rounded up to one */
    float* scales;           /* device [rows] */
} ebrl_i8_quant_args;

/* For each row: scale = max |y| / 127 rounded to a float, 2^-100 at least, and
 * code = y / scale rounded to the nearest whole number, ties to the even one.
 * y, its maximum and the quotients are computed in 64 bits, so that codes and
 * scales are those of the formulas.  The bytes from cols up to the next multiple
 * of 16 are set to zero, those behind it left as they were.  A row that holds a
 * value that is not finite, or whose scale would not be, gets codes of zero and
 * the scale NaN: its products are NaN.  Rows of x (and up) may have any stride
 * and the alignment of an element; 16-byte aligned ones are read faster.  codes and
 * scales must not overlap the inputs.  Returns EBRL_E_INVALID on bad arguments. */
int ebrl_op_i8_quant(const ebrl_i8_quant_args* args, void* stream);

typedef struct ebrl_i8_gemm_args {
    int32_t dtype;           /* EBRL_DTYPE_FP32 or _BF16: type of c and residual */
    int32_t M, N, K;         /* K: a multiple of 16, at most 131056 */
    const int8_t *a, *b;     /* device codes [M, K] and [N, K], 16-byte aligned */
    int64_t lda, ldb;        /* row strides in bytes: multiples of 16, >= K, below 2^23 */
    const float *scale_a, *scale_b;   /* device [M], [N] */
    const float* bias;       /* device [N], or NULL */
    const void* residual;    /* device [M, N], or NULL; may be c itself (with ldr = ldc) */
    int64_t ldr;             /* row stride in elements, >= N */
    void* c;                 /* device [M, N] */
    int64_t ldc;             /* row stride in elements, >= N */
    void* workspace;         /* device, 16-byte aligned; NULL where none is needed */
    int64_t workspace_bytes;
} ebrl_i8_gemm_args;

/* Bytes of workspace that a product of this size needs (host arithmetic on M, N
 * and K; no pointer is read), or EBRL_E_INVALID.  0: none.  A smaller M may need
 * more. */
int64_t ebrl_op_i8_gemm_workspace(const ebrl_i8_gemm_args* args);

/* The kernel that computes a product, for tests and timings that have to know which
 * one they reach; host arithmetic, no GPU needed.  plan[0] 0: 256 x 256 tiles, 1: LDS
 * ring, 2: decode; [1], [2] tile rows and columns (decode: rows loaded); [3] ranges
 * that K is cut into; [4] workgroups; [5] kernel 0: the parts each tile of the last
 * round is cut into.  Returns EBRL_E_INVALID on bad arguments. */
int ebrl_op_i8_gemm_plan(int32_t M, int32_t N, int32_t K, int32_t plan[6]);

/* c[m, n] = scale_a[m] scale_b[n] sum_k a[m, k] b[n, k] + bias[n] + residual[m, n].
 * The sum is exact (32-bit integers, which K's bound keeps from overflowing, codes
 * of -128 among them); it is rounded to a float, multiplied by scale_b, then by
 * scale_a, and bias and residual are added, each step rounded to 32 bits, the
 * result to c's type.  Results do not depend on the size of the call, the stream
 * or its compute units.  c, its residual and bias need the alignment of an element;
 * 16-byte aligned rows are stored faster.  c must not overlap the inputs but for
 * residual = c.
 *
 * The workspace holds partial sums where few outputs have a long K; what is in it
 * before a call does not matter.  Calls that may overlap in time need a workspace
 * each.  Returns EBRL_E_INVALID on bad arguments, too small a workspace, or where
 * the outputs are more than 2^23 tiles of 32 x 64. */
int ebrl_op_i8_gemm(const ebrl_i8_gemm_args* args, void* stream);

#ifdef __cplusplus
}
#endif
#endif /* EBRL_I8_H */

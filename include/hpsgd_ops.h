/*
 * libhpsgd, operators: what a program that trains or runs a language model needs beside the
 * replica update and the merge of hpsgd.h: the optimizer step over many tensors, and the layer in 8-bit
 * floating point that its gradients come from (norm, quantisation, matrix product).
 * (The HPSGD paper has no counterpart for any of them.)
 *
 * Conventions (in addition to those of hpsgd.h)
 *   - The operators need no hpsgd_init and keep nothing of a call: every buffer is the caller's, and work
 *     is enqueued on the stream that is given (a cudaStream_t; NULL = the default stream) and on
 *     no other.  They allocate nothing and wait for nothing, so they can be captured in a graph.  Like the
 *     rest of the library they are called from one host thread (the text of the last error, the launch count
 *     and what a device holds at a time are the process's).
 *   - Structs and arrays of structs are HOST memory, read during the call; the pointers in them
 *     are DEVICE pointers.
 *   - Arguments are checked before anything is enqueued.  A size of zero is legal and does nothing
 *     unless the call says otherwise.
 *   - Every reduction has a fixed order: the same inputs give the same bits.
 *   - Sums, moments and statistics are held in binary32 or wider whatever the stored types.
 *
 * The 8-bit block format.  128 consecutive values share one power of two.  A value is an E4M3 code
 * (1 sign, 4 exponent and 3 mantissa bits, largest magnitude 448, no infinity) times 2^e, where e is
 * the smallest integer >= -127 with 448 * 2^e >= the largest finite magnitude of the block; the scale
 * is stored as the byte e + 127 (E8M0).  The codes have an exponent of their own, so the relative
 * precision does not depend on where in its octave the scale lies: a power of two loses nothing
 * against an arbitrary factor, multiplying by it is exact, and values can be moved to blocks along the
 * other axis without being rounded again (except where they fall below the smallest code).  Values
 * that are not finite become the NaN code 0x7F and do not count for the scale.
 *
 * A matrix [rows x cols] in this format (its blocks run along the columns):
 *   codes    one byte each, row r at r * ld; ld >= cols, a multiple of 16, the address 16-byte aligned; the
 *            codes behind the last column, up to a multiple of 16, are written as zeros
 *   scales   the byte of block b of row r at ((b / 4) * lds + r) * 4 + b % 4, lds >= rows (four blocks make a
 *            32-bit word, and the words of consecutive rows follow one another); 4-byte aligned,
 *            ceil(ceil(cols / 128) / 4) * lds * 4 bytes; the bytes behind a row's last block are written as zeros
 */
#ifndef HPSGD_OPS_H_
#define HPSGD_OPS_H_

#include "hpsgd.h"

#ifdef __cplusplus
extern "C" {
#endif

/* ------------------------------------------------------------------------------------
 * AdamW over many tensors.
 * ---------------------------------------------------------------------------------- */

/*
 * One tensor of a step.  Element pointers need the alignment of their element; where the addresses
 * of param, grad and copy are multiples of 32 bytes (16 for bf16) and those of the moments of 32 bytes
 * (8 for 8-bit codes) the wide accesses are used, for that tensor alone.
 *   param         n values of the call's param_dtype, updated in place
 *   grad          n values of the call's grad_dtype
 *   m, v          state_bits 32: n floats each.  state_bits 8: n codes each; v holds the SQUARE ROOT of
 *                 the second moment.  All zero (codes and scales too) is the state before the first step.
 *   m_scale, v_scale   state_bits 8 only: ceil(n / 128) scale bytes each, block b covering the elements
 *                 [128 b, 128 b + 128)
 *   copy          n bf16 values that receive the new parameters rounded to nearest even (the copy a
 *                 bf16 forward pass reads), or NULL.  Only with param_dtype HPSGD_F32.
 *   weight_decay  decoupled decay of this tensor, >= 0
 *   rng_offset    position of the tensor's first element in the step's sequence of random bits: give
 *                 tensors of one step disjoint ranges [rng_offset, rng_offset + n)
 */
typedef struct hpsgd_adamw_tensor {
    void* param;
    const void* grad;
    void* m;
    void* v;
    uint8_t* m_scale;
    uint8_t* v_scale;
    void* copy;
    int64_t n;
    uint64_t rng_offset;
    double weight_decay;
} hpsgd_adamw_tensor;

/*
 * One AdamW step of every tensor, in as few launches as the table takes (one up to 360 tensors):
 *     g = grad * c                                    c = *grad_scale, 1 if NULL
 *     m = beta1 m + (1 - beta1) g
 *     v = beta2 v + (1 - beta2) g^2
 *     p = p (1 - lr weight_decay) - lr / (1 - beta1^step) * m / (sqrt(v) / sqrt(1 - beta2^step) + eps)
 * in binary32; the factors that do not depend on the element are computed in binary64 and rounded once.
 *
 * If grad_scale points to a value that is not finite (hpsgd_grad_norm writes one when the norm is not)
 * the call changes nothing: a step whose gradients overflowed is skipped without the host having to look.
 *
 * state_bits 8: the moments are read from and written to the 8-bit block format, m as it is and v as
 * r = sqrt(v), which halves the range that the codes have to span.  The parameter is stepped with the new
 * moments before they are rounded.  Rounding is stochastic, with 16 random bits for each: to nearest, an
 * average with beta2 = 0.999 that moves by 0.1 % a step would never leave a code whose neighbours are 6 to
 * 12 % away.  m goes to one of its two neighbours so that the expected value is m, r so that the expected
 * SQUARE is v; a positive v is never rounded to 0, which would leave eps alone to divide by.
 * param_dtype HPSGD_BF16: the new parameter is rounded stochastically to bf16 too, for the same reason.
 *
 * The 32 random bits x of element i (position q = rng_offset + i, all in uint32 arithmetic):
 *     key = mix(mix(mix(seed + M3) ^ step) + M4)      mix and M1..M4 as for hpsgd_gen_grads (64 bits)
 *     x = ((uint32)q ^ (uint32)key) * N1;  x ^= x >> 15;  x = (x + (uint32)(key >> 32) + (uint32)(q >> 32) * N3) * N2
 *     x ^= x >> 14;  x *= N3;  x ^= x >> 16           N1..N3 = frac(sqrt 2, 3, 5) * 2^32 with the low bit set
 * the upper 16 are m's, the lower 16 r's, and the upper 16 of x * N2 a bf16 parameter's.
 *
 * beta1, beta2 in [0, 1), eps >= 2^-126, lr >= 0, step >= 1 (the first step is 1).
 */
int hpsgd_adamw_step(const hpsgd_adamw_tensor* tensors, int n_tensors, int param_dtype, int grad_dtype, int state_bits,
                     double lr, double beta1, double beta2, double eps, int64_t step, uint64_t seed,
                     const float* grad_scale, void* stream);

/*
 * Global norm of the gradients of a table (only grad and n are read) and what clips it:
 *     out[0] = sqrt(sum over all tensors of grad^2)
 *     out[1] = max_norm / out[0] if out[0] > max_norm, else 1; NaN if the sum is not finite in binary32
 * Squares are added in binary32 eight at a time, those sums in binary64; the sum, its root and the quotient are rounded to binary32.  max_norm > 0; infinity is legal
 * (the norm alone).  `workspace`: HPSGD_GRAD_NORM_WORKSPACE bytes of device memory, 16-byte aligned, filled with
 * zeros before its first use; every call leaves it ready for the next.  Calls that share a workspace have to
 * be ordered on one stream.  Without tensors out is {0, 1}.
 */
#define HPSGD_GRAD_NORM_WORKSPACE 65536
int hpsgd_grad_norm(const hpsgd_adamw_tensor* tensors, int n_tensors, int grad_dtype, double max_norm,
                    void* workspace, float* out, void* stream);

/* ------------------------------------------------------------------------------------
 * Root-mean-square norm with the residual's addition and an 8-bit output.
 * ---------------------------------------------------------------------------------- */

/*
 * Per row of x [rows x cols]:
 *     h = x + residual            rounded to dtype, which is what is stored and what is normalised (the backward
 *                                 pass then sees the same numbers); h = x without a residual
 *     rstd = 1 / sqrt(mean(h^2) + eps)
 *     y = h * rstd * weight       in binary32, rounded once to what is stored
 *   dtype, weight_dtype   HPSGD_F32 or HPSGD_BF16
 *   residual, h     both or neither; h may be x's or the residual's own memory
 *   y8, y_scale     the 8-bit block format (both or neither);  y   values of dtype.  At least one of y8, y.
 *   rstd            rows floats, for the backward pass, or NULL
 *   ld*             elements (bytes for ldy8) from row to row; 0 = cols (for ldy8 cols up to a multiple of 16);
 *                   ldys: the lds of the scales, 0 = rows
 * Rows whose addresses and strides are multiples of 32 bytes (16 for bf16) take the wide accesses.  cols <= 16384
 * (else HPSGD_E_UNSUPPORTED).
 */
typedef struct hpsgd_rmsnorm_forward_args {
    int64_t rows, cols;
    double eps;
    int dtype, weight_dtype;
    const void* x;
    const void* residual;
    const void* weight;
    void* h;
    void* y;
    void* y8;
    uint8_t* y_scale;
    float* rstd;
    int64_t ldx, ldres, ldh, ldy, ldy8, ldys;
} hpsgd_rmsnorm_forward_args;
int hpsgd_rmsnorm_forward(const hpsgd_rmsnorm_forward_args* args, void* stream);

/*
 * Gradients of the norm, through its quantisation as if that were the identity.  With xn = h * rstd, d = dy * weight:
 *     dx = rstd * (d - xn * mean(d * xn)) + dres      the gradient of h, so of x and of the residual alike
 *     dweight = sum over rows of dy * xn              cols floats
 *   dy, dres, dx   values of dtype; dres (the gradient that reaches h by the residual stream) may be NULL; dx may be dy's
 *                  or dres's own memory
 *   workspace      hpsgd_rmsnorm_backward_bytes(rows, cols) bytes of device memory, 16-byte aligned; no contents needed
 * With rows = 0 dweight is set to zero.
 */
typedef struct hpsgd_rmsnorm_backward_args {
    int64_t rows, cols;
    int dtype, weight_dtype;
    const void* h;
    const void* weight;
    const float* rstd;
    const void* dy;
    const void* dres;
    void* dx;
    float* dweight;
    void* workspace;
    int64_t ldh, lddy, lddres, lddx;
} hpsgd_rmsnorm_backward_args;
size_t hpsgd_rmsnorm_backward_bytes(int64_t rows, int64_t cols);
int hpsgd_rmsnorm_backward(const hpsgd_rmsnorm_backward_args* args, void* stream);

/* ------------------------------------------------------------------------------------
 * To the 8-bit block format, along rows and along columns in one pass.
 * ---------------------------------------------------------------------------------- */

/*
 * x [rows x cols] -> q, scale: the matrix in the block format, and / or qt, scale_t: its transpose [cols x rows] in the
 * block format, whose blocks run along x's columns.  Rounding is to nearest even.
 *   dtype    HPSGD_F32, HPSGD_BF16, or HPSGD_FP8: x is itself in the block format (x_scale given; ldx bytes), and only the
 *            transpose can be asked for.  Moving to the other blocks is exact but for values below the new block's smallest code.
 *   ld*      elements (bytes for codes) from row to row; 0 = the least: cols for x, multiples of 16 for codes
 *   lds*     the lds of the scales, 0 = the rows of that matrix
 */
enum { HPSGD_FP8 = 2 };
typedef struct hpsgd_quantize_fp8_args {
    int64_t rows, cols;
    int dtype;
    const void* x;
    const uint8_t* x_scale;
    void* q;
    uint8_t* scale;
    void* qt;
    uint8_t* scale_t;
    int64_t ldx, ldxs, ldq, lds, ldqt, ldst;
} hpsgd_quantize_fp8_args;
int hpsgd_quantize_fp8(const hpsgd_quantize_fp8_args* args, void* stream);

/* ------------------------------------------------------------------------------------
 * Matrix product of two matrices in the 8-bit block format.
 * ---------------------------------------------------------------------------------- */

/*
 * D[m, n] = sum over k of A[m, k] B[n, k]      A [M x K] and B [N x K] in the block format, D of d_dtype, row-major
 * With x the input, w the weights [N x K] and dy the gradient of a layer's output, all three products of its training have this form:
 * y = (x, w); dx = (dy, w transposed); dw = (dy transposed, x transposed), the transposes from hpsgd_quantize_fp8.  With M = 1 (one
 * token) it streams the weights.
 *   Every product is exact, and they are added in binary32 (on the tensor cores, in an order that depends on the sizes alone).
 *   Values held as the NaN code make the results they enter NaN.
 *   d_dtype       HPSGD_F32 or HPSGD_BF16 (rounded once)
 *   accumulate    1: D += the product (HPSGD_F32 only), for gradients over several batches; one binary32 addition an element, subnormal numbers
 *                 included.  D is read and written like any other operand: calls that add to the same D have to be ordered
 *   ldd           elements from row to row of D, 0 = N; any alignment
 *   lda, ldb, ldsa, ldsb   as in hpsgd_quantize_fp8
 *   workspace     hpsgd_gemm_fp8_bytes(M, N, K) bytes of device memory (0 but for few rows and very long sums), 16-byte aligned; no contents needed.  Calls
 *                 that share a workspace have to be ordered on one stream.  workspace_bytes: its size.
 * K = 0 gives zeros.
 * The kernel waits for its own copies and products only, for two seconds at most (see hpsgd_ops_check).
 */
typedef struct hpsgd_gemm_fp8_args {
    int64_t M, N, K;
    const void* a;
    const uint8_t* a_scale;
    const void* b;
    const uint8_t* b_scale;
    void* d;
    void* workspace;
    size_t workspace_bytes;
    int64_t lda, ldsa, ldb, ldsb, ldd;
    int d_dtype, accumulate;
} hpsgd_gemm_fp8_args;
size_t hpsgd_gemm_fp8_bytes(int64_t M, int64_t N, int64_t K);
int hpsgd_gemm_fp8(const hpsgd_gemm_fp8_args* args, void* stream);

/*
 * Wait for `stream` and report what only the device can know: HPSGD_E_TIMEOUT if a wait inside hpsgd_gemm_fp8 ran out on this device
 * since the last call, HPSGD_E_CUDA if the work failed.  A tile of D (up to 256 rows and columns) whose waits ran out, in whichever of its parts
 * along k, is left as it was, and nothing is added to it; other tiles may have been written.  Products whose parts go through the workspace
 * write nothing from such a time-out on until it has been reported here (the whole device is waited for then).
 */
int hpsgd_ops_check(void* stream);

/*
 * Checked build only; HPSGD_E_UNSUPPORTED otherwise.  1: the barriers of hpsgd_gemm_fp8 are told to expect 16 bytes more than its copies
 * bring, so that its waits run out after two seconds: the way to see the time-out path (no results, HPSGD_E_TIMEOUT from
 * hpsgd_ops_check, the device usable as before) without a fault.  2: those of thread blocks with odd numbers only.
 */
int hpsgd_ops_debug_stall(int enable);

#ifdef __cplusplus
}
#endif

#endif /* HPSGD_OPS_H_ */

/*
 * libhpsgd, operators: what a program that trains or runs a language model needs beside the
 * replica update and the merge of hpsgd.h: the optimizer step over many tensors, the layer in 8-bit
 * floating point that its gradients come from (norm, quantisation, matrix product, gated feed-forward
 * layer), a gated recurrence over sequences, and the loss.
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

/* ------------------------------------------------------------------------------------
 * A gated linear recurrence over sequences.
 * ---------------------------------------------------------------------------------- */

/*
 * Rows are tokens, columns channels; per channel, with h in front of a sequence's first row its h0 (0 without):
 *     a = sigmoid(f)
 *     h = a h' + (1 - a) v        h' the row before
 *     y = h * sigmoid(o)          y = h without o
 * in binary32, y rounded once.  With rows == sequences it is a step of one token for each.
 *   dtype      of f, v, o, y: HPSGD_F32 or HPSGD_BF16
 *   offsets    DEVICE memory, sequences + 1 numbers: sequence s has the rows [offsets[s], offsets[s + 1]).  They have to ascend (equal ones: a
 *              sequence without rows, whose state goes through) and lie in [0, rows]; others give undefined results, but no access outside the
 *              call's memory.  Rows in front of the first sequence and behind the last are neither read nor written; a padded batch is one in which the padding
 *              of each sequence is a sequence too.  NULL: sequences of rows / sequences rows each (rows a multiple of sequences)
 *   h0         [sequences x cols], or NULL
 *   h_last     [sequences x cols], receives the state behind each sequence, or NULL; may be h0's own memory
 *   saved      hpsgd_gated_scan_saved_bytes(rows, cols) bytes for the backward pass, 16-byte aligned, or NULL
 *   ld*        elements from row to row; 0 = cols.  f, v and o may lie side by side in one matrix.
 * Rows whose addresses and strides are multiples of 16 bytes (of two elements for y, and for what the backward call writes) are copied ahead of their use;
 * others are read value by value, which takes about four times as long.  A state that is updated in place is no longer there for the backward call's h0.
 */
typedef struct hpsgd_gated_scan_forward_args {
    int64_t rows, cols, sequences;
    int dtype;
    const void* f;
    const void* v;
    const void* o;
    const int64_t* offsets;
    const float* h0;
    float* h_last;
    void* y;
    float* saved;
    int64_t ldf, ldv, ldo, ldy, ldh0, ldlast;
} hpsgd_gated_scan_forward_args;
size_t hpsgd_gated_scan_saved_bytes(int64_t rows, int64_t cols);
int hpsgd_gated_scan_forward(const hpsgd_gated_scan_forward_args* args, void* stream);

/*
 * Its gradients.  With g = dy sigmoid(o), to which dh_last is added in a sequence's last row, and G = g + a'' G'' ('' the row behind; nothing
 * comes into a sequence's last row):
 *     dv = G (1 - a)      df = G (h' - v) a (1 - a)      do = dy h sigmoid(o) (1 - sigmoid(o))      dh0 = a G of the first row
 *   f, v, o, offsets, h0   as in the forward call; saved: what it left
 *   dy, df, dv, d_o        values of dtype.  df, dv and d_o may each be, element for element, the memory of f, v, o or dy.
 *   dh_last                gradient of h_last, or NULL (0);  dh0: [sequences x cols], or NULL
 *   o and d_o              both or neither
 */
typedef struct hpsgd_gated_scan_backward_args {
    int64_t rows, cols, sequences;
    int dtype;
    const void* f;
    const void* v;
    const void* o;
    const int64_t* offsets;
    const float* h0;
    const float* saved;
    const void* dy;
    const float* dh_last;
    void* df;
    void* dv;
    void* d_o;
    float* dh0;
    int64_t ldf, ldv, ldo, ldh0, lddy, lddlast, lddf, lddv, lddo, lddh0;
} hpsgd_gated_scan_backward_args;
int hpsgd_gated_scan_backward(const hpsgd_gated_scan_backward_args* args, void* stream);

/* ------------------------------------------------------------------------------------
 * The loss over a label and a teacher's top logits.
 * ---------------------------------------------------------------------------------- */

/*
 * Per row z of logits [rows x vocab], with T the temperature:
 *     CE = lse(z) - z[label]                                                     lse(x) = log(sum exp(x))
 *     KL = sum over the teacher's entries j of p_j (log p_j - z[i_j] / T + lse(z / T))     p the softmax of the row's k teacher logits / T
 *     loss = label_weight CE + teacher_weight T^2 KL
 *     dlogits = c ( label_weight (softmax(z) - 1 at the label) + teacher_weight T (softmax(z / T) - p_j at i_j) )      c = grad_scale dloss[row]
 * in binary32; dlogits is rounded once.  Without a teacher it is cross-entropy.
 *   dtype, teacher_dtype   HPSGD_F32 or HPSGD_BF16, of logits and dlogits and of teacher_logits
 *   labels          rows numbers, or NULL; a negative one: the row has no label and no CE
 *   teacher_index, teacher_logits   [rows x k], k <= 1024 (else HPSGD_E_UNSUPPORTED); an entry whose index is negative or whose logit is
 *                   -infinity is not there, whatever stands in the other place, and a row without any has no KL.  Indices may repeat.
 *   loss            rows floats, or NULL;   lse: rows x 2 floats, lse(z) and lse(z / T), for the second call, or NULL
 *   dlogits         the gradient in the same pass, or NULL; may be the logits' own memory
 *   dloss           rows floats, the gradients of the rows' losses, or NULL (1).  Where c is 0, dlogits is 0 whatever the logits are.
 *   ld*             elements from row to row; 0 = vocab, for the teacher's two matrices k
 * Rows with neither label nor teacher have loss and gradient 0, whatever their logits are.  Logits of -infinity have probability 0 (a label or
 * a teacher's entry there makes the loss infinite); NaN and +infinity make their row NaN, and so does a label or an index that is not below vocab.
 * Finite logits may be of any size, a mask of the type's lowest value among them, in a part of a row or all over it, the teacher's too; rows whose largest
 * logit / T is beyond 2^20 log 2 take longer.
 * A term with weight 0 is left out: its arguments are not read.  Rows whose addresses and strides are multiples of 32 bytes (16 for bf16) take the wide
 * accesses.
 */
typedef struct hpsgd_distill_loss_args {
    int64_t rows, vocab, k;
    double temperature, label_weight, teacher_weight, grad_scale;
    int dtype, teacher_dtype;
    const void* logits;
    const int64_t* labels;
    const int32_t* teacher_index;
    const void* teacher_logits;
    float* loss;
    float* lse;
    void* dlogits;
    const float* dloss;
    int64_t ldlogits, ldteacher, lddlogits;
} hpsgd_distill_loss_args;
int hpsgd_distill_loss(const hpsgd_distill_loss_args* args, void* stream);

/*
 * dlogits alone, where dloss comes later: lse is what the first call wrote; loss is not touched.  An lse in binary32 carries half a unit of its last place into
 * every probability; beyond 2^20 log 2 the sums are taken from the logits again.
 */
int hpsgd_distill_loss_backward(const hpsgd_distill_loss_args* args, void* stream);

/* ------------------------------------------------------------------------------------
 * The gated feed-forward layer in the 8-bit block format.
 * ---------------------------------------------------------------------------------- */

/*
 * With x [M x K] and w [2 N x K] in the block format, w's first N rows the gate's weights and the others those of what it gates:
 *     g = x w[0..N)^T      u = x w[N..2N)^T      z = act(g) u        in binary32, z rounded once to what is stored
 *   act        HPSGD_SILU: g sigmoid(g).   HPSGD_GELU: g (1 + tanh(sqrt(2 / pi) (g + 0.044715 g^3))) / 2
 *   z8, z_scale    z [M x N] in the block format (both or neither): what the projection back takes;  z: values of z_dtype (HPSGD_F32 or HPSGD_BF16).
 *              At least one of z8, z.
 *   gu         [M x 2 N] bf16, receives g | u rounded, for the backward pass, or NULL
 *   ld*        as in hpsgd_quantize_fp8; ldz, ldgu: elements from row to row, 0 = N and 2 N
 * K >= 1.  With M = 1 (one token) it streams the weights.  Products are exact and added in binary32 on the tensor cores in an order that depends on the sizes alone
 * (a sum is off by about 2^-24 of the sum of its products' magnitudes); values held as the NaN code make the results they enter NaN.  The kernel waits for its own copies and products only, for two seconds at most (see hpsgd_ops_check).
 */
enum { HPSGD_SILU = 0, HPSGD_GELU = 1 };
typedef struct hpsgd_gated_ffn_forward_args {
    int64_t M, N, K;
    int act, z_dtype;
    const void* x;
    const uint8_t* x_scale;
    const void* w;
    const uint8_t* w_scale;
    void* z8;
    uint8_t* z_scale;
    void* z;
    void* gu;
    int64_t ldx, ldsx, ldw, ldsw, ldz8, ldsz, ldz, ldgu;
} hpsgd_gated_ffn_forward_args;
int hpsgd_gated_ffn_forward(const hpsgd_gated_ffn_forward_args* args, void* stream);

/*
 * What the layer's gradients are products of: with g, u as they are kept in gu,
 *     dg = dz u act'(g)      du = dz act(g)      d = dg | du  [M x 2 N]
 * in the block format along rows (dq) and along columns (dqt: the transpose [2 N x M]), and / or in bf16 (dgu); dx is then the product of dq and w's transpose,
 * the gradient of w that of dqt and x's transpose.
 *   dz         [M x N] of dz_dtype, the gradient of z (through its quantisation as if that were the identity)
 *   dgu        not gu's memory
 */
typedef struct hpsgd_gated_ffn_backward_args {
    int64_t M, N;
    int act, dz_dtype;
    const void* gu;
    const void* dz;
    void* dq;
    uint8_t* dq_scale;
    void* dqt;
    uint8_t* dqt_scale;
    void* dgu;
    int64_t ldgu, lddz, lddq, ldsdq, lddqt, ldsdqt, lddgu;
} hpsgd_gated_ffn_backward_args;
int hpsgd_gated_ffn_backward(const hpsgd_gated_ffn_backward_args* args, void* stream);

/*
 * Wait for `stream` and report what only the device can know: HPSGD_E_TIMEOUT if a wait inside hpsgd_gemm_fp8 or hpsgd_gated_ffn_forward ran out on this device
 * since the last call (on whatever stream: where there is one to report, the whole device is waited for, and both operators are named), HPSGD_E_CUDA if the
 * work failed.  A tile of D (up to 256 rows and columns) whose waits ran out, in whichever of its parts
 * along k, is left as it was, and nothing is added to it; other tiles may have been written.  Products whose parts go through the workspace
 * write nothing from such a time-out on until it has been reported here.
 */
int hpsgd_ops_check(void* stream);

/*
 * Checked build only; HPSGD_E_UNSUPPORTED otherwise.  1: the barriers of hpsgd_gemm_fp8 and hpsgd_gated_ffn_forward are told to expect 16
 * bytes more than their copies bring, so that their waits run out after two seconds: the way to see the time-out path (no results,
 * HPSGD_E_TIMEOUT from hpsgd_ops_check, the device usable as before) without a fault.  2: those of thread blocks with odd numbers only.
 */
int hpsgd_ops_debug_stall(int enable);

#ifdef __cplusplus
}
#endif

#endif /* HPSGD_OPS_H_ */

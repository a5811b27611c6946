/*
 * nvfp4mm.h -- C ABI of libnvfp4ss.so, second part: what a program does with 4-bit
 * matrices once it has them.  MXFP4 quantisation, the product of two quantised
 * matrices, the gated feed-forward block on quantised operands, and the gradients of
 * both, on NVIDIA GB300 (sm_103a).
 *
 * A quantised matrix [rows, cols] is held as
 *   codes  [rows, cols/2] packed E2M1 nibbles, as nvfp4ss.h describes them;
 *   sf     one scale code for each block along cols, in the 128x4-atom layout
 *          (NVFP4_SF_SWIZZLED of nvfp4ss.h, for either format with cols/block scale
 *          columns), whose padding bytes must be 0;
 *   S      NVFP4's fp32 global scale in device memory (NULL: 1, and for MXFP4 always NULL).
 * Formats:
 *   FP4_FMT_NVFP4  blocks of 16, E4M3 scales:  value q * s * S.
 *   FP4_FMT_MXFP4  blocks of 32, E8M0 scales:  value q * 2^(code - 127)
 *                  (OCP Microscaling Formats 1.0; code 255 is NaN).
 *
 * Conventions are those of nvfp4ss.h: row-major tensors, device-accessible pointers that
 * the caller owns, no allocation and no synchronisation, every call asynchronous on
 * `stream`, argument errors returned before any launch.  Products are exact, sums are
 * held in fp32, multiplied by the global scales in fp32 and rounded once to the output's type;
 * no result depends on timing: sums split over several thread blocks are added in a fixed
 * order.  That order follows from the sizes, so the same rows in calls of other sizes may differ in
 * fp32's last places.
 *   - cols (the contraction) of a product's operands is a multiple of 32 and at least 32,
 *     for either format: the tensor core's loads need rows of whole 16 bytes.
 *   - A product's operands have at most 8388480 rows (65535 * 128) and 2^30 columns, 8388480 where
 *     gradients are formed; larger ones return NVFP4_ERR_RANGE, and their workspace queries 0.
 *   - codes and sf of an operand are 16-byte aligned; dense tensors need their element's
 *     alignment, and run faster with 16-byte aligned bases and row strides.
 *   - Row strides (ld*) are in elements and at least the row's length.
 *   - A call with no rows or no columns of output launches nothing and returns NVFP4_OK.
 *     A gradient that sums over no rows or columns (no tokens: the weights') is zeros; such
 *     a call needs no workspace, and tensors without elements may be NULL.
 *   - status_dev: optional device int; bit 16 is OR-ed in when a bounded wait inside a
 *     kernel ran out (about a second; the outputs are then incomplete).
 *   - Outputs must not overlap inputs or each other.  Dense tensors may be columns of one buffer, their
 *     rows interleaved, where they have the same row stride.
 */
#ifndef NVFP4MM_H
#define NVFP4MM_H

#include "nvfp4ss.h"

#ifdef __cplusplus
extern "C" {
#endif

typedef enum { FP4_FMT_NVFP4 = 0, FP4_FMT_MXFP4 = 1 } fp4_format;
typedef enum { FP4_ACT_SILU = 0, FP4_ACT_GELU_TANH = 1 } fp4_activation;

/* One quantised matrix; rows and cols are arguments of the call. */
typedef struct {
    const uint8_t* codes;
    const uint8_t* sf;
    const float* S;
} fp4_operand;

/*
 * MXFP4 quantisation.  For each block of 32 elements, m = max |x|:
 *   X = 2^(floor(log2 m) - 2), at least 2^-127; scale code log2(X) + 127;
 *   q = RNE_E2M1(x / X), magnitudes past 6 to 6 (x / X < 8 by the choice of X).
 * Every step is exact but the rounding to E2M1.  A block of zeros, and one that holds a
 * NaN or an infinity, gets scale code 0 and nibbles that carry only the signs (the zero rule of
 * nvfp4ss.h); the latter also sets bit 0 of status_dev.
 *   x            [rows, cols] of type dt, row stride ldx; cols % 32 == 0, at most 2^30, and 128
 *                rows (or all, if fewer) hold at most 2^34 elements.  Bases and strides of whole
 *                32 bytes are read fastest.
 *   codes        [rows, cols/2], 8-byte aligned.
 *   sf_linear    optional [rows, cols/32] codes.
 *   sf_swizzled  optional, 128x4-atom layout: ceil(rows/128)*128 x ceil(cols/128)*4 bytes,
 *                4-byte aligned, padding written as 0.  At least one of the two.
 */
nvfp4_status mxfp4_quantize(const void* x, nvfp4_dtype dt, int64_t rows, int64_t cols, int64_t ldx, uint8_t* codes,
                            uint8_t* sf_linear, uint8_t* sf_swizzled, int* status_dev, void* stream);

/*
 * x_hat = fl32(q * 2^(code - 127)) of a matrix in MXFP4, written as fp32 or its RNE bf16.
 *   codes [rows, cols/2] (4-byte aligned), sf in `layout`, out [rows, cols] of out_dt,
 *   16-byte aligned; the limits on rows and cols are mxfp4_quantize's.
 */
nvfp4_status mxfp4_dequantize(const uint8_t* codes, const uint8_t* sf, nvfp4_sf_layout layout, int64_t rows,
                              int64_t cols, void* out, nvfp4_dtype out_dt, void* stream);

/*
 * D = A B^T of two quantised matrices in the same format: A [m, k] (activations, one row
 * a token), B [n, k] (an [out, in] weight).  D [m, n] of type out_dt, row stride ldd.
 * Both operands go to the tensor cores as they are.
 */
nvfp4_status fp4_matmul(fp4_format fmt, const fp4_operand* a, const fp4_operand* b, int64_t m, int64_t n, int64_t k,
                        void* D, nvfp4_dtype out_dt, int64_t ldd, int* status_dev, void* stream);

/*
 * Self-test of the products' bounded waits (failure detection): fp4_matmul whose waits for its
 * operands are made to give up after their limit, by barriers that expect one arrival too many.
 * status_dev (required) gets bit 16, D is not written and the CUDA context stays usable.
 */
nvfp4_status fp4_selftest_wait_timeout(fp4_format fmt, const fp4_operand* a, const fp4_operand* b, int64_t m, int64_t n,
                                       int64_t k, void* D, nvfp4_dtype out_dt, int64_t ldd, int* status_dev, void* stream);

/*
 * Gradients of fp4_matmul with respect to the values of its operands, from dD:
 *   dA = dD B [m, k],  dB = dD^T A [n, k],
 * all bf16 with row strides lddd, ldda, lddb; either of dA and dB may be NULL.  The
 * operands' values without S are exact in bf16 (those past fp32's range, of E8M0 codes 253 and
 * 254, are infinite), so the sums' only rounding is fp32's, then the results' to bf16.
 *   workspace  fp4_matmul_backward_workspace(m, n, k) bytes, 256-byte aligned.
 */
size_t fp4_matmul_backward_workspace(int64_t m, int64_t n, int64_t k);
nvfp4_status fp4_matmul_backward(fp4_format fmt, const fp4_operand* a, const fp4_operand* b, int64_t m, int64_t n,
                                 int64_t k, const void* dD, int64_t lddd, void* dA, int64_t ldda, void* dB,
                                 int64_t lddb, int* status_dev, void* workspace, size_t ws_bytes, void* stream);

/*
 * Gated feed-forward on quantised operands, in one kernel: with g = x Wg^T, u = x Wu^T,
 *   h = act(g) * u,   act(g) = g / (1 + exp(-g))                                 (SILU)
 *                     or g (1 + tanh(sqrt(2/pi) (g + 0.044715 g^3))) / 2    (GELU_TANH)
 * x [t, d], w_gate and w_up [f, d], all in fmt; g and u stay in fp32.
 *   h        optional [t, f] bf16, row stride ldh.
 *   h_codes, h_sf  optional (both or neither; f % 32 == 0): h in MXFP4, the codes and
 *            128x4-atom scales that mxfp4_quantize gives for the bf16 h, ready to be the
 *            next product's operand; status_dev bit 0 as there (a block of h that is not finite).
 *            h_codes 16-byte, h_sf 4-byte aligned.
 * At least one of the two forms.
 */
nvfp4_status fp4_gated_ff(fp4_format fmt, fp4_activation act, const fp4_operand* x, const fp4_operand* w_gate,
                          const fp4_operand* w_up, int64_t t, int64_t f, int64_t d, void* h, int64_t ldh,
                          uint8_t* h_codes, uint8_t* h_sf, int* status_dev, void* stream);

/*
 * Gradients of the gated feed-forward with respect to the values of its operands, from
 * dh [t, f] bf16 (row stride lddh).  g and u are computed again (nothing is kept from the
 * forward call), then
 *   dg = dh * u * act'(g),  du = dh * act(g)      (fp32, rounded once to bf16: by up to 2^-8,
 *                                                  the operands of the two lines that follow)
 *   dx = dg Wg + du Wu [t, d],  dWg = dg^T x,  dWu = du^T x [f, d]   (bf16, row strides)
 *   d_x      optional, row stride lddx.
 *   d_gate, d_up  optional (both or neither: frozen weights), row stride lddw.
 *   h        optional: the forward result too (row stride ldh).  fp4_gated_ff adds up fewer than 65
 *            tokens' sums in another order, so a few of its last bits may differ there.
 *   workspace  fp4_gated_ff_backward_workspace(t, f, d) bytes, 256-byte aligned.
 */
size_t fp4_gated_ff_backward_workspace(int64_t t, int64_t f, int64_t d);
nvfp4_status fp4_gated_ff_backward(fp4_format fmt, fp4_activation act, const fp4_operand* x,
                                   const fp4_operand* w_gate, const fp4_operand* w_up, int64_t t, int64_t f, int64_t d,
                                   const void* dh, int64_t lddh, void* d_x, int64_t lddx, void* d_gate, void* d_up,
                                   int64_t lddw, void* h, int64_t ldh, int* status_dev, void* workspace,
                                   size_t ws_bytes, void* stream);

#ifdef __cplusplus
}
#endif

#endif /* NVFP4MM_H */

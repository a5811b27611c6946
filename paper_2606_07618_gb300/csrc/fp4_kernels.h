// Internal interface between the host layer of nvfp4mm.h (fp4_api.cu) and its kernels.
// Not part of the public ABI.
#pragma once
#include <cstdint>
#include <cuda_runtime.h>

#include "fp4_plan.h"

namespace nvfp4 {

// ---- mxfp4.cu
cudaError_t launch_mxfp4_quantize(const void* x, int dtype, int64_t rows, int64_t cols, int64_t ldx, uint8_t* codes,
                                  uint8_t* sf_linear, uint8_t* sf_swizzled, int* status, int sms, cudaStream_t s);
cudaError_t launch_mxfp4_dequantize(const uint8_t* codes, const uint8_t* sf, int swizzled, int64_t rows, int64_t cols,
                                    void* out, int dtype, int sms, cudaStream_t s);
// out[r][c] = bf16(q * s) of quantised matrices of one width (without S), exact, 32-byte aligned; rows in
// [rows, rows_out) are written as zero.
struct Expansion {
    const uint8_t *codes, *sf;
    int64_t rows, rows_out;
    void* out;
};
cudaError_t launch_expand(int mx, const Expansion* m, int count, int64_t cols, cudaStream_t s);
// out[r][c] = in[r][c], bf16, for an input that TMA cannot read.
cudaError_t launch_repitch_bf16(const void* in, int64_t rows, int64_t cols, int64_t ldi, void* out, int64_t ldo,
                                cudaStream_t s);
cudaError_t launch_zero_bf16(int64_t rows, int64_t cols, void* out, int64_t ldo, cudaStream_t s);

// ---- fp4_gemm.cu
// An operand of a product.
struct Operand {
    const void* data;      // packed codes [rows, k/2]; bf16 [rows][ld], K along the row, or with `along` [k][ld]
    const uint8_t* sf;     // 128x4-atom scales; null for bf16
    const float* S;        // global scale or null
    int64_t rows, ld;      // ld: row stride in elements (bf16 only)
    int along;             // bf16: rows are contiguous, K steps by ld (always for p)
};

// One product: out[t][n] over t < q.rows, n < p.rows, from sums over k of q[t][k] p[n][k].
struct Product {
    int kind, mode, act;
    Operand p, p2, q;      // p2: the up projection's weight (gated modes); bf16: p2.S scales the second part of K
    int64_t k, k_part;     // bf16: where K's second part begins (a multiple of 64), or 0
    void* out;             // plain: D; gated modes: h (bf16) or null
    void* out2;            // plain: rows from row2 on go here (their own matrix, the size of the first), or null
    int64_t row2, rows1;   // the first one's rows; row2 is a multiple of 128
    int out_f32;
    int64_t ldo;
    uint8_t *h_codes, *h_sf;   // gated: h in MXFP4, or null
    const void* dh;        // gated grad: gradient of h, bf16
    int64_t lddh;
    void* dgu;             // gated grad: [t][2 fp] bf16: dg, du (columns past f zero)
    int64_t fp;
    int* status;
    int starve;            // 1: the waits for the operands run out (self-test)

    mm::Sizes sizes() const { return mm::Sizes{kind, mode, out_f32, q.rows, p.rows, k, q.ld}; }
};
cudaError_t launch_product(const Product& p, int sms, cudaStream_t s);
// ---- fp4_pair.cu: the same for many tokens
cudaError_t launch_pair(const Product& p, int sms, cudaStream_t s);

}  // namespace nvfp4

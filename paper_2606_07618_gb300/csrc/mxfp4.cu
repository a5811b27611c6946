// MXFP4 (E2M1 elements, one power-of-two E8M0 scale for each block of 32): quantisation
// and dequantisation, and the expansion to bf16 of the operands that gradients are formed with.
//
// All of them are bound by memory: a few instructions per element, each byte once.
#include <cuda_bf16.h>

#include "fp4_kernels.h"
#include "nvfp4_device.cuh"
#include "nvfp4_kernels.h"

namespace nvfp4 {
namespace {

__device__ __forceinline__ uint32_t div_by(uint32_t n, const FastDiv& d) {
    const uint32_t t = __umulhi(n, d.mul);
    return (t + ((n - t) >> d.s1)) >> d.s2;
}

// value of an E8M0 code (0: 2^-127, a subnormal; 255: NaN)
__device__ __forceinline__ float e8m0_value(uint32_t c) {
    return c == 0 ? __uint_as_float(0x00400000u) : c == 255 ? __uint_as_float(0x7FC00000u) : __uint_as_float(c << 23);
}
// two E2M1 codes of a byte as fp32
__device__ __forceinline__ void e2m1_pair(uint32_t byte, float& lo, float& hi) {
    uint32_t h2;
    asm("{\n\t.reg .b8 b;\n\t.reg .b16 t;\n\tcvt.u16.u32 t, %1;\n\tcvt.u8.u16 b, t;\n\tcvt.rn.f16x2.e2m1x2 %0, b;\n\t}"
        : "=r"(h2) : "r"(byte & 0xFFu));
    lo = f16bits_to_f32((uint16_t)(h2 & 0xFFFFu));
    hi = f16bits_to_f32((uint16_t)(h2 >> 16));
}
__device__ __forceinline__ uint32_t pack_bf16(float lo, float hi) {
    const __nv_bfloat162 v = __floats2bfloat162_rn(lo, hi);
    return *reinterpret_cast<const uint32_t*>(&v);
}

// ---------------------------------------------------------------------------
// Quantisation.  A lane holds 16 elements, two neighbours a block; the block's maximum is
// the larger of two lanes' integer maxima of |x| as bits, its exponent field gives X,
// and x / X is a multiplication by a power of two, so nothing rounds before the convert.
// A lane's loads are one or two 32-byte sectors; its codes are 8 bytes, a warp's 256.
struct MxParams {
    const void* x;
    int64_t rows, cols, ldx;
    uint8_t *codes, *sf_linear, *sf_swizzled;
    int* status;
    uint32_t segs, row_segs;     // of 16 elements
    uint32_t kb, kpad4;
    int early;                   // the next kernel may start beside this one
    FastDiv div;                 // by row_segs
};

enum { kWide = 0, kHalf = 1, kElement = 2 };   // loads of 32 bytes, 16 bytes, single elements

template <int BF16, int LOAD>
__device__ __forceinline__ void load_seg(const void* base, int64_t off, float (&y)[16]) {
    if (LOAD == kElement) {
#pragma unroll
        for (int i = 0; i < 16; i++)
            y[i] = BF16 ? __uint_as_float((uint32_t) reinterpret_cast<const uint16_t*>(base)[off + i] << 16)
                        : reinterpret_cast<const float*>(base)[off + i];
        return;
    }
    constexpr int kVec = BF16 ? 2 : 4;                       // 16-byte words
    uint4 v[kVec];
    const char* p = static_cast<const char*>(base) + off * (BF16 ? 2 : 4);
#pragma unroll
    for (int i = 0; i < kVec; i += 2) {
        if (LOAD == kWide) {
            ld_stream32<false>(p + 16 * i, v[i], v[i + 1]);
        } else {
            v[i] = ld_stream16<false>(p + 16 * i);
            v[i + 1] = ld_stream16<false>(p + 16 * i + 16);
        }
    }
#pragma unroll
    for (int i = 0; i < kVec; i++) {
        const uint32_t w[4] = {v[i].x, v[i].y, v[i].z, v[i].w};
#pragma unroll
        for (int j = 0; j < 4; j++) {
            if (BF16) {
                y[8 * i + 2 * j] = bf16lo(w[j]);
                y[8 * i + 2 * j + 1] = bf16hi(w[j]);
            } else {
                y[4 * i + j] = __uint_as_float(w[j]);
            }
        }
    }
}

template <int BF16, int LOAD>
__global__ void __launch_bounds__(256) mxfp4_quantize_kernel(MxParams p) {
    if (p.early) grid_launch_dependents();
    grid_dependency_wait();
    const uint32_t stride = gridDim.x * blockDim.x;
    const uint32_t padded = (p.segs + 31) & ~31u;            // whole warps: the shuffles name all lanes
    bool bad = false;
    for (uint32_t seg = blockIdx.x * blockDim.x + threadIdx.x; seg < padded; seg += stride) {
        const bool live = seg < p.segs;
        const uint32_t row = div_by(live ? seg : 0, p.div), c16 = (live ? seg : 0) - row * p.row_segs;
        float y[16];
        if (live) {
            load_seg<BF16, LOAD>(p.x, (int64_t)row * p.ldx + 16 * (int64_t)c16, y);
        } else {
#pragma unroll
            for (int i = 0; i < 16; i++) y[i] = 0.0f;
        }
        uint32_t m = 0;
#pragma unroll
        for (int i = 0; i < 16; i++) m = max(m, __float_as_uint(y[i]) & 0x7FFFFFFFu);
        m = max(m, __shfl_xor_sync(0xFFFFFFFFu, m, 1));
        const uint32_t e = m >> 23;
        const bool finite = e != 255;
        bad |= !finite;
        const uint32_t code = finite && e > 2 ? e - 2 : 0;
        const float inv = __uint_as_float((254u - code) << 23);  // 2^(127 - code)
        if (!finite)
#pragma unroll
            for (int i = 0; i < 16; i++) y[i] = copysignf(0.0f, y[i]);
        const u64 inv2 = pack2(inv, inv);
        u64 t[8];
#pragma unroll
        for (int i = 0; i < 8; i++) t[i] = mul2(pack2(y[2 * i], y[2 * i + 1]), inv2);
        if (!live) continue;
        reinterpret_cast<uint2*>(p.codes)[seg] = make_uint2(e2m1x8(t[0], t[1], t[2], t[3]), e2m1x8(t[4], t[5], t[6], t[7]));
        if ((seg & 1) == 0) {
            const uint32_t k = c16 >> 1;
            if (p.sf_linear) p.sf_linear[(int64_t)row * p.kb + k] = (uint8_t)code;
            if (p.sf_swizzled) {
                uint8_t* at = p.sf_swizzled + swizzle_offset(row, k, p.kpad4);
                *at = (uint8_t)code;
                if (k == p.kb - 1)                           // the row's last word: its padding
                    for (uint32_t j = 1; j < 4 - (k & 3); j++) at[j] = 0;
            }
        }
    }
    if (p.sf_swizzled) {                                     // rows up to a multiple of 128
        const uint32_t pad_rows = (uint32_t)(-p.rows & 127);
        for (uint32_t i = blockIdx.x * blockDim.x + threadIdx.x; i < pad_rows * p.kpad4; i += stride) {
            const int64_t r = p.rows + i / p.kpad4;
            *reinterpret_cast<uint32_t*>(p.sf_swizzled + swizzle_offset(r, 4 * (int64_t)(i % p.kpad4), p.kpad4)) = 0;
        }
    }
    if (bad && p.status) atomicOr(p.status, 1);
}

// ---------------------------------------------------------------------------
// Dequantisation: 8 codes (a word) to a lane, four words in flight.
template <int OUT_BF16, int SWIZZLED>
__global__ void __launch_bounds__(256)
    mxfp4_dequantize_kernel(const uint8_t* codes, const uint8_t* sf, uint32_t words, uint32_t kb, uint32_t kpad4,
                            FastDiv div, void* out) {
    constexpr int kUnroll = 4;
    grid_dependency_wait();
    const uint32_t stride = gridDim.x * blockDim.x * kUnroll;
    for (uint32_t w0 = (blockIdx.x * blockDim.x + (threadIdx.x & ~31u)) * kUnroll + (threadIdx.x & 31); w0 < words;
         w0 += stride) {
        uint32_t c[kUnroll], s[kUnroll];
#pragma unroll
        for (int u = 0; u < kUnroll; u++) {
            const uint32_t w = w0 + 32 * u;
            if (w < words) {
                const uint32_t blk = w >> 2;
                c[u] = ld_u32(reinterpret_cast<const uint32_t*>(codes) + w);
                if (SWIZZLED) {
                    const uint32_t row = div_by(blk, div);
                    s[u] = sf[swizzle_offset32(row, blk - row * kb, kpad4)];
                } else {
                    s[u] = sf[blk];
                }
            }
        }
#pragma unroll
        for (int u = 0; u < kUnroll; u++) {
            const uint32_t w = w0 + 32 * u;
            if (w >= words) break;
            const float v = e8m0_value(s[u]);
            float f[8];
#pragma unroll
            for (int j = 0; j < 4; j++) {
                e2m1_pair(c[u] >> (8 * j), f[2 * j], f[2 * j + 1]);
                f[2 * j] = __fmul_rn(f[2 * j], v);
                f[2 * j + 1] = __fmul_rn(f[2 * j + 1], v);
            }
            if (OUT_BF16) {
                reinterpret_cast<uint4*>(out)[w] = make_uint4(pack_bf16(f[0], f[1]), pack_bf16(f[2], f[3]),
                                                              pack_bf16(f[4], f[5]), pack_bf16(f[6], f[7]));
            } else {
                reinterpret_cast<float4*>(out)[2 * (int64_t)w] = make_float4(f[0], f[1], f[2], f[3]);
                reinterpret_cast<float4*>(out)[2 * (int64_t)w + 1] = make_float4(f[4], f[5], f[6], f[7]);
            }
        }
    }
}

// ---------------------------------------------------------------------------
// The values of quantised matrices without S in bf16: exact, as q has two significant bits and
// an E4M3 scale four.  16 codes to a lane, 32 bytes out; four in flight.  Up to three matrices of one width to a
// launch, their tiles of 1024 segments one after the other (a gradient call's all: training, 100 x 501 x 608, 17.1 us,
// 18.7 with a launch for each operand; 2048 x 4096 x 4096 101.4, 105.5).
struct ExpandPart {
    const uint8_t *codes, *sf;
    uint4* out;
    uint32_t segs, segs_out;     // of 16 elements: those there are, those to write
};
struct ExpandParams {
    ExpandPart part[3];
    uint32_t first[3];           // the tile that each starts with
    uint32_t row_segs, kpad4;
    FastDiv div;                 // by row_segs
};
template <int MX>
__global__ void __launch_bounds__(256) expand_kernel(const __grid_constant__ ExpandParams P) {
    constexpr int kUnroll = 4;
    grid_dependency_wait();
    grid_launch_dependents();                                // the product: 1.6 us of a small training step
    const int which = blockIdx.x >= P.first[2] ? 2 : blockIdx.x >= P.first[1] ? 1 : 0;
    const ExpandPart& m = P.part[which];
    const uint32_t s0 = ((blockIdx.x - P.first[which]) * blockDim.x + (threadIdx.x & ~31u)) * kUnroll + (threadIdx.x & 31);
    uint2 c[kUnroll];
    uint32_t s[kUnroll];
#pragma unroll
    for (int u = 0; u < kUnroll; u++) {
        const uint32_t seg = s0 + 32 * u;
        c[u] = make_uint2(0, 0);
        s[u] = MX ? 127 : 0;                                 // rows past the matrix: zero codes
        if (seg < m.segs) {
            const uint32_t row = div_by(seg, P.div), k = seg - row * P.row_segs;
            c[u] = reinterpret_cast<const uint2*>(m.codes)[seg];
            s[u] = m.sf[swizzle_offset(row, MX ? k >> 1 : k, P.kpad4)];
        }
    }
#pragma unroll
    for (int u = 0; u < kUnroll; u++) {
        const uint32_t seg = s0 + 32 * u;
        if (seg >= m.segs_out) break;
        const float v = MX ? e8m0_value(s[u]) : f16bits_to_f32(e4m3_to_f16bits(s[u]));
        uint32_t w[8];
#pragma unroll
        for (int j = 0; j < 8; j++) {
            float a, b;
            e2m1_pair((j < 4 ? c[u].x : c[u].y) >> (8 * (j & 3)), a, b);
            w[j] = pack_bf16(__fmul_rn(a, v), __fmul_rn(b, v));
        }
        uint4* at = m.out + 2 * (int64_t)seg;
        asm volatile("st.global.v8.b32 [%0], {%1, %2, %3, %4, %5, %6, %7, %8};"
                     ::"l"(at), "r"(w[0]), "r"(w[1]), "r"(w[2]), "r"(w[3]), "r"(w[4]), "r"(w[5]), "r"(w[6]), "r"(w[7]) : "memory");
    }
}

__global__ void __launch_bounds__(256)
    repitch_bf16_kernel(const uint16_t* in, int64_t rows, int64_t cols, int64_t ldi, uint16_t* out, int64_t ldo) {
    grid_dependency_wait();
    grid_launch_dependents();
    for (int64_t r = blockIdx.x; r < rows; r += gridDim.x)
        for (int64_t c = threadIdx.x; c < cols; c += blockDim.x) out[r * ldo + c] = in[r * ldi + c];
}

__global__ void __launch_bounds__(256) zero_bf16_kernel(int64_t rows, int64_t cols, uint16_t* out, int64_t ldo) {
    grid_dependency_wait();
    for (int64_t r = blockIdx.x; r < rows; r += gridDim.x)
        for (int64_t c = threadIdx.x; c < cols; c += blockDim.x) out[r * ldo + c] = 0;
}

template <typename... P, typename... Args>
cudaError_t launch_grid(void (*kernel)(P...), dim3 grid, int threads, cudaStream_t s, Args... args) {
    cudaLaunchConfig_t cfg = {};
    cfg.gridDim = grid;
    cfg.blockDim = dim3((unsigned)threads);
    cfg.stream = s;
    cudaLaunchAttribute attr[1];
    attr[0].id = cudaLaunchAttributeProgrammaticStreamSerialization;
    attr[0].val.programmaticStreamSerializationAllowed = 1;
    cfg.attrs = attr;
    cfg.numAttrs = 1;
    return cudaLaunchKernelEx(&cfg, kernel, static_cast<P>(args)...);
}

template <int BF16>
cudaError_t launch_quantize_as(const MxParams& p, int load, int64_t grid, cudaStream_t s) {
    return launch_dependent(load == kWide   ? mxfp4_quantize_kernel<BF16, kWide>
                            : load == kHalf ? mxfp4_quantize_kernel<BF16, kHalf>
                                            : mxfp4_quantize_kernel<BF16, kElement>,
                            grid, 256, s, p);
}

}  // namespace

cudaError_t launch_mxfp4_quantize(const void* x, int dtype, int64_t rows, int64_t cols, int64_t ldx, uint8_t* codes,
                                  uint8_t* sf_linear, uint8_t* sf_swizzled, int* status, int sms, cudaStream_t s) {
    const int64_t esize = dtype == 0 ? 2 : 4, kb = cols / 32, kpad4 = (kb + 3) / 4;
    const uintptr_t bits = reinterpret_cast<uintptr_t>(x) | (uintptr_t)(rows > 1 ? ldx * esize : 0);
    const int load = (bits & 31) == 0 ? kWide : (bits & 15) == 0 ? kHalf : kElement;
    // segments are counted in 32 bits: rows in groups of whole 128 (one group below 2^30 segments)
    const int64_t most = ((int64_t)1 << 30) / (cols / 16) / 128 * 128, group = most > 0 ? most : 128;
    for (int64_t r = 0; r < rows; r += group) {
        MxParams p;
        p.rows = rows - r < group ? rows - r : group;
        p.cols = cols;
        p.ldx = ldx;
        p.x = static_cast<const char*>(x) + r * ldx * esize;
        p.codes = codes + r * (cols / 2);
        p.sf_linear = sf_linear ? sf_linear + r * kb : nullptr;
        p.sf_swizzled = sf_swizzled ? sf_swizzled + r * kpad4 * 4 : nullptr;
        p.status = status;
        p.row_segs = (uint32_t)(cols / 16);
        p.segs = (uint32_t)(p.rows * p.row_segs);
        p.kb = (uint32_t)kb;
        p.kpad4 = (uint32_t)kpad4;
        p.div = make_fast_div(p.row_segs);
        int64_t grid = ((int64_t)p.segs + 255) / 256;        // 16 CTAs per SM: 14336 x 4096 bf16 and back 51.3 us, 55.4 with 8, 53.7 with no limit
        if (grid > (int64_t)sms * 16) grid = (int64_t)sms * 16;
        // One wave of CTAs: the product that follows sets itself up meanwhile (16 x 4096 and its product with 4096 x 4096
        // 6.1 us, 7.4 without).  In a longer grid the next kernel's waiting CTAs take the place of this one's (3001 x 2848
        // fp32 and back 20.5, 19.5 without).
        p.early = grid <= (int64_t)sms * 8;
        const cudaError_t e = dtype == 0 ? launch_quantize_as<1>(p, load, grid, s) : launch_quantize_as<0>(p, load, grid, s);
        if (e != cudaSuccess) return e;
    }
    return cudaSuccess;
}

cudaError_t launch_mxfp4_dequantize(const uint8_t* codes, const uint8_t* sf, int swizzled, int64_t rows, int64_t cols,
                                    void* out, int dtype, int sms, cudaStream_t s) {
    const int64_t kb = cols / 32, kpad4 = (kb + 3) / 4, esize = dtype == 0 ? 2 : 4;
    const int64_t most = ((int64_t)1 << 30) / (cols / 8) / 128 * 128, group = most > 0 ? most : 128;
    const FastDiv div = make_fast_div((uint32_t)kb);
    for (int64_t r = 0; r < rows; r += group) {
        const int64_t n = rows - r < group ? rows - r : group, words = n * (cols / 8);
        const int64_t grid = (words + 1023) / 1024;          // one tile to a warp (fp32 14336 x 4096 105 us, 109 with 16 CTAs per SM)
        const auto k = dtype == 0 ? (swizzled ? mxfp4_dequantize_kernel<1, 1> : mxfp4_dequantize_kernel<1, 0>)
                                  : (swizzled ? mxfp4_dequantize_kernel<0, 1> : mxfp4_dequantize_kernel<0, 0>);
        const cudaError_t e = launch_dependent(k, grid, 256, s, codes + r * (cols / 2), sf + r * (swizzled ? kpad4 * 4 : kb),
                                               (uint32_t)words, (uint32_t)kb, (uint32_t)kpad4, div,
                                               static_cast<void*>(static_cast<char*>(out) + r * cols * esize));
        if (e != cudaSuccess) return e;
    }
    return cudaSuccess;
}

cudaError_t launch_expand(int mx, const Expansion* m, int count, int64_t cols, cudaStream_t s) {
    ExpandParams P = {};
    P.row_segs = (uint32_t)(cols / 16);
    P.kpad4 = (uint32_t)((cols / (mx ? 32 : 16) + 3) / 4);
    P.div = make_fast_div(P.row_segs);
    // segments are counted in 32 bits: rows in groups of whole 128, as in quantisation
    const int64_t most = ((int64_t)1 << 30) / P.row_segs / 128 * 128, group = most > 0 ? most : 128;
    uint32_t tiles = 0;
    int parts = 0;
    for (int i = 0; i < count; i++)
        for (int64_t r = 0; r < m[i].rows_out; r += group) {
            const int64_t n_out = m[i].rows_out - r < group ? m[i].rows_out - r : group, left = m[i].rows - r;
            const int64_t n = left < 0 ? 0 : left < n_out ? left : n_out;
            P.part[parts] = ExpandPart{m[i].codes + r * (cols / 2), m[i].sf + r * P.kpad4 * 4,
                                       reinterpret_cast<uint4*>(static_cast<char*>(m[i].out) + r * cols * 2),
                                       (uint32_t)(n * P.row_segs), (uint32_t)(n_out * P.row_segs)};
            P.first[parts++] = tiles;
            tiles += (P.part[parts - 1].segs_out + 1023) / 1024;
            if (parts < 3 && !(i == count - 1 && r + group >= m[i].rows_out)) continue;
            for (int j = parts; j < 3; j++) P.first[j] = tiles;  // no tile
            const cudaError_t e = launch_grid(mx ? expand_kernel<1> : expand_kernel<0>, dim3(tiles), 256, s, P);
            if (e != cudaSuccess) return e;
            tiles = 0;
            parts = 0;
        }
    return cudaSuccess;
}

cudaError_t launch_repitch_bf16(const void* in, int64_t rows, int64_t cols, int64_t ldi, void* out, int64_t ldo,
                                cudaStream_t s) {
    return launch_grid(repitch_bf16_kernel, dim3((unsigned)(rows < 65535 ? rows : 65535)), 256, s,
                       static_cast<const uint16_t*>(in), rows, cols, ldi, static_cast<uint16_t*>(out), ldo);
}

cudaError_t launch_zero_bf16(int64_t rows, int64_t cols, void* out, int64_t ldo, cudaStream_t s) {
    return launch_grid(zero_bf16_kernel, dim3((unsigned)(rows < 65535 ? rows : 65535)), 256, s, rows, cols,
                       static_cast<uint16_t*>(out), ldo);
}

}  // namespace nvfp4

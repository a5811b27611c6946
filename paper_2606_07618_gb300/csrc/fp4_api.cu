// Host side of include/nvfp4mm.h: argument, alignment and overlap checks (all before any
// launch), then dispatch.  As in api.cu nothing allocates, frees or synchronises.
#include <climits>
#include <cstdint>

#include <cuda_runtime.h>

#include "fp4_kernels.h"
#include "host_checks.h"
#include "nvfp4mm.h"

using namespace nvfp4;

namespace {

// Grid limits: 128 rows or columns to a tile, 65535 tiles along a grid dimension.
constexpr int64_t kMaxRows = 65535ll * 128;
constexpr int64_t kMaxCols = 1ll << 30;                      // 32-bit tensor-map coordinates

// Conversions count a launch's parts in 32 bits, and a launch covers whole groups of 128 rows.
constexpr int64_t kMaxGroup = 1ll << 34;                     // elements

int64_t up(int64_t n, int64_t to) { return (n + to - 1) / to * to; }

// Rows of `width` bytes, `stride` bytes apart (one row: any run of bytes).
struct Span {
    const void* p;
    int64_t rows, width, stride;
    int64_t bytes() const { return (rows - 1) * stride + width; }
};

// Whether two spans have a byte in common.  Rows of one stride, the columns of one buffer, may
// interleave: one's columns then lie beside the other's modulo the stride.
bool overlap(const Span& a, const Span& b) {
    if (!nvfp4::overlap(a.p, a.bytes(), b.p, b.bytes())) return false;
    const int64_t stride = a.rows == 1 ? b.stride : a.stride;
    if ((a.rows == 1 && b.rows == 1) || (b.rows > 1 && b.stride != stride)) return true;
    int64_t at = (int64_t)(reinterpret_cast<uintptr_t>(b.p) - reinterpret_cast<uintptr_t>(a.p)) % stride;
    if (at < 0) at += stride;
    return at < a.width || at + b.width > stride;
}

// Memory that a call reads and writes.
struct Memory {
    Span r[16], w[16];
    int nr = 0, nw = 0;
    void read(const void* p, int64_t n) { read(p, 1, n, 0, 1); }
    void write(const void* p, int64_t n) { write(p, 1, n, 0, 1); }
    // [rows, cols] of elements of `esize` bytes with row stride ld
    void read(const void* p, int64_t rows, int64_t cols, int64_t ld, int64_t esize) {
        if (p && rows > 0 && cols > 0) r[nr++] = Span{p, rows, cols * esize, ld * esize};
    }
    void write(const void* p, int64_t rows, int64_t cols, int64_t ld, int64_t esize) {
        if (p && rows > 0 && cols > 0) w[nw++] = Span{p, rows, cols * esize, ld * esize};
    }
    nvfp4_status check() const {
        for (int i = 0; i < nw; i++) {
            for (int j = 0; j < nr; j++)
                if (overlap(w[i], r[j])) return NVFP4_ERR_INVALID_ARG;
            for (int j = i + 1; j < nw; j++)
                if (overlap(w[i], w[j])) return NVFP4_ERR_INVALID_ARG;
        }
        for (int i = 0; i < nw; i++)
            if (!device_accessible(w[i].p)) return NVFP4_ERR_INVALID_ARG;
        for (int i = 0; i < nr; i++)
            if (!device_accessible(r[i].p)) return NVFP4_ERR_INVALID_ARG;
        return NVFP4_OK;
    }
};

// Sizes of a dense tensor: rows and row stride that address arithmetic in bytes can hold.
nvfp4_status check_dense(const void* p, int64_t rows, int64_t cols, int64_t ld, int64_t esize) {
    if (!p) return NVFP4_ERR_INVALID_ARG;
    if (ld < cols) return NVFP4_ERR_INVALID_ARG;
    int64_t n;
    if (!mul_ok(rows, ld, &n) || n > INT64_MAX / 8) return NVFP4_ERR_RANGE;
    return aligned(p, (uintptr_t)esize) ? NVFP4_OK : NVFP4_ERR_ALIGNMENT;
}

nvfp4_status check_format(fp4_format fmt, int64_t k) {
    if (fmt != FP4_FMT_NVFP4 && fmt != FP4_FMT_MXFP4) return NVFP4_ERR_INVALID_ARG;
    if (k < 32 || k % 32 != 0) return NVFP4_ERR_UNSUPPORTED;
    return k <= kMaxCols ? NVFP4_OK : NVFP4_ERR_RANGE;
}

nvfp4_status check_rows(int64_t rows) { return rows < 0 ? NVFP4_ERR_INVALID_ARG : rows > kMaxRows ? NVFP4_ERR_RANGE : NVFP4_OK; }

int64_t sf_bytes(fp4_format fmt, int64_t rows, int64_t k) {
    return up(rows, 128) * up(k / (fmt == FP4_FMT_MXFP4 ? 32 : 16), 4);
}

nvfp4_status check_operand(fp4_format fmt, const fp4_operand* o, int64_t rows, int64_t k, Memory* mem) {
    if (!o || !o->codes || !o->sf) return NVFP4_ERR_INVALID_ARG;
    if (fmt == FP4_FMT_MXFP4 && o->S) return NVFP4_ERR_INVALID_ARG;
    if (!aligned(o->codes, 16) || !aligned(o->sf, 16) || !aligned(o->S, 4)) return NVFP4_ERR_ALIGNMENT;
    mem->read(o->codes, rows * (k / 2));
    mem->read(o->sf, sf_bytes(fmt, rows, k));
    mem->read(o->S, 4);
    return NVFP4_OK;
}

Operand operand(const fp4_operand* o, int64_t rows) { return Operand{o->codes, o->sf, o->S, rows, 0, 0}; }

nvfp4_status result(cudaError_t e) {
    return e == cudaSuccess ? NVFP4_OK : e == cudaErrorNotSupported ? NVFP4_ERR_UNSUPPORTED : NVFP4_ERR_CUDA;
}

// A bf16 product for a gradient: out[t][n] = S sum_k q[t][k] p[k][n].
Product grad_product(const void* p, int64_t n, int64_t ldp, const float* S, const void* q, int64_t qrows, int64_t ldq,
                     int along, int64_t k, void* out, int64_t ldo, int* status) {
    Product g = {};
    g.kind = kBf16;
    g.mode = kPlain;
    g.p = Operand{p, nullptr, S, n, ldp, 1};
    g.q = Operand{q, nullptr, nullptr, qrows, ldq, along};
    g.k = k;
    g.out = out;
    g.ldo = ldo;
    g.status = status;
    return g;
}

// Gradients that sum over no rows or no columns: zeros.  A tensor without elements may be null.
struct ZeroGrad {
    void* p;
    int64_t rows, cols, ld;
};
template <int N>
nvfp4_status zero_grads(const ZeroGrad (&g)[N], cudaStream_t s) {
    Memory mem;
    for (const ZeroGrad& z : g) {
        if (!z.p || z.rows == 0) continue;
        const nvfp4_status st = check_dense(z.p, z.rows, z.cols, z.ld, 2);
        if (st != NVFP4_OK) return st;
        mem.write(z.p, z.rows, z.cols, z.ld, 2);
    }
    const nvfp4_status st = mem.check();
    if (st != NVFP4_OK) return st;
    for (const ZeroGrad& z : g)
        if (z.p && z.rows > 0) {
            const cudaError_t e = launch_zero_bf16(z.rows, z.cols, z.p, z.ld, s);
            if (e != cudaSuccess) return result(e);
        }
    return NVFP4_OK;
}

// Parts of a workspace, each to a multiple of 256 bytes.
struct Parts {
    char* base;
    int64_t used = 0;
    explicit Parts(void* ws) : base(static_cast<char*>(ws)) {}
    void* take(int64_t bytes) {
        void* p = base + used;
        used += up(bytes, 256);
        return p;
    }
};

// bf16 buffers of fp4_matmul_backward: the values of B and A, and dD where TMA cannot read its rows.
struct MatmulGrad {
    int64_t ldn, b, a, d;
    MatmulGrad(int64_t m, int64_t n, int64_t k) : ldn(up(n, 8)), b(n * k * 2), a(m * k * 2), d(m * ldn * 2) {}
    size_t bytes() const { return (size_t)(up(b, 256) + up(a, 256) + up(d, 256)); }
};

// and of fp4_gated_ff_backward: the values of both weights, one after the other (gate's rows up to a
// multiple of 128), and of x; dg and du side by side.
struct GatedGrad {
    int64_t fp, w, x, dgu;
    GatedGrad(int64_t t, int64_t f, int64_t d) : fp(up(f, 128)), w(2 * fp * d * 2), x(t * d * 2), dgu(t * 2 * fp * 2) {}
    size_t bytes() const { return (size_t)(up(w, 256) + up(x, 256) + up(dgu, 256)); }
};

}  // namespace

extern "C" {

nvfp4_status mxfp4_quantize(const void* x, nvfp4_dtype dt, int64_t rows, int64_t cols, int64_t ldx, uint8_t* codes,
                            uint8_t* sf_linear, uint8_t* sf_swizzled, int* status_dev, void* stream) {
    if ((dt != NVFP4_IN_BF16 && dt != NVFP4_IN_F32) || rows < 0 || cols < 0 || cols % 32 != 0) return NVFP4_ERR_INVALID_ARG;
    if (cols > kMaxCols || (rows < 128 ? rows : 128) * cols > kMaxGroup) return NVFP4_ERR_RANGE;
    if (rows == 0 || cols == 0) return NVFP4_OK;
    const int64_t esize = dt == NVFP4_IN_BF16 ? 2 : 4;
    if (!codes || (!sf_linear && !sf_swizzled)) return NVFP4_ERR_INVALID_ARG;
    const nvfp4_status st = check_dense(x, rows, cols, ldx, esize);
    if (st != NVFP4_OK) return st;
    if (!aligned(codes, 8) || !aligned(sf_swizzled, 4) || !aligned(status_dev, 4)) return NVFP4_ERR_ALIGNMENT;
    Memory mem;
    mem.read(x, rows, cols, ldx, esize);
    mem.write(codes, rows * (cols / 2));
    mem.write(sf_linear, rows * (cols / 32));
    mem.write(sf_swizzled, sf_bytes(FP4_FMT_MXFP4, rows, cols));
    mem.write(status_dev, 4);
    const nvfp4_status ms = mem.check();
    if (ms != NVFP4_OK) return ms;
    const int sms = sm_count();
    if (sms <= 0) return NVFP4_ERR_CUDA;
    return result(launch_mxfp4_quantize(x, dt == NVFP4_IN_BF16 ? 0 : 1, rows, cols, ldx, codes, sf_linear, sf_swizzled,
                                        status_dev, sms, static_cast<cudaStream_t>(stream)));
}

nvfp4_status mxfp4_dequantize(const uint8_t* codes, const uint8_t* sf, nvfp4_sf_layout layout, int64_t rows,
                              int64_t cols, void* out, nvfp4_dtype out_dt, void* stream) {
    if ((out_dt != NVFP4_IN_BF16 && out_dt != NVFP4_IN_F32) || (layout != NVFP4_SF_LINEAR && layout != NVFP4_SF_SWIZZLED) ||
        rows < 0 || cols < 0 || cols % 32 != 0)
        return NVFP4_ERR_INVALID_ARG;
    if (cols > kMaxCols || (rows < 128 ? rows : 128) * cols > kMaxGroup) return NVFP4_ERR_RANGE;
    if (rows == 0 || cols == 0) return NVFP4_OK;
    if (!codes || !sf) return NVFP4_ERR_INVALID_ARG;
    const int64_t esize = out_dt == NVFP4_IN_BF16 ? 2 : 4;
    const nvfp4_status st = check_dense(out, rows, cols, cols, esize);
    if (st != NVFP4_OK) return st;
    if (!aligned(codes, 4) || !aligned(out, 16)) return NVFP4_ERR_ALIGNMENT;
    const int swizzled = layout == NVFP4_SF_SWIZZLED;
    Memory mem;
    mem.read(codes, rows * (cols / 2));
    mem.read(sf, swizzled ? sf_bytes(FP4_FMT_MXFP4, rows, cols) : rows * (cols / 32));
    mem.write(out, rows * cols * esize);
    const nvfp4_status ms = mem.check();
    if (ms != NVFP4_OK) return ms;
    const int sms = sm_count();
    if (sms <= 0) return NVFP4_ERR_CUDA;
    return result(launch_mxfp4_dequantize(codes, sf, swizzled, rows, cols, out, out_dt == NVFP4_IN_BF16 ? 0 : 1, sms,
                                          static_cast<cudaStream_t>(stream)));
}

}  // extern "C"

namespace {
nvfp4_status matmul_common(fp4_format fmt, const fp4_operand* a, const fp4_operand* b, int64_t m, int64_t n, int64_t k,
                           void* D, nvfp4_dtype out_dt, int64_t ldd, int* status_dev, int starve, void* stream) {
    nvfp4_status st;
    if (out_dt != NVFP4_IN_BF16 && out_dt != NVFP4_IN_F32) return NVFP4_ERR_INVALID_ARG;
    if ((st = check_format(fmt, k)) != NVFP4_OK || (st = check_rows(m)) != NVFP4_OK || (st = check_rows(n)) != NVFP4_OK)
        return st;
    if (m == 0 || n == 0) return NVFP4_OK;
    const int64_t esize = out_dt == NVFP4_IN_BF16 ? 2 : 4;
    Memory mem;
    if ((st = check_operand(fmt, a, m, k, &mem)) != NVFP4_OK || (st = check_operand(fmt, b, n, k, &mem)) != NVFP4_OK ||
        (st = check_dense(D, m, n, ldd, esize)) != NVFP4_OK)
        return st;
    if (!aligned(status_dev, 4)) return NVFP4_ERR_ALIGNMENT;
    mem.write(D, m, n, ldd, esize);
    mem.write(status_dev, 4);
    if ((st = mem.check()) != NVFP4_OK) return st;
    const int sms = sm_count();
    if (sms <= 0) return NVFP4_ERR_CUDA;
    Product p = {};
    p.kind = fmt == FP4_FMT_MXFP4 ? kMxfp4 : kNvfp4;
    p.mode = kPlain;
    p.p = operand(b, n);
    p.q = operand(a, m);
    p.k = k;
    p.out = D;
    p.out_f32 = out_dt == NVFP4_IN_F32;
    p.ldo = ldd;
    p.status = status_dev;
    p.starve = starve;
    return result(launch_product(p, sms, static_cast<cudaStream_t>(stream)));
}
}  // namespace

extern "C" {

nvfp4_status fp4_matmul(fp4_format fmt, const fp4_operand* a, const fp4_operand* b, int64_t m, int64_t n, int64_t k,
                        void* D, nvfp4_dtype out_dt, int64_t ldd, int* status_dev, void* stream) {
    return matmul_common(fmt, a, b, m, n, k, D, out_dt, ldd, status_dev, 0, stream);
}

nvfp4_status fp4_selftest_wait_timeout(fp4_format fmt, const fp4_operand* a, const fp4_operand* b, int64_t m, int64_t n,
                                       int64_t k, void* D, nvfp4_dtype out_dt, int64_t ldd, int* status_dev, void* stream) {
    if (!status_dev) return NVFP4_ERR_INVALID_ARG;
    return matmul_common(fmt, a, b, m, n, k, D, out_dt, ldd, status_dev, 1, stream);
}

size_t fp4_matmul_backward_workspace(int64_t m, int64_t n, int64_t k) {
    if (m <= 0 || n <= 0 || k <= 0 || m > kMaxRows || n > kMaxRows || k > kMaxRows) return 0;
    return MatmulGrad(m, n, k).bytes();
}

nvfp4_status fp4_matmul_backward(fp4_format fmt, const fp4_operand* a, const fp4_operand* b, int64_t m, int64_t n,
                                 int64_t k, const void* dD, int64_t lddd, void* dA, int64_t ldda, void* dB,
                                 int64_t lddb, int* status_dev, void* workspace, size_t ws_bytes, void* stream) {
    nvfp4_status st;
    if ((st = check_format(fmt, k)) != NVFP4_OK || (st = check_rows(m)) != NVFP4_OK || (st = check_rows(n)) != NVFP4_OK)
        return st;
    if (k > kMaxRows) return NVFP4_ERR_RANGE;
    if (m == 0 || n == 0) {
        const ZeroGrad z[] = {{dA, m, k, ldda}, {dB, n, k, lddb}};
        return zero_grads(z, static_cast<cudaStream_t>(stream));
    }
    if (!dA && !dB) return NVFP4_ERR_INVALID_ARG;
    const MatmulGrad g(m, n, k);
    Memory mem;
    if ((st = check_operand(fmt, a, m, k, &mem)) != NVFP4_OK || (st = check_operand(fmt, b, n, k, &mem)) != NVFP4_OK ||
        (st = check_dense(dD, m, n, lddd, 2)) != NVFP4_OK || (dA && (st = check_dense(dA, m, k, ldda, 2)) != NVFP4_OK) ||
        (dB && (st = check_dense(dB, n, k, lddb, 2)) != NVFP4_OK))
        return st;
    if (!workspace || ws_bytes < g.bytes()) return NVFP4_ERR_INVALID_ARG;
    if (!aligned(workspace, 256) || !aligned(status_dev, 4)) return NVFP4_ERR_ALIGNMENT;
    mem.read(dD, m, n, lddd, 2);
    mem.write(dA, m, k, ldda, 2);
    mem.write(dB, n, k, lddb, 2);
    mem.write(workspace, (int64_t)g.bytes());
    mem.write(status_dev, 4);
    if ((st = mem.check()) != NVFP4_OK) return st;
    const int sms = sm_count();
    if (sms <= 0) return NVFP4_ERR_CUDA;
    const cudaStream_t s = static_cast<cudaStream_t>(stream);
    const int mx = fmt == FP4_FMT_MXFP4;
    Parts ws(workspace);
    void *bv = ws.take(g.b), *av = ws.take(g.a), *dv = ws.take(g.d);
    const void* d = dD;
    int64_t ldd = lddd;
    cudaError_t e = cudaSuccess;
    if (!aligned(dD, 16) || lddd % 8 != 0) {                 // rows that TMA cannot read
        e = launch_repitch_bf16(dD, m, n, lddd, dv, g.ldn, s);
        d = dv;
        ldd = g.ldn;
    }
    Expansion x[2];
    int nx = 0;
    if (dA) x[nx++] = Expansion{b->codes, b->sf, n, n, bv};
    if (dB) x[nx++] = Expansion{a->codes, a->sf, m, m, av};
    if (e == cudaSuccess) e = launch_expand(mx, x, nx, k, s);
    if (dA && e == cudaSuccess) e = launch_product(grad_product(bv, k, k, b->S, d, m, ldd, 0, n, dA, ldda, status_dev), sms, s);
    if (dB && e == cudaSuccess) e = launch_product(grad_product(av, k, k, a->S, d, n, ldd, 1, m, dB, lddb, status_dev), sms, s);
    return result(e);
}

nvfp4_status fp4_gated_ff(fp4_format fmt, fp4_activation act, const fp4_operand* x, const fp4_operand* w_gate,
                          const fp4_operand* w_up, int64_t t, int64_t f, int64_t d, void* h, int64_t ldh,
                          uint8_t* h_codes, uint8_t* h_sf, int* status_dev, void* stream) {
    nvfp4_status st;
    if (act != FP4_ACT_SILU && act != FP4_ACT_GELU_TANH) return NVFP4_ERR_INVALID_ARG;
    if ((st = check_format(fmt, d)) != NVFP4_OK || (st = check_rows(t)) != NVFP4_OK || (st = check_rows(f)) != NVFP4_OK)
        return st;
    if (!h_codes != !h_sf || (h_codes && f % 32 != 0)) return NVFP4_ERR_INVALID_ARG;
    if (t == 0 || f == 0) return NVFP4_OK;
    if (!h && !h_codes) return NVFP4_ERR_INVALID_ARG;
    Memory mem;
    if ((st = check_operand(fmt, x, t, d, &mem)) != NVFP4_OK || (st = check_operand(fmt, w_gate, f, d, &mem)) != NVFP4_OK ||
        (st = check_operand(fmt, w_up, f, d, &mem)) != NVFP4_OK || (h && (st = check_dense(h, t, f, ldh, 2)) != NVFP4_OK))
        return st;
    if (!aligned(h_codes, 16) || !aligned(h_sf, 4) || !aligned(status_dev, 4)) return NVFP4_ERR_ALIGNMENT;
    mem.write(h, t, f, ldh, 2);
    mem.write(h_codes, t * (f / 2));
    if (h_sf) mem.write(h_sf, sf_bytes(FP4_FMT_MXFP4, t, f));
    mem.write(status_dev, 4);
    if ((st = mem.check()) != NVFP4_OK) return st;
    const int sms = sm_count();
    if (sms <= 0) return NVFP4_ERR_CUDA;
    Product p = {};
    p.kind = fmt == FP4_FMT_MXFP4 ? kMxfp4 : kNvfp4;
    p.mode = kGated;
    p.act = act;
    p.p = operand(w_gate, f);
    p.p2 = operand(w_up, f);
    p.q = operand(x, t);
    p.k = d;
    p.out = h;
    p.ldo = ldh;
    p.h_codes = h_codes;
    p.h_sf = h_sf;
    p.status = status_dev;
    return result(launch_product(p, sms, static_cast<cudaStream_t>(stream)));
}

size_t fp4_gated_ff_backward_workspace(int64_t t, int64_t f, int64_t d) {
    if (t <= 0 || f <= 0 || d <= 0 || t > kMaxRows || f > kMaxRows || d > kMaxRows) return 0;
    return GatedGrad(t, f, d).bytes();
}

nvfp4_status fp4_gated_ff_backward(fp4_format fmt, fp4_activation act, const fp4_operand* x,
                                   const fp4_operand* w_gate, const fp4_operand* w_up, int64_t t, int64_t f, int64_t d,
                                   const void* dh, int64_t lddh, void* d_x, int64_t lddx, void* d_gate, void* d_up,
                                   int64_t lddw, void* h, int64_t ldh, int* status_dev, void* workspace,
                                   size_t ws_bytes, void* stream) {
    nvfp4_status st;
    if (act != FP4_ACT_SILU && act != FP4_ACT_GELU_TANH) return NVFP4_ERR_INVALID_ARG;
    if ((st = check_format(fmt, d)) != NVFP4_OK || (st = check_rows(t)) != NVFP4_OK || (st = check_rows(f)) != NVFP4_OK)
        return st;
    if (d > kMaxRows) return NVFP4_ERR_RANGE;
    if (!d_gate != !d_up) return NVFP4_ERR_INVALID_ARG;
    if (t == 0 || f == 0) {
        const ZeroGrad z[] = {{d_x, t, d, lddx}, {d_gate, f, d, lddw}, {d_up, f, d, lddw}};
        return zero_grads(z, static_cast<cudaStream_t>(stream));
    }
    if (!d_x && !d_gate) return NVFP4_ERR_INVALID_ARG;
    const GatedGrad g(t, f, d);
    Memory mem;
    if ((st = check_operand(fmt, x, t, d, &mem)) != NVFP4_OK || (st = check_operand(fmt, w_gate, f, d, &mem)) != NVFP4_OK ||
        (st = check_operand(fmt, w_up, f, d, &mem)) != NVFP4_OK || (st = check_dense(dh, t, f, lddh, 2)) != NVFP4_OK ||
        (d_x && (st = check_dense(d_x, t, d, lddx, 2)) != NVFP4_OK) ||
        (d_gate && (st = check_dense(d_gate, f, d, lddw, 2)) != NVFP4_OK) ||
        (d_up && (st = check_dense(d_up, f, d, lddw, 2)) != NVFP4_OK) ||
        (h && (st = check_dense(h, t, f, ldh, 2)) != NVFP4_OK))
        return st;
    if (!workspace || ws_bytes < g.bytes()) return NVFP4_ERR_INVALID_ARG;
    if (!aligned(workspace, 256) || !aligned(status_dev, 4)) return NVFP4_ERR_ALIGNMENT;
    mem.read(dh, t, f, lddh, 2);
    mem.write(d_x, t, d, lddx, 2);
    mem.write(d_gate, f, d, lddw, 2);
    mem.write(d_up, f, d, lddw, 2);
    mem.write(h, t, f, ldh, 2);
    mem.write(workspace, (int64_t)g.bytes());
    mem.write(status_dev, 4);
    if ((st = mem.check()) != NVFP4_OK) return st;
    const int sms = sm_count();
    if (sms <= 0) return NVFP4_ERR_CUDA;
    const cudaStream_t s = static_cast<cudaStream_t>(stream);
    const int mx = fmt == FP4_FMT_MXFP4;
    Parts ws(workspace);
    void *wv = ws.take(g.w), *xv = ws.take(g.x), *dgu = ws.take(g.dgu);

    Product p = {};
    p.kind = mx ? kMxfp4 : kNvfp4;
    p.mode = kGatedGrad;
    p.act = act;
    p.p = operand(w_gate, f);
    p.p2 = operand(w_up, f);
    p.q = operand(x, t);
    p.k = d;
    p.out = h;
    p.ldo = ldh;
    p.dh = dh;
    p.lddh = lddh;
    p.dgu = dgu;
    p.fp = g.fp;
    p.status = status_dev;
    cudaError_t e = launch_product(p, sms, s);
    Expansion v[3];
    int nv = 0;
    if (d_x) {
        v[nv++] = Expansion{w_gate->codes, w_gate->sf, f, g.fp, wv};
        v[nv++] = Expansion{w_up->codes, w_up->sf, f, g.fp, static_cast<char*>(wv) + g.fp * d * 2};
    }
    if (d_gate) v[nv++] = Expansion{x->codes, x->sf, t, t, xv};
    if (e == cudaSuccess) e = launch_expand(mx, v, nv, d, s);
    if (d_x && e == cudaSuccess) {
        // gate's half of the contraction and up's have a global scale each
        Product q = grad_product(wv, d, d, w_gate->S, dgu, t, 2 * g.fp, 0, 2 * g.fp, d_x, lddx, status_dev);
        q.p2.S = w_up->S;
        if (!mx) q.k_part = g.fp;
        e = launch_product(q, sms, s);
    }
    if (d_gate && e == cudaSuccess) {
        // one product for both: dg's columns of dgu are its rows 0.. , du's its rows fp..
        Product q = grad_product(xv, d, d, x->S, dgu, g.fp + f, 2 * g.fp, 1, t, d_gate, lddw, status_dev);
        q.out2 = d_up;
        q.row2 = g.fp;
        q.rows1 = f;
        e = launch_product(q, sms, s);
    }
    return result(e);
}

}  // extern "C"

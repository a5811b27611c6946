// Tokens into the NVFP4 key/value cache and back (nvfp4_kv_write, nvfp4_kv_read).
//
// Both are bound by memory, the sweep by its arithmetic (eleven candidates a block, the
// arithmetic and code of quantize_kernel.cuh).  A warp covers 8 tokens by 4 blocks of 16: a
// token's 4 blocks are 32 bytes of codes, a whole sector, and a block's scales of 8 tokens lie side by
// side, so that neither side's scattered accesses take many more sectors than they hold.
#include "kv_kernels.h"
#include "quantize_kernel.cuh"

namespace nvfp4 {
namespace kv {
namespace {

// Place of a token's block in the pool: page, offset in it.
struct Place {
    int64_t page;
    int at;
};
__device__ __forceinline__ int64_t row_of(const Cache& c, int64_t page, int head, int part) {
    return (page * c.heads + head) * 2 + part;
}
__device__ __forceinline__ uint8_t* codes_at(const Cache& c, const Place& w, int head, int part, int block) {
    return c.codes + ((row_of(c, w.page, head, part) << c.page_log2) + w.at) * (c.dim / 2) + block * 8;
}
__device__ __forceinline__ uint8_t* sf_at(const Cache& c, const Place& w, int head, int part, int block) {
    return c.sf + ((row_of(c, w.page, head, part) * (c.dim / 16) + block) << c.page_log2) + w.at;
}

template <int DT>
__device__ __forceinline__ void load_block(const Tensor& t, int64_t e, Raw& r) {
    if (t.vec) {
        const char* p = static_cast<const char*>(t.p) + e * (DT == 0 ? 2 : 4);
        r.a = ld_stream16<false>(p);
        r.b = ld_stream16<false>(p + 16);
        if (DT != 0) {
            r.c = ld_stream16<false>(p + 32);
            r.d = ld_stream16<false>(p + 48);
        }
        return;
    }
    uint32_t w[16];
    if (DT == 0) {
        const uint16_t* p = static_cast<const uint16_t*>(t.p) + e;
#pragma unroll
        for (int i = 0; i < 8; i++) w[i] = p[2 * i] | (uint32_t)p[2 * i + 1] << 16;
    } else {
        const uint32_t* p = static_cast<const uint32_t*>(t.p) + e;
#pragma unroll
        for (int i = 0; i < 16; i++) w[i] = p[i];
        r.c = make_uint4(w[8], w[9], w[10], w[11]);
        r.d = make_uint4(w[12], w[13], w[14], w[15]);
    }
    r.a = make_uint4(w[0], w[1], w[2], w[3]);
    r.b = make_uint4(w[4], w[5], w[6], w[7]);
}

// One warp's work: tokens 8 i .. 8 i + 7, blocks 4 j .. of a head of k or v.
struct Item {
    int64_t token;
    int head, part, block;
};
__device__ __forceinline__ Item item_of(int64_t w, int heads, int quads, int parts, int lane) {
    const uint32_t per = (uint32_t)(heads * quads * parts);
    const int64_t group = w / per;
    uint32_t r = (uint32_t)(w - group * per);
    Item it;
    it.block = (int)(r % quads) * 4 + (lane & 3);
    r /= quads;
    it.head = (int)(r % heads);
    it.part = (int)(r / heads);
    it.token = group * 8 + (lane >> 2);
    return it;
}

template <int DT, int METHOD>
__global__ void __launch_bounds__(256, METHOD == 0 ? 2 : 4) write_kernel(Write p, int64_t items) {
    __shared__ Cand tab[kTabN];
    grid_launch_dependents();
    build_table(tab);
    __syncthreads();
    grid_dependency_wait();
    const int lane = threadIdx.x & 31;
    const int quads = p.c.dim / 64, only = p.in[0].p ? 0 : 1, parts = p.in[0].p && p.in[1].p ? 2 : 1;
    float E[2];
    bool usable[2];
#pragma unroll
    for (int i = 0; i < 2; i++) {
        const float S = p.in[i].p ? ld_f32(i ? p.c.S_v : p.c.S_k) : 1.0f;
        E[i] = __frcp_rn(S);
        usable[i] = S > 0.0f && isfinite(S) && isfinite(E[i]);
        if (!usable[i]) E[i] = 1.0f;
    }
    const int64_t slots = p.c.pages << p.c.page_log2;
    bool bad = false, outside = false;
    for (int64_t w = (int64_t)blockIdx.x * 8 + (threadIdx.x >> 5); w < items; w += (int64_t)gridDim.x * 8) {
        const Item it = item_of(w, p.c.heads, quads, parts, lane);
        const int part = it.part + only;
        bool valid = it.token < p.tokens;
        int64_t slot = valid ? p.slots[it.token] : -1;
        if (slot >= slots) outside = true;
        valid = slot >= 0 && slot < slots;
        u64 y2[8];
        float m = 0.0f, ma = 0.0f, mb = 0.0f;
        if (valid) {
            Raw raw;
            const Tensor& t = p.in[part];
            load_block<DT>(t, it.token * t.token + it.head * t.head + it.block * 16, raw);
            const u64 E2 = part ? pack2(E[1], E[1]) : pack2(E[0], E[0]);
            m = METHOD == 0 ? raw_to_y_halves<DT>(raw, E2, y2, ma, mb) : raw_to_y<DT>(raw, E2, y2);
            bad |= !(m < __int_as_float(0x7f800000));
        } else {
#pragma unroll
            for (int j = 0; j < 8; j++) y2[j] = 0ull;
        }
        const bool zero = zero_block(usable[part], m);
        int code;
        if (METHOD == 0) {
            const int I0 = e4m3_floor_code_of_sixth(m);
            u64 none[8];
            float best;
            code = I0 - 3 + default_window_argmin<0, 16, false>(y2, none, ma, mb, tab + (I0 - 3 + kTabOff), best, true, false);
        } else {
            code = max((int)e4m3_rn_code(sixth(m)), 1);
        }
        uint32_t packed[2];
        if (zero) {
            code = 0;
#pragma unroll
            for (int h = 0; h < 2; h++) {
                packed[h] = 0;
#pragma unroll
                for (int j = 0; j < 4; j++) {
                    float a, b;
                    unpack2(y2[4 * h + j], a, b);
                    packed[h] |= ((signbit(a) ? 0x08u : 0u) | (signbit(b) ? 0x80u : 0u)) << (8 * j);
                }
            }
        } else {
            const float r = tab[code + kTabOff].r;
            const u64 r2 = pack2(r, r);
#pragma unroll
            for (int h = 0; h < 2; h++)
                packed[h] = e2m1x8(mul2(y2[4 * h], r2), mul2(y2[4 * h + 1], r2), mul2(y2[4 * h + 2], r2),
                                   mul2(y2[4 * h + 3], r2));
        }
        if (valid) {
            const Place at{slot >> p.c.page_log2, (int)(slot & ((1 << p.c.page_log2) - 1))};
            *reinterpret_cast<uint2*>(codes_at(p.c, at, it.head, part, it.block)) = make_uint2(packed[0], packed[1]);
            *sf_at(p.c, at, it.head, part, it.block) = (uint8_t)code;
        }
    }
    if (p.status) {
        if (__any_sync(0xffffffffu, bad) && lane == 0) atomicOr(p.status, kStatusNonFinite);
        if (__any_sync(0xffffffffu, outside) && lane == 0) atomicOr(p.status, kStatusBounds);
    }
}

// Sequence of row r: the last b with offsets[b] <= r; batch where r is behind the last one.
__device__ __forceinline__ int64_t sequence_of(const int32_t* offsets, int64_t batch, int64_t r) {
    int64_t lo = 0, hi = batch + 1;
    while (hi > lo) {
        const int64_t mid = (lo + hi) >> 1;
        if (offsets[mid] > r) hi = mid;
        else lo = mid + 1;
    }
    return lo - 1;
}

template <int DT>
__global__ void __launch_bounds__(256) read_kernel(Read p, int64_t items) {
    grid_launch_dependents();
    grid_dependency_wait();
    const int lane = threadIdx.x & 31;
    const int quads = p.c.dim / 64, only = p.out[0].p ? 0 : 1, parts = p.out[0].p && p.out[1].p ? 2 : 1;
    bool outside = false;
    for (int64_t w = (int64_t)blockIdx.x * 8 + (threadIdx.x >> 5); w < items; w += (int64_t)gridDim.x * 8) {
        const Item it = item_of(w, p.c.heads, quads, parts, lane);
        const int part = it.part + only;
        if (it.token >= p.tokens) continue;
        const int64_t b = sequence_of(p.offsets, p.batch, it.token);
        if (b < 0 || b >= p.batch) continue;
        const int64_t j = (p.starts ? p.starts[b] : 0) + (it.token - p.offsets[b]);
        int64_t page = -1;
        if (j >= 0 && (j >> p.c.page_log2) < p.width) page = p.table[b * p.table_ld + (j >> p.c.page_log2)];
        const bool ok = page >= 0 && page < p.c.pages;
        outside |= !ok;
        uint2 q = make_uint2(0, 0);
        uint32_t sf = 0;
        if (ok) {
            const Place at{page, (int)(j & ((1 << p.c.page_log2) - 1))};
            q = *reinterpret_cast<const uint2*>(codes_at(p.c, at, it.head, part, it.block));
            sf = *sf_at(p.c, at, it.head, part, it.block);
        }
        const float s = f16bits_to_f32(e4m3_to_f16bits(sf)), S = ld_f32(part ? p.c.S_v : p.c.S_k);
        float v[16];
#pragma unroll
        for (int i = 0; i < 8; i++) {
            uint32_t h;
            const uint16_t byte = (uint16_t)(((i < 4 ? q.x : q.y) >> (8 * (i & 3))) & 0xFF);
            asm("{\n\t.reg .b8 lo, hi;\n\tmov.b16 {lo, hi}, %1;\n\tcvt.rn.f16x2.e2m1x2 %0, lo;\n\t}" : "=r"(h) : "h"(byte));
            // q s is exact, q s S is rounded once
            v[2 * i] = __fmul_rn(__fmul_rn(f16bits_to_f32((uint16_t)h), s), S);
            v[2 * i + 1] = __fmul_rn(__fmul_rn(f16bits_to_f32((uint16_t)(h >> 16)), s), S);
        }
        if (!ok) {
#pragma unroll
            for (int i = 0; i < 16; i++) v[i] = 0.0f;
        }
        const Tensor& t = p.out[part];
        const int64_t e = it.token * t.token + it.head * t.head + it.block * 16;
        uint32_t o[16];
#pragma unroll
        for (int i = 0; i < 16; i++) o[i] = __float_as_uint(v[i]);
        if (DT == 0) {
#pragma unroll
            for (int i = 0; i < 8; i++)
                asm("cvt.rn.bf16x2.f32 %0, %1, %2;" : "=r"(o[i]) : "f"(v[2 * i + 1]), "f"(v[2 * i]));
        }
        constexpr int N = DT == 0 ? 8 : 16;                      // words
        if (t.vec) {
            uint4* d = reinterpret_cast<uint4*>(static_cast<char*>(t.p) + e * (DT == 0 ? 2 : 4));
#pragma unroll
            for (int i = 0; i < N / 4; i++) d[i] = make_uint4(o[4 * i], o[4 * i + 1], o[4 * i + 2], o[4 * i + 3]);
        } else if (DT == 0) {
            uint16_t* d = static_cast<uint16_t*>(t.p) + e;
#pragma unroll
            for (int i = 0; i < 16; i++) d[i] = (uint16_t)(o[i / 2] >> (16 * (i & 1)));
        } else {
            uint32_t* d = static_cast<uint32_t*>(t.p) + e;
#pragma unroll
            for (int i = 0; i < 16; i++) d[i] = o[i];
        }
    }
    if (p.status && __any_sync(0xffffffffu, outside) && lane == 0) atomicOr(p.status, kStatusBounds);
}

int64_t warps(int64_t tokens, const Cache& c, const Tensor (&t)[2]) {
    return (tokens + 7) / 8 * c.heads * (c.dim / 64) * ((t[0].p != nullptr) + (t[1].p != nullptr));
}

template <int DT, int METHOD>
cudaError_t launch_write_one(const Write& p, int64_t items, int sms, cudaStream_t s) {
    static std::atomic<int> occ[kOccDevices];
    const int64_t cap = (int64_t)sms * occupancy_per_sm(occ, write_kernel<DT, METHOD>, 256), need = (items + 7) / 8;
    return launch_dependent(write_kernel<DT, METHOD>, need < cap ? need : cap, 256, s, p, items);
}

}  // namespace

cudaError_t launch_write(const Write& p, int sms, cudaStream_t s) {
    const int64_t items = warps(p.tokens, p.c, p.in);
    if (p.dtype == 0) return p.method == 0 ? launch_write_one<0, 0>(p, items, sms, s) : launch_write_one<0, 1>(p, items, sms, s);
    return p.method == 0 ? launch_write_one<1, 0>(p, items, sms, s) : launch_write_one<1, 1>(p, items, sms, s);
}

cudaError_t launch_read(const Read& p, int sms, cudaStream_t s) {
    const int64_t items = warps(p.tokens, p.c, p.out), need = (items + 7) / 8, cap = (int64_t)sms * 8;
    const int64_t grid = need < cap ? need : cap;
    return p.dtype == 0 ? launch_dependent(read_kernel<0>, grid, 256, s, p, items)
                        : launch_dependent(read_kernel<1>, grid, 256, s, p, items);
}

}  // namespace kv
}  // namespace nvfp4

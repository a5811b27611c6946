// Tokens into the NVFP4 key/value cache and back (nvfp4_kv_write, nvfp4_kv_read).
//
// Both are bound by memory, the sweep by its arithmetic (eleven candidates a block, the
// arithmetic and code of quantize_kernel.cuh).  A warp covers 8 tokens by 4 blocks of 16: a
// token's 4 blocks are 32 bytes of codes, a whole sector, and a block's scales of 8 tokens lie side by
// side, so that neither side's scattered accesses take many more sectors than they hold.  A warp keeps to its
// blocks of one head and walks the tokens, so that its addresses are a page's and a token's multiples.
//
// 65536 tokens of 8 heads of 128, bf16 (268 MB of keys and values, 75 MB of cache): written with block maxima in 64 us (51 at
// the copy rate), swept in 203 (the sweep of as many elements by scalesweep_quantize: 194), read back in 75.
#include "kv_kernels.h"
#include "quantize_kernel.cuh"

namespace nvfp4 {
namespace kv {
namespace {

// A column's block in the pool: byte offsets of page 0's token 0, and of a page.
struct Place {
    uint8_t *codes, *sf;
    int64_t page_codes, page_sf;
    int row;                             // bytes of a token's codes
    __device__ __forceinline__ Place(const Cache& c, int head, int part, int block) {
        const int64_t at = (int64_t)(head * 2 + part) << c.page_log2;
        row = c.dim / 2;
        codes = c.codes + at * row + block * 8;
        sf = c.sf + at * (c.dim / 16) + ((int64_t)block << c.page_log2);
        page_sf = (int64_t)(c.heads * 2) * (c.dim / 16) << c.page_log2;
        page_codes = 8 * page_sf;
    }
    __device__ __forceinline__ uint2* codes_of(int64_t page, int at) const {
        return reinterpret_cast<uint2*>(codes + page * page_codes + at * row);
    }
    __device__ __forceinline__ uint8_t* sf_of(int64_t page, int at) const { return sf + page * page_sf + at; }
};

template <int DT>
__device__ __forceinline__ void load_block(const Tensor& t, int64_t e, Raw& r) {
    const char* p = static_cast<const char*>(t.p) + e * (DT == 0 ? 2 : 4);
    if (t.vec == 2) {
        ld_stream32<false>(p, r.a, r.b);
        if (DT != 0) ld_stream32<false>(p + 32, r.c, r.d);
        return;
    }
    if (t.vec == 1) {
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

// A warp's column: four blocks of a head of k or v, of which it takes groups of 8 tokens, `step` groups apart.
struct Column {
    int head, part, block;
    int64_t group, step;
};
struct Grid {
    int columns;                         // of all heads and parts
    int64_t groups, step;
};
__device__ __forceinline__ Column column_of(const Grid& grid, int heads, int quads, int lane) {
    const int64_t w = (int64_t)blockIdx.x * 8 + (threadIdx.x >> 5);
    Column c;
    c.group = w / grid.columns;
    int r = (int)(w - c.group * grid.columns);
    c.block = r % quads * 4 + (lane & 3);
    r /= quads;
    c.head = r % heads;
    c.part = r / heads;
    c.step = grid.step;
    if (c.group >= grid.step) c.group = grid.groups;            // warps that fill up the last block
    return c;
}

template <int DT, int METHOD>
__global__ void __launch_bounds__(256, METHOD == 0 ? 2 : DT == 0 ? 4 : 3) write_kernel(Write p, Grid grid) {
    __shared__ Cand tab[kTabN];
    grid_launch_dependents();
    build_table(tab);
    __syncthreads();
    grid_dependency_wait();
    const int lane = threadIdx.x & 31;
    const Column col = column_of(grid, p.c.heads, p.c.dim / 64, lane);
    const int part = p.in[0].p ? col.part : 1;
    const Tensor in = part ? p.in[1] : p.in[0];
    const Place place(p.c, col.head, part, col.block);
    const float S = ld_f32(part ? p.c.S_v : p.c.S_k);
    float E = __frcp_rn(S);
    const bool usable = S > 0.0f && isfinite(S) && isfinite(E);
    if (!usable) E = 1.0f;
    const u64 E2 = pack2(E, E);
    const int64_t slots = p.c.pages << p.c.page_log2, from = (int64_t)col.head * in.head + col.block * 16;
    bool bad = false, outside = false;
    // the next group's place and elements are on their way while this one is quantised
    Raw next;
    int64_t next_slot = -1;
    auto fetch = [&](int64_t group) {
        const int64_t token = group * 8 + (lane >> 2);
        next_slot = -1;
        if (group < grid.groups && token < p.tokens) {
            next_slot = p.slots[token];
            load_block<DT>(in, token * in.token + from, next);
        }
    };
    fetch(col.group);
    for (int64_t group = col.group; group < grid.groups; group += col.step) {
        const int64_t slot = next_slot;
        Raw raw = next;
        fetch(group + col.step);
        outside |= slot >= slots;
        const bool valid = slot >= 0 && slot < slots;
        u64 y2[8];
        float m = 0.0f, ma = 0.0f, mb = 0.0f;
        if (valid) {
            m = METHOD == 0 ? raw_to_y_halves<DT>(raw, E2, y2, ma, mb) : raw_to_y<DT>(raw, E2, y2);
            bad |= !(m < __int_as_float(0x7f800000));
        } else {
#pragma unroll
            for (int j = 0; j < 8; j++) y2[j] = 0ull;
        }
        const bool zero = zero_block(usable, m);
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
            const int64_t page = slot >> p.c.page_log2;
            const int at = (int)(slot & ((1 << p.c.page_log2) - 1));
            *place.codes_of(page, at) = make_uint2(packed[0], packed[1]);
            *place.sf_of(page, at) = (uint8_t)code;
        }
    }
    if (p.status) {
        if (__any_sync(0xffffffffu, bad) && lane == 0) atomicOr(p.status, kStatusNonFinite);
        if (__any_sync(0xffffffffu, outside) && lane == 0) atomicOr(p.status, kStatusBounds);
    }
}

// Sequence of row r: the last b with offsets[b] <= r; batch where r is behind the last one.
__device__ __forceinline__ int sequence_of(const int32_t* offsets, int batch, int r) {
    unsigned lo = 0, hi = (unsigned)batch + 1;
    while (hi > lo) {
        const unsigned mid = (lo + hi) >> 1;
        if (offsets[mid] > r) hi = mid;
        else lo = mid + 1;
    }
    return (int)lo - 1;
}

// kGroups of a warp's groups at a time, their loads side by side.
constexpr int kGroups = 4;

template <int DT>
__global__ void __launch_bounds__(256) read_kernel(Read p, Grid grid) {
    grid_launch_dependents();
    grid_dependency_wait();
    const int lane = threadIdx.x & 31;
    const Column col = column_of(grid, p.c.heads, p.c.dim / 64, lane);
    const int part = p.out[0].p ? col.part : 1;
    const Tensor t = part ? p.out[1] : p.out[0];
    const Place place(p.c, col.head, part, col.block);
    const float S = ld_f32(part ? p.c.S_v : p.c.S_k);
    const int64_t from = (int64_t)col.head * t.head + col.block * 16;
    const int page_log2 = p.c.page_log2, page_mask = (1 << page_log2) - 1;
    bool outside = false;
    int b = -1, first = 0, past = 0, start = 0;                  // the last sequence found, its rows and first token
    for (int64_t group = col.group; group < grid.groups; group += kGroups * col.step) {
        int token[kGroups], page[kGroups], at[kGroups];          // tokens, pages and what they count fit 31 bits
#pragma unroll
        for (int k = 0; k < kGroups; k++) {
            const int64_t row = (group + k * col.step) * 8 + (lane >> 2);
            token[k] = group + k * col.step < grid.groups && row < p.tokens ? (int)row : -1;
            page[k] = -1, at[k] = 0;
            if (token[k] < 0) continue;
            if (token[k] < first || token[k] >= past) {
                b = sequence_of(p.offsets, (int)p.batch, token[k]);
                const bool in = b >= 0 && b < p.batch;
                first = in ? p.offsets[b] : 0, past = in ? p.offsets[b + 1] : 0;
                if (!in) {
                    token[k] = -1;                               // behind the last sequence
                    continue;
                }
                start = p.starts ? p.starts[b] : 0;
            }
            const int64_t j = (int64_t)start + (token[k] - first);
            if (j >= 0 && (j >> page_log2) < p.width) page[k] = p.table[b * p.table_ld + (j >> page_log2)];
            at[k] = (int)j & page_mask;
        }
        uint2 codes[kGroups];
        uint32_t scale[kGroups];
        bool there[kGroups];
#pragma unroll
        for (int k = 0; k < kGroups; k++) {
            there[k] = page[k] >= 0 && page[k] < p.c.pages;
            outside |= token[k] >= 0 && !there[k];
            codes[k] = make_uint2(0, 0), scale[k] = 0;
            if (there[k]) {
                codes[k] = *place.codes_of(page[k], at[k]);
                scale[k] = *place.sf_of(page[k], at[k]);
            }
        }
#pragma unroll
        for (int k = 0; k < kGroups; k++) {
        if (token[k] < 0) continue;
        const uint16_t s = e4m3_to_f16bits(scale[k]);
        float v[16];
#pragma unroll
        for (int i = 0; i < 8; i++) {
            // q s is exact, q s S is rounded once
            const uint16_t byte = (uint16_t)(((i < 4 ? codes[k].x : codes[k].y) >> (8 * (i & 3))) & 0xFF);
            asm("{\n\t.reg .b8 lo, hi;\n\t.reg .b32 h;\n\t.reg .b16 a, b;\n\tmov.b16 {lo, hi}, %2;\n\tcvt.rn.f16x2.e2m1x2 h, lo;\n\t"
                "mov.b32 {a, b}, h;\n\tfma.rn.f32.f16 %0, a, %3, %4;\n\tfma.rn.f32.f16 %1, b, %3, %4;\n\t}"
                : "=f"(v[2 * i]), "=f"(v[2 * i + 1]) : "h"(byte), "h"(s), "f"(-0.0f));
            unpack2(mul2(pack2(v[2 * i], v[2 * i + 1]), pack2(S, S)), v[2 * i], v[2 * i + 1]);
        }
        if (!there[k]) {
#pragma unroll
            for (int i = 0; i < 16; i++) v[i] = 0.0f;
        }
        const int64_t e = token[k] * t.token + from;
        uint32_t o[16];
#pragma unroll
        for (int i = 0; i < 16; i++) o[i] = __float_as_uint(v[i]);
        if (DT == 0) {
#pragma unroll
            for (int i = 0; i < 8; i++)
                asm("cvt.rn.bf16x2.f32 %0, %1, %2;" : "=r"(o[i]) : "f"(v[2 * i + 1]), "f"(v[2 * i]));
        }
        constexpr int N = DT == 0 ? 8 : 16;                      // words
        if (t.vec == 2) {                                        // a sector at a time
            char* d = static_cast<char*>(t.p) + e * (DT == 0 ? 2 : 4);
#pragma unroll
            for (int i = 0; i < N; i += 8)
                asm volatile("st.global.v8.b32 [%0], {%1, %2, %3, %4, %5, %6, %7, %8};" ::"l"(d + 4 * i), "r"(o[i]), "r"(o[i + 1]),
                             "r"(o[i + 2]), "r"(o[i + 3]), "r"(o[i + 4]), "r"(o[i + 5]), "r"(o[i + 6]), "r"(o[i + 7]) : "memory");
        } else if (t.vec == 1) {
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
    }
    if (p.status && __any_sync(0xffffffffu, outside) && lane == 0) atomicOr(p.status, kStatusBounds);
}

// Columns of all heads and parts, and as many warps to each as fill the GPU (at most one a group of tokens).
Grid make_grid(int64_t tokens, const Cache& c, const Tensor (&t)[2], int64_t warps, int64_t* blocks) {
    Grid g;
    g.columns = c.heads * (c.dim / 64) * ((t[0].p != nullptr) + (t[1].p != nullptr));
    g.groups = (tokens + 7) / 8;
    g.step = warps / g.columns;
    g.step = g.step < 1 ? 1 : g.step < g.groups ? g.step : g.groups;
    *blocks = (g.step * g.columns + 7) / 8;
    return g;
}

template <int DT, int METHOD>
cudaError_t launch_write_one(const Write& p, int sms, cudaStream_t s) {
    static std::atomic<int> occ[kOccDevices];
    int64_t blocks;
    const Grid g = make_grid(p.tokens, p.c, p.in, (int64_t)sms * 8 * occupancy_per_sm(occ, write_kernel<DT, METHOD>, 256), &blocks);
    return launch_dependent(write_kernel<DT, METHOD>, blocks, 256, s, p, g);
}

}  // namespace

cudaError_t launch_write(const Write& p, int sms, cudaStream_t s) {
    if (p.dtype == 0) return p.method == 0 ? launch_write_one<0, 0>(p, sms, s) : launch_write_one<0, 1>(p, sms, s);
    return p.method == 0 ? launch_write_one<1, 0>(p, sms, s) : launch_write_one<1, 1>(p, sms, s);
}

cudaError_t launch_read(const Read& p, int sms, cudaStream_t s) {
    int64_t blocks;
    const Grid g = make_grid(p.tokens, p.c, p.out, (int64_t)sms * 8 * 6, &blocks);
    return p.dtype == 0 ? launch_dependent(read_kernel<0>, blocks, 256, s, p, g) : launch_dependent(read_kernel<1>, blocks, 256, s, p, g);
}

}  // namespace kv
}  // namespace nvfp4

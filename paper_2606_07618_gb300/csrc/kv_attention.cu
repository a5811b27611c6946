// Attention over the NVFP4 key/value cache for few rows a key head (nvfp4_kv_attention,
// nvfp4_kv_attention_prefix).
//
// A value q s (without S) has at most 6 significant bits (2 of E2M1, 4 of E4M3) and lies in 2^-10 .. 2688, so fp16
// holds it exactly; a query's row is scaled by a power of two to below 2 and is exact in fp16 too
// but for elements below 2^-14 of the row's largest.  Both products run on mma.sync
// m16n8k16 (fp16 operands, fp32 sums): with 8 or 16 rows they are 6% of the instructions, and an operand of
// registers is what the converted codes already are (tcgen05 would want them in shared memory first).
//
// What bounds it is instruction issue: a warp's tile of 64 tokens (dim 128, 8 rows) takes about 1070 instructions, of
// them 256 conversions, 256 multiplications by the blocks' scales and 64 MMAs, for 9.2 KB of cache.  16 sequences of
// 4096 tokens with 8 key heads (75.8 MB, 11.2 us at the copy rate) take 20.9 us: 11 us of issue at the 2.8 instructions a
// cycle that the loop reaches, and what a block spends before and after its four tiles a warp.
//
// Transposed products, so that the rows of queries are the MMA's narrow dimension:
//   S^T [tokens 16, rows 8] = K Q^T,   O^T [dim 16, rows 8] += V^T P^T.
// The order of the contracted index is free, as long as both operands share it.  A warp
// takes 64 tokens; lane (g, t) = (lane / 4, lane % 4) reads
//   keys:   of tokens 16 (g/2) + (g&1) + 2i, i = 0..7, the dim/4 elements from t dim/4 on,
//           and their scales of 16 tokens with one load a block;
//   values: of tokens 16 t .. 16 t + 15, the dim/8 elements from g dim/8 on,
// each by asynchronous copies of its own to shared memory, keys and values in turn one tile ahead: 40 registers fewer than
// loads kept in flight, so four blocks an SM instead of three (24.3 -> 22.4 us then).
// Rows r and r + 8 of m-tile i of S^T are then tokens 16 (r/2) + 4i + (r&1) and two further, whose
// weights, transposed by movmatrix, are the operand for the values of tokens 16 t + 4i .. + 3.
// Two tokens' codes of one dim are brought side by side as nibbles, so that one conversion gives the
// pair of fp16 that the MMA wants.
//
// Softmax runs over the tiles of a warp with a running maximum, which is followed only when it has grown by more than
// 2^8: weights are held 2^7-fold, so that they stay below fp16's largest, and O is rarely scaled.  Rows whose logits may
// pass 2^22 round them first (kWideFactor; it costs the others 1%: 20.7 -> 20.9 us, dim 64 and 16 rows 52.2 -> 53.3).  Warps, and the parts
// that a long cache is split into, are joined by their maxima, in a fixed order.
#include <climits>

#include "kv_kernels.h"
#include "nvfp4_device.cuh"

namespace nvfp4 {
namespace kv {
namespace {

constexpr int kThreads = 128;
constexpr float kWeightBits = 7.0f, kGrowth = 8.0f;

__device__ __forceinline__ float neg_inf() { return __int_as_float(0xff800000); }
// The larger one; NaN if either is, so that a query with NaN gives NaN.
__device__ __forceinline__ float max_nan(float a, float b) {
    float d;
    asm("max.NaN.f32 %0, %1, %2;" : "=f"(d) : "f"(a), "f"(b));
    return d;
}
__device__ __forceinline__ float max3_nan(float a, float b, float c) {
    float d;
    asm("max.NaN.f32 %0, %1, %2, %3;" : "=f"(d) : "f"(a), "f"(b), "f"(c));
    return d;
}
__device__ __forceinline__ float ex2(float x) {
    float y;
    asm("ex2.approx.ftz.f32 %0, %1;" : "=f"(y) : "f"(x));
    return y;
}
__device__ __forceinline__ uint32_t mul_h2(uint32_t a, uint32_t b) {
    uint32_t d;
    asm("mul.rn.f16x2 %0, %1, %2;" : "=r"(d) : "r"(a), "r"(b));
    return d;
}
// Four bytes of E2M1 pairs -> four fp16 pairs.
__device__ __forceinline__ void e2m1x8_to_f16(uint32_t w, uint32_t (&h)[4]) {
    asm("{\n\t.reg .b8 a, b, c, d;\n\tmov.b32 {a, b, c, d}, %4;\n\t"
        "cvt.rn.f16x2.e2m1x2 %0, a;\n\tcvt.rn.f16x2.e2m1x2 %1, b;\n\t"
        "cvt.rn.f16x2.e2m1x2 %2, c;\n\tcvt.rn.f16x2.e2m1x2 %3, d;\n\t}"
        : "=r"(h[0]), "=r"(h[1]), "=r"(h[2]), "=r"(h[3]) : "r"(w));
}
// Two E4M3 codes (16 bits) -> an fp16 pair.
__device__ __forceinline__ uint32_t e4m3x2_to_f16(uint32_t codes) {
    uint32_t h;
    asm("cvt.rn.f16x2.e4m3x2 %0, %1;" : "=r"(h) : "h"((uint16_t)codes));
    return h;
}
__device__ __forceinline__ void mma16(float (&d)[4], const uint32_t (&a)[4], uint32_t b0, uint32_t b1) {
    asm("mma.sync.aligned.m16n8k16.row.col.f32.f16.f16.f32 {%0, %1, %2, %3}, {%4, %5, %6, %7}, {%8, %9}, {%0, %1, %2, %3};"
        : "+f"(d[0]), "+f"(d[1]), "+f"(d[2]), "+f"(d[3])
        : "r"(a[0]), "r"(a[1]), "r"(a[2]), "r"(a[3]), "r"(b0), "r"(b1));
}
// The same onto nothing.
__device__ __forceinline__ void mma16_first(float (&d)[4], const uint32_t (&a)[4], uint32_t b0, uint32_t b1) {
    asm("mma.sync.aligned.m16n8k16.row.col.f32.f16.f16.f32 {%0, %1, %2, %3}, {%4, %5, %6, %7}, {%8, %9}, {%10, %10, %10, %10};"
        : "=f"(d[0]), "=f"(d[1]), "=f"(d[2]), "=f"(d[3])
        : "r"(a[0]), "r"(a[1]), "r"(a[2]), "r"(a[3]), "r"(b0), "r"(b1), "f"(0.0f));
}
__device__ __forceinline__ uint32_t transpose8x8(uint32_t a) {
    uint32_t d;
    asm("movmatrix.sync.aligned.m8n8.trans.b16 %0, %1;" : "=r"(d) : "r"(a));
    return d;
}
__device__ __forceinline__ uint32_t f16x2(float lo, float hi) {
    uint32_t r;
    asm("cvt.rn.f16x2.f32 %0, %1, %2;" : "=r"(r) : "f"(hi), "f"(lo));
    return r;
}

template <int D, int NT>
struct Tile {
    static constexpr int R = 8 * NT;
    static constexpr int KW = D / 32;    // words of codes of a token that a lane reads: keys
    static constexpr int VW = D / 64;    // and values
    static constexpr int KB = D / 64;    // key blocks of a lane
    // A warp's tile in shared memory, [word group][lane]: keys' codes and scales, values' codes and scales.
    static constexpr int kKeys = 8 * 32 * KW * 4, kKeySf = kKeys + KB * 512, kValues = kKeySf + 16 * 32 * VW * 4, kWarp = kValues + 512;
    static constexpr int kSums = 4 * R * D * 4;                  // the warps' sums, over the tiles
    static constexpr int kSmem = 4 * kWarp > kSums ? 4 * kWarp : kSums;
};

template <int BYTES>
__device__ __forceinline__ void copy_async(uint32_t dst, const uint8_t* src) {
    if (BYTES == 16) asm volatile("cp.async.cg.shared.global [%0], [%1], 16;" ::"r"(dst), "l"(src) : "memory");
    else asm volatile("cp.async.ca.shared.global [%0], [%1], %2;" ::"r"(dst), "l"(src), "n"(BYTES) : "memory");
}
__device__ __forceinline__ void copy_commit() { asm volatile("cp.async.commit_group;" ::: "memory"); }
template <int N>
__device__ __forceinline__ void copy_wait() { asm volatile("cp.async.wait_group %0;" ::"n"(N) : "memory"); }
template <int W>
__device__ __forceinline__ void ld_shared(uint32_t a, uint32_t (&w)[W]) {
    if constexpr (W == 4)
        asm volatile("ld.shared.v4.u32 {%0, %1, %2, %3}, [%4];" : "=r"(w[0]), "=r"(w[1]), "=r"(w[2]), "=r"(w[3]) : "r"(a) : "memory");
    else if constexpr (W == 2)
        asm volatile("ld.shared.v2.u32 {%0, %1}, [%2];" : "=r"(w[0]), "=r"(w[1]) : "r"(a) : "memory");
    else
        asm volatile("ld.shared.u32 %0, [%1];" : "=r"(w[0]) : "r"(a) : "memory");
}

// Where a block's result goes: to out; to out together with the other blocks of its cluster, the parts of the
// same rows; to the workspace, for join_kernel.
enum Join { kAlone, kCluster, kWorkspace };

__device__ __forceinline__ uint32_t cluster_addr(const void* p, uint32_t rank) {
    uint32_t a;
    asm("mapa.shared::cluster.u32 %0, %1, %2;" : "=r"(a) : "r"((uint32_t)__cvta_generic_to_shared(p)), "r"(rank));
    return a;
}
__device__ __forceinline__ float ld_cluster(uint32_t a) {
    float v;
    asm volatile("ld.shared::cluster.f32 %0, [%1];" : "=f"(v) : "r"(a) : "memory");
    return v;
}
__device__ __forceinline__ float4 ld_cluster4(uint32_t a) {
    float4 v;
    asm volatile("ld.shared::cluster.v4.f32 {%0, %1, %2, %3}, [%4];" : "=f"(v.x), "=f"(v.y), "=f"(v.z), "=f"(v.w) : "r"(a) : "memory");
    return v;
}
__device__ __forceinline__ void cluster_arrive() { asm volatile("barrier.cluster.arrive.release.aligned;" ::: "memory"); }
__device__ __forceinline__ void cluster_wait() { asm volatile("barrier.cluster.wait.acquire.aligned;" ::: "memory"); }

// Four elements of a row's result: top its largest logit (base 2), sum that of its weights, v weights times values.
// merge: parts of the prefix in the workspace that are added.
template <int D, bool PART>
__device__ __forceinline__ void write_row(const Attention& p, int64_t part, int64_t token, int64_t h, int d, float4 v, float top,
                                          float sum, int merge) {
    if (PART) {
        const int64_t at = (part * p.tokens + token) * p.q_heads + h;
        *reinterpret_cast<float4*>(static_cast<float*>(p.workspace) + at * D + d) = v;
        if (d == 0) reinterpret_cast<float2*>(static_cast<char*>(p.workspace) + p.plan.values)[at] = make_float2(top, sum);
        return;
    }
    if (merge > 0) {
        const int64_t at = token * p.q_heads + h, stride = p.tokens * p.q_heads;
        const float2* ml = reinterpret_cast<const float2*>(static_cast<const char*>(p.workspace) + p.plan.values) + at;
        const float* vals = static_cast<const float*>(p.workspace) + at * D + d;
        float most = top;
#pragma unroll 8
        for (int k = 0; k < merge; k++) most = max_nan(most, ml[k * stride].x);
        const float w = top == neg_inf() ? 0.0f : ex2(top - most);
        v.x *= w, v.y *= w, v.z *= w, v.w *= w;
        sum *= w;
        top = most;
#pragma unroll 8
        for (int k = 0; k < merge; k++) {
            const float2 m = ml[k * stride];
            const float4 u = *reinterpret_cast<const float4*>(vals + k * stride * D);
            const float x = m.x == neg_inf() ? 0.0f : ex2(m.x - top);
            sum += m.y * x;
            v.x += u.x * x, v.y += u.y * x, v.z += u.z * x, v.w += u.w * x;
        }
    }
    const bool empty = top == neg_inf();
    const float f = empty ? 0.0f : ld_f32(p.c.S_v) / sum;
    const float o[4] = {empty ? 0.0f : v.x * f, empty ? 0.0f : v.y * f, empty ? 0.0f : v.z * f, empty ? 0.0f : v.w * f};
    uint32_t w[2];
#pragma unroll
    for (int i = 0; i < 2; i++) asm("cvt.rn.bf16x2.f32 %0, %1, %2;" : "=r"(w[i]) : "f"(o[2 * i + 1]), "f"(o[2 * i]));
    uint16_t* out = static_cast<uint16_t*>(p.out.p) + token * p.out.token + h * p.out.head + d;
    if (p.out.vec) {
        *reinterpret_cast<uint2*>(out) = make_uint2(w[0], w[1]);
    } else {
#pragma unroll
        for (int i = 0; i < 4; i++) out[i] = (uint16_t)(w[i / 2] >> (16 * (i & 1)));
    }
    if (p.lse && d == 0) p.lse[token * p.q_heads + h] = empty ? neg_inf() : (top + log2f(sum) - kWeightBits) * 0.6931471805599453f;
}

template <int D, int NT, bool PREFIX, int JOIN>
__global__ void __launch_bounds__(kThreads, blocks_per_sm(D, 8 * NT)) rows_kernel(Attention p, Pass pass, int64_t part0) {
    constexpr bool PART = JOIN == kWorkspace;
    using T = Tile<D, NT>;
    __shared__ alignas(16) uint8_t s_mem[T::kSmem];
    float* s_o = reinterpret_cast<float*>(s_mem);                // [warps][R][D], over the tiles
    __shared__ float s_m[4][T::R], s_l[4][T::R], s_top[T::R], s_sum[T::R];
    if (!p.second) grid_dependency_wait();
    grid_launch_dependents();                                    // behind the wait: the next pass counts on it
    struct AtEnd {
        int wait;
        __device__ ~AtEnd() {
            if (wait) grid_dependency_wait();
        }
    } at_end{p.second};
    const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5, g = lane >> 2, t = lane & 3;
    const int head = blockIdx.y, group = p.group;
    const uint32_t parts = (uint32_t)pass.parts, b = blockIdx.x / parts, part = blockIdx.x - b * parts;

    const float S_k = ld_f32(p.c.S_k);
    int64_t row0 = 0, n, len;
    const int32_t* table;
    int64_t width;
    bool outside = false;
    if (PREFIX) {
        n = p.tokens;
        len = *p.prefix_len;
        table = p.prefix;
        width = p.prefix_width;
    } else {
        row0 = p.offsets[b];
        n = p.offsets[b + 1] - row0;
        len = p.lens[b];
        table = p.table + b * p.table_ld;
        width = p.width;
        if (row0 < 0 || n < 0 || row0 + n > p.tokens) {
            outside = true;
            n = 0;
        }
    }
    if (len < 0 || len > (width << p.c.page_log2)) {
        outside = true;
        len = len < 0 ? 0 : width << p.c.page_log2;
    }
    const bool causal = !PREFIX && p.causal;
    const int rows = (int)(PREFIX || n < p.max_q ? n : p.max_q) * group;     // at most 16
    if (p.status && outside && threadIdx.x == 0 && head == 0) atomicOr(p.status, kStatusBounds);
    if (rows == 0) return;
    // query and head of the group of row r < 16: r / group by a multiplication (group <= 16)
    const uint32_t inverse = 65536u / (uint32_t)group + 1;
    auto query_of = [&](int r) { return (int)(r * inverse >> 16); };
    // keys that the last row sees; tokens fit 31 bits
    const int shift = causal ? (int)(len - n) + 1 : (int)len, each = causal ? 1 : 0;      // row r sees shift + each query_of(r)
    const int chunk = (int)part_tokens32((uint32_t)len, parts, kWarpTokens);
    const int begin = (int)min((int64_t)part * chunk, (int64_t)INT_MAX), sees = shift + each * query_of(rows - 1);
    const int end = sees - begin > chunk ? begin + chunk : sees;
    if (PART && begin >= end) return;

    // the queries' elements: row 8 nt + g, from t D/4 on
    uint32_t qw[NT][D / 8];
#pragma unroll
    for (int nt = 0; nt < NT; nt++) {
        const int r = 8 * nt + g, i = query_of(r);
#pragma unroll
        for (int k = 0; k < D / 8; k++) qw[nt][k] = 0;
        if (r < rows) {
            const uint16_t* q = static_cast<const uint16_t*>(p.q.p) + (row0 + i) * p.q.token +
                                ((int64_t)head * group + (r - i * group)) * p.q.head + t * (D / 4);
            if (p.q.vec) {
#pragma unroll
                for (int k = 0; k < D / 32; k++) {
                    const uint4 v = *reinterpret_cast<const uint4*>(q + 8 * k);
                    qw[nt][4 * k] = v.x, qw[nt][4 * k + 1] = v.y, qw[nt][4 * k + 2] = v.z, qw[nt][4 * k + 3] = v.w;
                }
            } else {
#pragma unroll
                for (int k = 0; k < D / 8; k++) qw[nt][k] = q[2 * k] | (uint32_t)q[2 * k + 1] << 16;
            }
        }
    }

    // What the lane reads of a tile from token k0 on: keys of the 16-token group g / 2, values of group t.  A page that is
    // not there (behind the end, outside the pool) is read as page 0 and hidden afterwards.
    const int page_log2 = p.c.page_log2, page_mask = (1 << page_log2) - 1, pool = (int)p.c.pages;
    const int64_t page_codes = (int64_t)p.c.heads * D << page_log2, page_sf = page_codes / 8;      // bytes of a page
    const uint8_t *k_codes = p.c.codes + (((int64_t)head * D) << page_log2) + (g & 1) * (D / 2) + t * (D / 8);
    const uint8_t *k_sf = p.c.sf + ((head * 2ll * (D / 16) + t * T::KB) << page_log2);
    const uint8_t *v_codes = p.c.codes + (((int64_t)head * D + D / 2) << page_log2) + g * (D / 16);
    const uint8_t *v_sf = p.c.sf + (((head * 2ll + 1) * (D / 16) + g * D / 128) << page_log2);
    auto page_of = [&](int j) {
        int pg = -1;
        if (j < end) {
            pg = table[j >> page_log2];
            if ((unsigned)pg >= (unsigned)pool) outside = true, pg = -1;
        }
        return pg;
    };
    // a lane copies what it reads itself
    const uint32_t mine = (uint32_t)__cvta_generic_to_shared(s_mem) + warp * T::kWarp;
    const uint32_t m_kc = mine + lane * T::KW * 4, m_ks = mine + T::kKeys + lane * 16, m_vc = mine + T::kKeySf + lane * T::VW * 4,
                   m_vs = mine + T::kValues + lane * 16;
    auto load_keys = [&](int k0, int pg) {
        const int64_t page = pg < 0 ? 0 : pg;
        const int at = (k0 + 16 * (g >> 1)) & page_mask;
        const uint8_t *c = k_codes + page * page_codes + at * (D / 2), *f = k_sf + page * page_sf + at;
#pragma unroll
        for (int i = 0; i < 8; i++) copy_async<4 * T::KW>(m_kc + i * 32 * T::KW * 4, c + i * D);
#pragma unroll
        for (int i = 0; i < T::KB; i++) copy_async<16>(m_ks + i * 512, f + (i << page_log2));
    };
    auto load_values = [&](int k0, int pg) {
        const int64_t page = pg < 0 ? 0 : pg;
        const int at = (k0 + 16 * t) & page_mask;
        const uint8_t *c = v_codes + page * page_codes + at * (D / 2), *f = v_sf + page * page_sf + at;
#pragma unroll
        for (int i = 0; i < 16; i++) copy_async<4 * T::VW>(m_vc + i * 32 * T::VW * 4, c + i * (D / 2));
        copy_async<16>(m_vs, f);
    };
    constexpr int kStride = 4 * kWarpTokens;
    const int start = begin + warp * kWarpTokens;
    int kpg = page_of(start + 16 * (g >> 1)), vpg = page_of(start + 16 * t);
    int kpg1 = page_of(start + kStride + 16 * (g >> 1)), vpg1 = page_of(start + kStride + 16 * t);
    if (start < end) load_keys(start, kpg);
    copy_commit();
    if (start < end) load_values(start, vpg);
    copy_commit();

    // queries in fp16, scaled by a power of two a row, as the narrow operand
    uint32_t qf[NT][2 * T::KW][2];
    float fac[NT][2], m[NT][2], l[NT][2];
    int lim[NT][2], least = end;                                 // keys that a column's row sees, that every row sees
    const float S = S_k * p.scale * 1.4426950408889634f;
#pragma unroll
    for (int nt = 0; nt < NT; nt++) {
        uint32_t top = 0;                                        // bf16 bits of the row's largest magnitude
#pragma unroll
        for (int i = 0; i < D / 8; i++) top = max(top, max(qw[nt][i] & 0x7FFFu, (qw[nt][i] >> 16) & 0x7FFFu));
        top = max(top, __shfl_xor_sync(0xffffffffu, top, 1));
        top = max(top, __shfl_xor_sync(0xffffffffu, top, 2));
        // 2^-e of the largest's exponent e, within fp32's normal powers; none for infinities and NaN
        int e = (int)(top >> 7) - 127;
        if (e == 128) e = 0;
        e = e < -126 ? -126 : e > 126 ? 126 : e;
        const float down = __int_as_float((127 - e) << 23), up = __int_as_float((127 + e) << 23);
#pragma unroll
        for (int i = 0; i < D / 8; i++)
            qf[nt][i / 2][i & 1] = f16x2(bf16lo(qw[nt][i]) * down, bf16hi(qw[nt][i]) * down);
#pragma unroll
        for (int c = 0; c < 2; c++) {                            // columns 2t, 2t + 1 of the MMA's result
            const int r = 8 * nt + 2 * t + c;
            fac[nt][c] = S * __shfl_sync(0xffffffffu, up, (2 * t + c) * 4);
            if (fac[nt][c] == 0.0f) fac[nt][c] = 1e-37f;         // hidden scores, -inf, stay that
            if (fac[nt][c] > kWideFactor) least = INT_MIN;
            lim[nt][c] = r < rows ? shift + each * query_of(r) : 0;
            if (r < rows) least = min(least, lim[nt][c]);
            m[nt][c] = neg_inf();
            l[nt][c] = 0.0f;
        }
    }
    least = min(least, __shfl_xor_sync(0xffffffffu, least, 1));
    least = min(least, __shfl_xor_sync(0xffffffffu, least, 2));
    // wide rows: every tile takes the masks' branch, which has the first factors
    const bool wide = least == INT_MIN;
    if (wide) {
#pragma unroll
        for (int nt = 0; nt < NT; nt++)
#pragma unroll
            for (int c = 0; c < 2; c++) {
                const bool first = fac[nt][c] > kWideFactor;
                if (g == 0) s_m[warp][8 * nt + 2 * t + c] = first ? fac[nt][c] : 1.0f;
                if (first) fac[nt][c] = 1.0f;
            }
        __syncwarp();
    }
    float o[NT][D / 16][4];
#pragma unroll
    for (int nt = 0; nt < NT; nt++)
#pragma unroll
        for (int i = 0; i < D / 16; i++)
#pragma unroll
            for (int c = 0; c < 4; c++) o[nt][i][c] = 0.0f;

    // a tile's keys are copied over the last one's as soon as those are used, its values likewise (two groups of copies in
    // flight, keys' and values'), and its page numbers come one tile earlier
    for (int k0 = start; k0 < end; k0 += kStride) {
        const bool kv_ok = kpg >= 0, vv_ok = vpg >= 0, more = k0 + kStride < end;
        copy_wait<1>();
        __syncwarp();                                            // lanes had page numbers of their own to fetch
        uint32_t ks[T::KB][4];
#pragma unroll
        for (int i = 0; i < T::KB; i++) ld_shared(m_ks + i * 512, ks[i]);
        float sc[NT][4][4];
        const uint32_t pick0 = g & 1 ? 0x11u : 0x00u, pick1 = g & 1 ? 0x33u : 0x22u;      // the token's byte, twice
#pragma unroll
        for (int i = 0; i < 4; i++) {
            uint32_t s0[T::KB], s1[T::KB];
#pragma unroll
            for (int k = 0; k < T::KB; k++) {
                s0[k] = e4m3x2_to_f16(__byte_perm(ks[k][i], 0, pick0));
                s1[k] = e4m3x2_to_f16(__byte_perm(ks[k][i], 0, pick1));
            }
            uint32_t k0c[T::KW], k1c[T::KW];
            ld_shared(m_kc + 2 * i * 32 * T::KW * 4, k0c);
            ld_shared(m_kc + (2 * i + 1) * 32 * T::KW * 4, k1c);
#pragma unroll
            for (int w = 0; w < T::KW; w++) {
                uint32_t x[4], y[4];
                e2m1x8_to_f16(k0c[w], x);
                e2m1x8_to_f16(k1c[w], y);
#pragma unroll
                for (int h = 0; h < 2; h++) {
                    const uint32_t a[4] = {mul_h2(x[2 * h], s0[w / 2]), mul_h2(y[2 * h], s1[w / 2]),
                                           mul_h2(x[2 * h + 1], s0[w / 2]), mul_h2(y[2 * h + 1], s1[w / 2])};
#pragma unroll
                    for (int nt = 0; nt < NT; nt++) {
                        if (w + h == 0) mma16_first(sc[nt][i], a, qf[nt][0][0], qf[nt][0][1]);
                        else mma16(sc[nt][i], a, qf[nt][2 * w + h][0], qf[nt][2 * w + h][1]);
                    }
                }
            }
        }
        if (more) load_keys(k0 + kStride, kpg1);
        copy_commit();
        // Weights with the row's maximum so far; one that has grown by more than 2^kGrowth (always at the first keys) takes
        // its place, and O and the sum are scaled.
        if (!__all_sync(0xffffffffu, k0 + kWarpTokens <= least && kv_ok)) {
#pragma unroll
            for (int nt = 0; nt < NT; nt++)
#pragma unroll
                for (int i = 0; i < 4; i++)
#pragma unroll
                    for (int c = 0; c < 4; c++) {
                        const int j = k0 + 16 * (g >> 1) + 4 * i + (g & 1) + (c & 2);
                        if (wide) sc[nt][i][c] = __fmul_rn(sc[nt][i][c], s_m[warp][8 * nt + 2 * t + (c & 1)]);
                        if (!kv_ok || j >= lim[nt][c & 1] || j >= end) sc[nt][i][c] = neg_inf();
                    }
        }
        float top[NT][2];
        bool grown = false;
#pragma unroll
        for (int nt = 0; nt < NT; nt++)
#pragma unroll
            for (int c = 0; c < 2; c++) {
                float x = max3_nan(sc[nt][0][c], sc[nt][0][c + 2], sc[nt][1][c]);
                x = max3_nan(x, sc[nt][1][c + 2], sc[nt][2][c]);
                x = max3_nan(x, sc[nt][2][c + 2], sc[nt][3][c]);
                x = max_nan(x, sc[nt][3][c + 2]);
#pragma unroll
                for (int i = 4; i < 32; i *= 2) x = max_nan(x, __shfl_xor_sync(0xffffffffu, x, i));
                top[nt][c] = x * fac[nt][c];
                grown |= !(top[nt][c] <= __fadd_rd(m[nt][c], kGrowth));      // NaN: it becomes the maximum
            }
        if (__any_sync(0xffffffffu, grown)) {
#pragma unroll
            for (int nt = 0; nt < NT; nt++)
#pragma unroll
                for (int c = 0; c < 2; c++) {
                    const bool up = !(top[nt][c] <= __fadd_rd(m[nt][c], kGrowth));
                    const float alpha = !up ? 1.0f : m[nt][c] == neg_inf() ? 0.0f :
                                        ex2(__fadd_rd(kWeightBits, -top[nt][c]) - __fadd_rd(kWeightBits, -m[nt][c]));
                    if (up) m[nt][c] = top[nt][c];
                    l[nt][c] *= alpha;
#pragma unroll
                    for (int i = 0; i < D / 16; i++) o[nt][i][c] *= alpha, o[nt][i][c + 2] *= alpha;
                }
            __syncwarp();
        }
        uint32_t pt[NT][4][2];
#pragma unroll
        for (int nt = 0; nt < NT; nt++) {
            float base[2];
#pragma unroll
            for (int c = 0; c < 2; c++) base[c] = m[nt][c] == neg_inf() ? 0.0f : __fadd_rd(kWeightBits, -m[nt][c]);
#pragma unroll
            for (int i = 0; i < 4; i++)
#pragma unroll
                for (int h = 0; h < 2; h++) {
                    const float w0 = ex2(__fmaf_rn(sc[nt][i][2 * h], fac[nt][0], base[0]));
                    const float w1 = ex2(__fmaf_rn(sc[nt][i][2 * h + 1], fac[nt][1], base[1]));
                    l[nt][0] += w0, l[nt][1] += w1;
                    pt[nt][i][h] = transpose8x8(f16x2(w0, w1));
                }
        }
        copy_wait<1>();
        uint32_t vs[4];
        ld_shared(m_vs, vs);
        // scale bytes behind the last token may be anything, NaN among it, and 0 NaN is no 0
        if (!vv_ok || k0 + 16 * t + 16 > end) {
#pragma unroll
            for (int j = 0; j < 4; j++)
#pragma unroll
                for (int c = 0; c < 4; c++)
                    if (!vv_ok || k0 + 16 * t + 4 * j + c >= end) vs[j] &= ~(0xFFu << (8 * c));
        }
        __syncwarp();
#pragma unroll
        for (int i = 0; i < 4; i++) {
            const uint32_t s01 = e4m3x2_to_f16(vs[i] & 0xFFFF), s23 = e4m3x2_to_f16(vs[i] >> 16);
            uint32_t vc[4][T::VW];
#pragma unroll
            for (int c = 0; c < 4; c++) ld_shared(m_vc + (4 * i + c) * 32 * T::VW * 4, vc[c]);
#pragma unroll
            for (int w = 0; w < T::VW; w++) {
                constexpr uint32_t kLow = 0x0F0F0F0Fu;
                const uint32_t a = vc[0][w], b2 = vc[1][w], c = vc[2][w], d = vc[3][w];
                uint32_t lo01[4], hi01[4], lo23[4], hi23[4];
                e2m1x8_to_f16((a & kLow) | ((b2 << 4) & ~kLow), lo01);
                e2m1x8_to_f16(((a >> 4) & kLow) | (b2 & ~kLow), hi01);
                e2m1x8_to_f16((c & kLow) | ((d << 4) & ~kLow), lo23);
                e2m1x8_to_f16(((c >> 4) & kLow) | (d & ~kLow), hi23);
#pragma unroll
                for (int r = 0; r < 4; r++) {
                    const uint32_t v[4] = {mul_h2(lo01[r], s01), mul_h2(hi01[r], s01), mul_h2(lo23[r], s23), mul_h2(hi23[r], s23)};
#pragma unroll
                    for (int nt = 0; nt < NT; nt++) mma16(o[nt][4 * w + r], v, pt[nt][i][0], pt[nt][i][1]);
                }
            }
        }
        if (more) load_values(k0 + kStride, vpg1);
        copy_commit();
        kpg = kpg1, vpg = vpg1;
        kpg1 = page_of(k0 + 2 * kStride + 16 * (g >> 1)), vpg1 = page_of(k0 + 2 * kStride + 16 * t);
    }
    if (p.status && __any_sync(0xffffffffu, outside) && lane == 0) atomicOr(p.status, kStatusBounds);

    if (wide) {
#pragma unroll
        for (int nt = 0; nt < NT; nt++)
#pragma unroll
            for (int c = 0; c < 2; c++) {
                // what 7 - m lost
                const float norm = m[nt][c] == neg_inf() ? 1.0f : ex2(kWeightBits - (m[nt][c] + __fadd_rd(kWeightBits, -m[nt][c])));
                l[nt][c] *= norm;
#pragma unroll
                for (int i = 0; i < D / 16; i++) o[nt][i][c] *= norm, o[nt][i][c + 2] *= norm;
            }
        __syncwarp();                                            // done with the factors in s_m
    }

    // join the four warps
#pragma unroll
    for (int nt = 0; nt < NT; nt++)
#pragma unroll
        for (int c = 0; c < 2; c++)
#pragma unroll
            for (int i = 4; i < 32; i *= 2) l[nt][c] += __shfl_xor_sync(0xffffffffu, l[nt][c], i);
    if (g == 0) {
#pragma unroll
        for (int nt = 0; nt < NT; nt++)
#pragma unroll
            for (int c = 0; c < 2; c++) {
                s_m[warp][8 * nt + 2 * t + c] = m[nt][c];
                s_l[warp][8 * nt + 2 * t + c] = l[nt][c];
            }
    }
    __syncthreads();
    // 16 bytes d/4 of a row of sums; neighbouring rows' are apart in their banks
    auto place = [](int w, int r, int q) { return ((w * T::R + r) * (D / 4) + (q ^ (r & 7))) * 4; };
#pragma unroll
    for (int nt = 0; nt < NT; nt++)
#pragma unroll
        for (int c = 0; c < 2; c++) {
            const int r = 8 * nt + 2 * t + c;
            const float top = max_nan(max_nan(s_m[0][r], s_m[1][r]), max_nan(s_m[2][r], s_m[3][r]));
            const float w = m[nt][c] == neg_inf() ? 0.0f : ex2(m[nt][c] - top);
            // the lane's dims of this row: g D/8 + 0, 1, ..
#pragma unroll
            for (int i = 0; i < D / 16; i += 2)
                *reinterpret_cast<float4*>(s_o + place(warp, r, g * (D / 32) + i / 2)) =
                    make_float4(o[nt][i][c] * w, o[nt][i][c + 2] * w, o[nt][i + 1][c] * w, o[nt][i + 1][c + 2] * w);
        }
    if (threadIdx.x < T::R) {
        const int r = threadIdx.x;
        float top = neg_inf(), sum = 0.0f;
#pragma unroll
        for (int w = 0; w < 4; w++) top = max_nan(top, s_m[w][r]);
#pragma unroll
        for (int w = 0; w < 4; w++) sum += s_m[w][r] == neg_inf() ? 0.0f : s_l[w][r] * ex2(s_m[w][r] - top);
        s_top[r] = top, s_sum[r] = sum;
    }
    __syncthreads();
    // parts of the prefix to be added
    int merge = 0;
    if (JOIN != kWorkspace && p.plan.merge) {
        const int64_t most = p.prefix_width << page_log2;
        int64_t n2 = *p.prefix_len;
        n2 = n2 < 0 ? 0 : n2 > most ? most : n2;
        const uint32_t size = part_tokens32((uint32_t)n2, (uint32_t)p.plan.prefix.parts, (uint32_t)p.plan.prefix.step());
        merge = (int)(((uint32_t)n2 + size - 1) / size);
        grid_dependency_wait();                                  // its pass
    }
    // the block's sums, four neighbouring elements to a thread, into the first warp's place
    for (int x = threadIdx.x; x < rows * (D / 4); x += kThreads) {
        const int r = x / (D / 4), q = x % (D / 4);
        float4 v = *reinterpret_cast<const float4*>(s_o + place(0, r, q));
#pragma unroll
        for (int w = 1; w < 4; w++) {
            const float4 u = *reinterpret_cast<const float4*>(s_o + place(w, r, q));
            v.x += u.x, v.y += u.y, v.z += u.z, v.w += u.w;
        }
        if (JOIN == kCluster) {
            *reinterpret_cast<float4*>(s_o + place(0, r, q)) = v;
        } else {
            const int i = query_of(r);
            write_row<D, PART>(p, part0 + part, row0 + i, (int64_t)head * group + (r - i * group), 4 * q, v, s_top[r], s_sum[r], merge);
        }
    }
    if (JOIN == kCluster) {
        __syncwarp();                                            // half a warp may have had a row more
        cluster_arrive();
        cluster_wait();
        for (int x = (int)part * kThreads + threadIdx.x; x < rows * (D / 4); x += (int)parts * kThreads) {
            const int r = x / (D / 4), q = x % (D / 4);
            float tops[kMaxCluster], top = neg_inf(), sum = 0.0f;
#pragma unroll
            for (uint32_t k = 0; k < kMaxCluster; k++) {
                tops[k] = k < parts ? ld_cluster(cluster_addr(&s_top[r], k)) : neg_inf();
                top = max_nan(top, tops[k]);
            }
            float4 v = make_float4(0.0f, 0.0f, 0.0f, 0.0f);
#pragma unroll
            for (uint32_t k = 0; k < kMaxCluster; k++) {
                if (k >= parts || tops[k] == neg_inf()) continue;
                const float w = ex2(tops[k] - top);
                const float4 u = ld_cluster4(cluster_addr(s_o + place(0, r, q), k));
                sum += ld_cluster(cluster_addr(&s_sum[r], k)) * w;
                v.x += u.x * w, v.y += u.y * w, v.z += u.z * w, v.w += u.w * w;
            }
            const int i = query_of(r);
            write_row<D, false>(p, 0, row0 + i, (int64_t)head * group + (r - i * group), 4 * q, v, top, sum, merge);
        }
        __syncwarp();
        cluster_arrive();                                        // a block's memory stays until the others have read it
        cluster_wait();
    }
}

// A row's parts joined: a block of four warps for each row, every fourth part to a warp.
constexpr int kJoinWarps = 4;
template <int D>
__global__ void __launch_bounds__(32 * kJoinWarps) join_kernel(Attention p) {
    __shared__ float s_o[kJoinWarps][D], s_sum[kJoinWarps];
    grid_launch_dependents();
    grid_dependency_wait();
    const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
    const int64_t at = blockIdx.x;
    const int64_t token = at / p.q_heads, h = at - token * p.q_heads;
    int64_t lo = 0, hi = p.batch + 1;
    while (hi > lo) {
        const int64_t mid = (lo + hi) >> 1;
        if (p.offsets[mid] > token) hi = mid;
        else lo = mid + 1;
    }
    const int64_t b = lo - 1;
    if (b < 0 || b >= p.batch) return;
    const int64_t n = p.offsets[b + 1] - p.offsets[b], i = token - p.offsets[b];
    if (i >= p.max_q || n < 0 || p.offsets[b] < 0 || p.offsets[b] + n > p.tokens) return;
    int64_t len = p.lens[b], most = p.width << p.c.page_log2;
    len = len < 0 ? 0 : len > most ? most : len;
    const int64_t sees = p.causal ? len - n + i + 1 : len;
    const int64_t chunk = part_tokens(len, p.plan.own.parts, p.plan.own.step());
    const int64_t own = sees <= 0 ? 0 : (sees + chunk - 1) / chunk;
    int64_t shared = 0;
    if (p.prefix_len) {
        int64_t len2 = *p.prefix_len;
        most = p.prefix_width << p.c.page_log2;
        len2 = len2 < 0 ? 0 : len2 > most ? most : len2;
        if (p.plan.prefix.parts) {
            const int64_t c2 = part_tokens(len2, p.plan.prefix.parts, p.plan.prefix.step());
            shared = (len2 + c2 - 1) / c2;
        }
    }
    // parts 0 .. own - 1 and those of the prefix, behind the most that a sequence has
    const float2* ml = reinterpret_cast<const float2*>(static_cast<const char*>(p.workspace) + p.plan.values);
    const float* vals = static_cast<const float*>(p.workspace);
    const int64_t stride = p.tokens * p.q_heads, parts = own + shared;
    float top = neg_inf();
    for (int64_t k = lane; k < parts; k += 32) {                 // every warp looks at all of them
        const float2 v = ml[(k < own ? k : p.plan.own.parts + k - own) * stride + at];
        top = max_nan(top, v.x);
    }
#pragma unroll
    for (int k = 16; k; k /= 2) top = max_nan(top, __shfl_xor_sync(0xffffffffu, top, k));
    constexpr int N = D / 32;
    float sum = 0.0f, o[N];
#pragma unroll
    for (int k = 0; k < N; k++) o[k] = 0.0f;
#pragma unroll 4
    for (int64_t k = warp; k < parts; k += kJoinWarps) {
        const int64_t x = (k < own ? k : p.plan.own.parts + k - own) * stride + at;
        const float2 v = ml[x];
        const float w = v.x == neg_inf() ? 0.0f : ex2(v.x - top);
        sum += v.y * w;
        float q[N];
        if constexpr (N == 4) {
            const float4 f = *reinterpret_cast<const float4*>(vals + x * D + lane * 4);
            q[0] = f.x, q[1] = f.y, q[2] = f.z, q[3] = f.w;
        } else {
            const float2 f = *reinterpret_cast<const float2*>(vals + x * D + lane * 2);
            q[0] = f.x, q[1] = f.y;
        }
#pragma unroll
        for (int c = 0; c < N; c++) o[c] += q[c] * w;
    }
#pragma unroll
    for (int c = 0; c < N; c++) s_o[warp][lane * N + c] = o[c];
    if (lane == 0) s_sum[warp] = sum;
    __syncthreads();
    if (warp != 0) return;
#pragma unroll
    for (int k = 1; k < kJoinWarps; k++) {
        sum += s_sum[k];
#pragma unroll
        for (int c = 0; c < N; c++) o[c] += s_o[k][lane * N + c];
    }
    const float f = top == neg_inf() ? 0.0f : ld_f32(p.c.S_v) / sum;
    uint16_t* out = static_cast<uint16_t*>(p.out.p) + token * p.out.token + h * p.out.head + lane * N;
    uint32_t w[N / 2];
#pragma unroll
    for (int c = 0; c < N / 2; c++) {
        const float a = top == neg_inf() ? 0.0f : o[2 * c] * f, b2 = top == neg_inf() ? 0.0f : o[2 * c + 1] * f;
        asm("cvt.rn.bf16x2.f32 %0, %1, %2;" : "=r"(w[c]) : "f"(b2), "f"(a));
    }
    if (p.out.vec) {
        if constexpr (N == 4) *reinterpret_cast<uint2*>(out) = make_uint2(w[0], w[1]);
        else *reinterpret_cast<uint32_t*>(out) = w[0];
    } else {
#pragma unroll
        for (int c = 0; c < N; c++) out[c] = (uint16_t)(w[c / 2] >> (16 * (c & 1)));
    }
    if (p.lse && lane == 0)
        p.lse[at] = top == neg_inf() ? neg_inf() : (top + log2f(sum) - kWeightBits) * 0.6931471805599453f;
}

template <int D, int NT, bool PREFIX, int JOIN>
cudaError_t launch_rows(const Attention& p, const Pass& pass, int64_t part0, cudaStream_t s) {
    cudaLaunchConfig_t cfg = {};
    cfg.gridDim = dim3((unsigned)((PREFIX ? 1 : p.batch) * pass.parts), (unsigned)p.c.heads);
    cfg.blockDim = dim3(kThreads);
    cfg.stream = s;
    cudaLaunchAttribute attr[2];
    attr[0].id = cudaLaunchAttributeProgrammaticStreamSerialization;
    attr[0].val.programmaticStreamSerializationAllowed = 1;
    attr[1].id = cudaLaunchAttributeClusterDimension;
    attr[1].val.clusterDim.x = (unsigned)pass.parts;
    attr[1].val.clusterDim.y = attr[1].val.clusterDim.z = 1;
    cfg.attrs = attr;
    cfg.numAttrs = JOIN == kCluster ? 2 : 1;
    return cudaLaunchKernelEx(&cfg, rows_kernel<D, NT, PREFIX, JOIN>, p, pass, part0);
}

template <int D, int NT>
cudaError_t dispatch(const Attention& p, const Pass& pass, bool prefix, int64_t part0, cudaStream_t s) {
    if (prefix) return launch_rows<D, NT, true, kWorkspace>(p, pass, part0, s);
    if (p.plan.through && !p.plan.merge) return launch_rows<D, NT, false, kWorkspace>(p, pass, part0, s);
    return pass.parts > 1 ? launch_rows<D, NT, false, kCluster>(p, pass, part0, s) : launch_rows<D, NT, false, kAlone>(p, pass, part0, s);
}

template <int D>
cudaError_t launch_pass(const Attention& p, const Pass& pass, bool prefix, int64_t part0, cudaStream_t s) {
    if (pass.rows >= kTileRows) return launch_tiles(p, pass, prefix, part0, s);
    return pass.rows == 8 ? dispatch<D, 1>(p, pass, prefix, part0, s) : dispatch<D, 2>(p, pass, prefix, part0, s);
}

template <int D>
cudaError_t launch(const Attention& p, cudaStream_t s) {
    const Plan& plan = p.plan;
    if (!plan.prefix.parts) {
        const cudaError_t e = launch_pass<D>(p, plan.own, false, 0, s);
        return e != cudaSuccess || !plan.through ? e : launch_dependent(join_kernel<D>, p.tokens * p.q_heads, 32 * kJoinWarps, s, p);
    }
    Attention second = p;
    second.second = 1;
    cudaError_t e = launch_pass<D>(p, plan.prefix, true, plan.merge ? 0 : plan.own.parts, s);
    if (e == cudaSuccess) e = launch_pass<D>(second, plan.own, false, 0, s);
    if (e == cudaSuccess && !plan.merge) e = launch_dependent(join_kernel<D>, p.tokens * p.q_heads, 32 * kJoinWarps, s, p);
    return e;
}

}  // namespace

cudaError_t launch_attention(const Attention& p, cudaStream_t s) {
    return p.c.dim == 64 ? launch<64>(p, s) : launch<128>(p, s);
}

}  // namespace kv
}  // namespace nvfp4

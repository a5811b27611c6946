// Device parts that the products on quantised operands share: tensor-core
// instructions past those of tc_gemm.cuh, operand formats, the activation, and what
// the epilogues write.
#pragma once
#include <cuda_bf16.h>

#include "fp4_kernels.h"
#include "tc_gemm.cuh"

namespace nvfp4 {
namespace mm {

using namespace tc;

// Instruction descriptor.  kind::f16: D fp32 (bits 4-5 = 1), A and B bf16 (7-9, 10-12 =
// 1), N >> 3 (17-22), M >> 4 (24-28).  kind::mxf4nvf4: A and B E2M1 (7-9, 10-12 = 1), N >> 3
// (17-22), scales UE4M3 = 0 or UE8M0 = 1 (23), M >> 7 (27-28), which of a cell's scale
// bytes the MMA takes for B (4-5) and A (29-30).  Operands K-major but where bits 15 (A) and 16 (B)
// say otherwise, K = 32 bytes.
__host__ __device__ constexpr uint32_t idesc(int kind, int m, int n) {
    return kind == kBf16 ? (1u << 4) | (1u << 7) | (1u << 10) | ((uint32_t)(n >> 3) << 17) | ((uint32_t)(m >> 4) << 24)
                         : (1u << 7) | (1u << 10) | ((uint32_t)(n >> 3) << 17) | (kind == kMxfp4 ? 1u << 23 : 0u) |
                               ((uint32_t)(m >> 7) << 27);
}
constexpr uint32_t kAlongA = 1u << 15, kAlongB = 1u << 16;
__host__ __device__ constexpr uint32_t sf_id(uint32_t id) { return id << 4 | id << 29; }

// Descriptor of a 512-byte scale atom for tcgen05.cp: no swizzle, 16-byte rows, 8-row
// groups 128 bytes apart.
__device__ __forceinline__ uint64_t atom_desc(uint32_t addr) {
    return (uint64_t)((addr >> 4) & 0x3FFFu) | (uint64_t)(128 >> 4) << 16 | (uint64_t)(128 >> 4) << 32 | (uint64_t)1 << 46;
}

template <int CG>
__device__ __forceinline__ void cp_atom(uint32_t taddr, uint64_t desc) {
    if (CG == 1)
        asm volatile("tcgen05.cp.cta_group::1.32x128b.warpx4 [%0], %1;" ::"r"(taddr), "l"(desc) : "memory");
    else
        asm volatile("tcgen05.cp.cta_group::2.32x128b.warpx4 [%0], %1;" ::"r"(taddr), "l"(desc) : "memory");
}

#define MM_MMA(CG, KIND)                                                                                            \
    "{\n\t.reg .pred p;\n\tsetp.ne.b32 p, %4, 0;\n\ttcgen05.mma.cta_group::" CG ".kind::" KIND " [%0], %1, %2, %3, " \
    "[%5], [%6], p;\n\t}"
template <int KIND, int CG>
__device__ __forceinline__ void mma(uint32_t d, uint64_t a, uint64_t b, uint32_t id, uint32_t accumulate, uint32_t sfa,
                                    uint32_t sfb) {
    static_assert(KIND != kBf16 || CG == 2, "bf16 products are pairs'");
    if (KIND == kBf16) {
        asm volatile("{\n\t.reg .pred p;\n\tsetp.ne.b32 p, %4, 0;\n\ttcgen05.mma.cta_group::2.kind::f16 [%0], %1, %2, %3, p;\n\t}"
                     ::"r"(d), "l"(a), "l"(b), "r"(id), "r"(accumulate) : "memory");
    } else if (KIND == kNvfp4) {
        if (CG == 1)
            asm volatile(MM_MMA("1", "mxf4nvf4.block_scale.scale_vec::4X")
                         ::"r"(d), "l"(a), "l"(b), "r"(id), "r"(accumulate), "r"(sfa), "r"(sfb) : "memory");
        else
            asm volatile(MM_MMA("2", "mxf4nvf4.block_scale.scale_vec::4X")
                         ::"r"(d), "l"(a), "l"(b), "r"(id), "r"(accumulate), "r"(sfa), "r"(sfb) : "memory");
    } else {
        if (CG == 1)
            asm volatile(MM_MMA("1", "mxf4nvf4.block_scale.scale_vec::2X")
                         ::"r"(d), "l"(a), "l"(b), "r"(id), "r"(accumulate), "r"(sfa), "r"(sfb) : "memory");
        else
            asm volatile(MM_MMA("2", "mxf4nvf4.block_scale.scale_vec::2X")
                         ::"r"(d), "l"(a), "l"(b), "r"(id), "r"(accumulate), "r"(sfa), "r"(sfb) : "memory");
    }
}
#undef MM_MMA

__device__ __forceinline__ void tma_load_3d(uint32_t dst, const CUtensorMap* map, int c0, int c1, int c2, uint32_t bar) {
    asm volatile(
        "cp.async.bulk.tensor.3d.shared::cluster.global.tile.mbarrier::complete_tx::bytes [%0], [%1, {%2, %3, %4}], [%5];"
        ::"r"(dst), "l"(reinterpret_cast<uint64_t>(map)), "r"(c0), "r"(c1), "r"(c2), "r"(bar)
        : "memory");
}

__device__ __forceinline__ void tmem_wait16(float (&a)[16]) {
    asm volatile("tcgen05.wait::ld.sync.aligned;"
                 : "+f"(a[0]), "+f"(a[1]), "+f"(a[2]), "+f"(a[3]), "+f"(a[4]), "+f"(a[5]), "+f"(a[6]), "+f"(a[7]),
                   "+f"(a[8]), "+f"(a[9]), "+f"(a[10]), "+f"(a[11]), "+f"(a[12]), "+f"(a[13]), "+f"(a[14]), "+f"(a[15])
                 :: "memory");
}

// 32 consecutive accumulator columns; there after tmem_wait32, which names them.
__device__ __forceinline__ void tmem_ld32(uint32_t taddr, float (&v)[32]) {
    asm volatile(
        "tcgen05.ld.sync.aligned.32x32b.x32.b32 "
        "{%0, %1, %2, %3, %4, %5, %6, %7, %8, %9, %10, %11, %12, %13, %14, %15, "
        "%16, %17, %18, %19, %20, %21, %22, %23, %24, %25, %26, %27, %28, %29, %30, %31}, [%32];"
        : "=f"(v[0]), "=f"(v[1]), "=f"(v[2]), "=f"(v[3]), "=f"(v[4]), "=f"(v[5]), "=f"(v[6]), "=f"(v[7]),
          "=f"(v[8]), "=f"(v[9]), "=f"(v[10]), "=f"(v[11]), "=f"(v[12]), "=f"(v[13]), "=f"(v[14]), "=f"(v[15]),
          "=f"(v[16]), "=f"(v[17]), "=f"(v[18]), "=f"(v[19]), "=f"(v[20]), "=f"(v[21]), "=f"(v[22]), "=f"(v[23]),
          "=f"(v[24]), "=f"(v[25]), "=f"(v[26]), "=f"(v[27]), "=f"(v[28]), "=f"(v[29]), "=f"(v[30]), "=f"(v[31])
        : "r"(taddr)
        : "memory");
}
__device__ __forceinline__ void tmem_wait32(float (&v)[32]) {
    asm volatile("tcgen05.wait::ld.sync.aligned;"
        : "+f"(v[0]), "+f"(v[1]), "+f"(v[2]), "+f"(v[3]), "+f"(v[4]), "+f"(v[5]), "+f"(v[6]), "+f"(v[7]),
          "+f"(v[8]), "+f"(v[9]), "+f"(v[10]), "+f"(v[11]), "+f"(v[12]), "+f"(v[13]), "+f"(v[14]), "+f"(v[15]),
          "+f"(v[16]), "+f"(v[17]), "+f"(v[18]), "+f"(v[19]), "+f"(v[20]), "+f"(v[21]), "+f"(v[22]), "+f"(v[23]),
          "+f"(v[24]), "+f"(v[25]), "+f"(v[26]), "+f"(v[27]), "+f"(v[28]), "+f"(v[29]), "+f"(v[30]), "+f"(v[31])
        :: "memory");
}

// One thread of a converged warp.  A role's warp runs its loop with all lanes and elects
// one to issue: the operands of TMA and tensor-core instructions then stay in uniform registers,
// where a branch on the thread's number cost ~50 cycles an instruction to move them there
// (a stage of 12 scale copies and 4 MMAs: 1500 cycles for 512 of MMA).
__device__ __forceinline__ bool elect_one() {
    uint32_t p;
    asm volatile("{\n\t.reg .pred q;\n\telect.sync _|q, 0xFFFFFFFF;\n\tselp.u32 %0, 1, 0, q;\n\t}" : "=r"(p));
    return p != 0;
}
__device__ __forceinline__ int warp_index() { return __shfl_sync(0xFFFFFFFFu, (int)(threadIdx.x >> 5), 0); }

// mbar_wait by all lanes of a warp, with one answer for all of them.
__device__ __forceinline__ bool mbar_wait_warp(uint32_t bar, uint32_t parity) {
    if (__all_sync(0xFFFFFFFFu, mbar_try_wait(bar, parity))) return true;
    const unsigned long long t0 = now_ns();
    while (!__all_sync(0xFFFFFFFFu, mbar_try_wait(bar, parity)))
        if (__any_sync(0xFFFFFFFFu, now_ns() - t0 > kWaitNs)) return false;
    return true;
}

// A ring of K-stages: slot, its address and the parity of its current use.
struct Ring {
    uint32_t first, at;
    int slot = 0;
    uint32_t parity = 0;
    __device__ __forceinline__ explicit Ring(uint32_t base, uint32_t parity_ = 0) : first(base), at(base), parity(parity_) {}
    __device__ __forceinline__ void next(int stages, int bytes) {
        at += bytes;
        if (++slot == stages) slot = 0, at = first, parity ^= 1;
    }
};

__device__ __forceinline__ uint32_t cluster_rank() {
    uint32_t r;
    asm("mov.u32 %0, %%cluster_ctarank;" : "=r"(r));
    return r;
}
__device__ __forceinline__ void cluster_barrier() {
    asm volatile("barrier.cluster.arrive.release.aligned;\n\tbarrier.cluster.wait.acquire.aligned;" ::: "memory");
}
__device__ __forceinline__ uint32_t at_rank(uint32_t addr, uint32_t rank) {
    uint32_t r;
    asm("mapa.shared::cluster.u32 %0, %1, %2;" : "=r"(r) : "r"(addr), "r"(rank));
    return r;
}
__device__ __forceinline__ float ld_cluster(uint32_t addr) {
    float v;
    asm volatile("ld.shared::cluster.f32 %0, [%1];" : "=f"(v) : "r"(addr) : "memory");
    return v;
}
__device__ __forceinline__ void st_cluster(uint32_t addr, int v) {
    asm volatile("st.shared::cluster.b32 [%0], %1;" ::"r"(addr), "r"(v) : "memory");
}
__device__ __forceinline__ void st_cluster(uint32_t addr, float v) {
    asm volatile("st.shared::cluster.f32 [%0], %1;" ::"r"(addr), "f"(v) : "memory");
}

// What the accumulators become.
struct Epilogue {
    int act;
    int64_t T, N;                  // rows (tokens) and columns of the result
    const float *s_p, *s_p2, *s_q; // global scales or null
    void* out;                     // D, or h (bf16) or null
    void* out2;                    // rows from row2 on (pairs of CTAs, plain) or null
    int64_t row2, rows1;
    int out_f32;
    int64_t ldo;
    uint8_t *h_codes, *h_sf;
    uint32_t h_kpad4;
    const uint16_t* dh;
    int64_t lddh;
    uint16_t* dgu;
    int64_t fp;
    int* status;
};

// act(g) and, where wanted, its derivative.  Both activations are g * p with p a sigmoid
// (of g, or of 2 z for (1 + tanh z) / 2).  z is the sigmoid's argument, dz its derivative.  p and 1 - p are
// 1 / (1 + e) and e / (1 + e), e = exp(-|z|): neither is a difference, and the quotient's divisor is at most 2, so
// both keep their relative accuracy down to fp32's smallest numbers.  exp and the reciprocal by their fast forms:
// CUDA documents 2 + |1.173 z| units of 2^-23 for the first, which with what rounding z makes of it is below 2^-14
// wherever e is not zero; bf16 results are rounded by up to 2^-8.
__device__ __forceinline__ float fast_rcp(float x) {
    float r;
    asm("rcp.approx.ftz.f32 %0, %1;" : "=f"(r) : "f"(x));
    return r;
}
template <bool GRAD>
__device__ __forceinline__ float gate_by(float g, float z, float dz, float& da) {
    const float e = __expf(-fabsf(z)), r = fast_rcp(1.0f + e), s = r * e;
    const float p = z < 0.0f ? s : r, a = g * p;
    if (GRAD) da = fmaf(a * (z < 0.0f ? r : s), dz, p);
    return a;
}
template <bool GRAD>
__device__ __forceinline__ void gelu_argument(float g, float& z, float& dz) {
    // dz is a factor of a (1 - p), which is 0 long before |g| = 2^10, so g^2 need not overflow there
    const float g2 = GRAD ? fminf(g * g, 1048576.0f) : g * g;
    z = 1.5957691216f * g * fmaf(0.044715f, g2, 1.0f);       // 2 sqrt(2/pi)
    if (GRAD) dz = 1.5957691216f * fmaf(0.134145f, g2, 1.0f);
}
template <bool GRAD>
__device__ __forceinline__ float activate(int act, float g, float& da) {
    float z = g, dz = 1.0f;
    if (act == 1) gelu_argument<GRAD>(g, z, dz);
    return gate_by<GRAD>(g, z, dz, da);
}
// The same for 32 values in place, the branch on the activation outside.
template <bool GRAD>
__device__ __forceinline__ void activate32(int act, float (&g)[32], float* da) {
    float unused;
    if (act == 1) {
#pragma unroll
        for (int j = 0; j < 32; j++) {
            float z, dz = 1.0f;
            gelu_argument<GRAD>(g[j], z, dz);
            g[j] = gate_by<GRAD>(g[j], z, dz, GRAD ? da[j] : unused);
        }
    } else {
#pragma unroll
        for (int j = 0; j < 32; j++) g[j] = gate_by<GRAD>(g[j], g[j], 1.0f, GRAD ? da[j] : unused);
    }
}

__device__ __forceinline__ uint16_t bf16_bits(float x) { return __bfloat16_as_ushort(__float2bfloat16_rn(x)); }
__device__ __forceinline__ float bf16_value(uint16_t b) { return __uint_as_float((uint32_t)b << 16); }
__device__ __forceinline__ float scale_or_1(const float* s) { return s ? ld_f32(s) : 1.0f; }

// ---- host side
inline bool make_operand_map(CUtensorMap* m, const Operand& o, int kind, int64_t k, uint32_t box_rows) {
    const EncodeTiledFn enc = encode_fn();
    if (!enc) return false;
    const bool bf = kind == kBf16;
    // K along the row: boxes of 128 bytes of K by box_rows; else 64 rows by 64 steps of K
    const cuuint64_t dims[2] = {(cuuint64_t)(!bf ? k / 2 : o.along ? o.rows : k), (cuuint64_t)(o.along ? k : o.rows)};
    const cuuint64_t strides[1] = {(cuuint64_t)(bf ? 2 * o.ld : k / 2)};
    const cuuint32_t box[2] = {bf ? 64u : 128u, o.along ? 64u : box_rows};
    const cuuint32_t es[2] = {1, 1};
    return enc(m, bf ? CU_TENSOR_MAP_DATA_TYPE_BFLOAT16 : CU_TENSOR_MAP_DATA_TYPE_UINT8, 2, const_cast<void*>(o.data), dims,
               strides, box, es, CU_TENSOR_MAP_INTERLEAVE_NONE, CU_TENSOR_MAP_SWIZZLE_128B, CU_TENSOR_MAP_L2_PROMOTION_L2_256B,
               CU_TENSOR_MAP_FLOAT_OOB_FILL_NONE) == CUDA_SUCCESS;
}

// The scale atoms as [row block][atom along K][128 words], `blocks` of the first to a box.
inline bool make_scale_map(CUtensorMap* m, const Operand& o, int kind, int64_t k, int blocks = 1) {
    const EncodeTiledFn enc = encode_fn();
    if (!enc) return false;
    const int64_t kb = k / (kind == kMxfp4 ? 32 : 16), k4 = (kb + 3) / 4;
    const cuuint64_t dims[3] = {128, (cuuint64_t)k4, (cuuint64_t)((o.rows + 127) / 128)};
    const cuuint64_t strides[2] = {(cuuint64_t)kAtom, (cuuint64_t)(k4 * kAtom)};
    const cuuint32_t box[3] = {128, (cuuint32_t)atoms(kind), (cuuint32_t)blocks};
    const cuuint32_t es[3] = {1, 1, 1};
    return enc(m, CU_TENSOR_MAP_DATA_TYPE_UINT32, 3, const_cast<uint8_t*>(o.sf), dims, strides, box, es,
               CU_TENSOR_MAP_INTERLEAVE_NONE, CU_TENSOR_MAP_SWIZZLE_NONE, CU_TENSOR_MAP_L2_PROMOTION_L2_256B,
               CU_TENSOR_MAP_FLOAT_OOB_FILL_NONE) == CUDA_SUCCESS;
}

inline Epilogue make_epilogue(const Product& p) {
    Epilogue e = {};
    e.act = p.act;
    e.T = p.q.rows;
    e.N = p.p.rows;
    e.s_p = p.p.S;
    e.s_p2 = p.p2.S;
    e.s_q = p.q.S;
    e.out = p.out;
    e.out2 = p.out2;
    e.row2 = p.row2;
    e.rows1 = p.out2 ? p.rows1 : p.q.rows;
    e.out_f32 = p.out_f32;
    e.ldo = p.ldo;
    e.h_codes = p.h_codes;
    e.h_sf = p.h_sf;
    e.h_kpad4 = (uint32_t)((p.p.rows / 32 + 3) / 4);
    e.dh = static_cast<const uint16_t*>(p.dh);
    e.lddh = p.lddh;
    e.dgu = static_cast<uint16_t*>(p.dgu);
    e.fp = p.fp;
    e.status = p.status;
    return e;
}

}  // namespace mm
}  // namespace nvfp4

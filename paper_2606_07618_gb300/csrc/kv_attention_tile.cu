// Attention over the NVFP4 key/value cache for many rows a key head: prompts, and batches that
// share a prefix (nvfp4_kv_attention, nvfp4_kv_attention_prefix), on tcgen05.
//
// A block takes 256 rows (query, head of the group) of one key head, as two tiles of 128, and
// walks the keys of its part 128 at a time; where it has one tile of rows, the even and the odd keys are its two streams,
// joined at the end.  Codes become fp16 once for all rows: q s (without S) is exact in fp16, as are queries scaled by a
// power of two a row (kv_attention.cu), so both products are kind::f16 MMAs with fp32 sums.
//
//   warps 8-11  a thread a token: its codes and scales from global memory (the next two items' bytes are in
//               flight while this one waits for room), converted, into 128-byte-swizzled shared
//               memory: keys read by the MMA along their rows, values across theirs
//   warp 12     issues S = Q K^T of both streams, then, as soon as a stream's weights are there, its
//               O += P V and its next S: while one stream's softmax runs, the tensor cores do the other's
//               products
//   warps 0-7   softmax, a thread a row: maximum, weights to fp16 over the scores' own columns of
//               tensor memory (P is the MMA's operand from there), the sum; O stays in tensor memory.
//               O is scaled only when a row's maximum has grown by more than 2^8 (weights are held
//               2^7-fold, so that they stay below fp16's largest; large logits: kWideFactor).
//
// Tensor memory: scores of both streams 2 x 128 columns, O 2 x dim.  Shared memory: Q 64 KB, two stages each
// of keys and values of 32 KB (dim 128).
//
// A step of 256 rows and 128 keys (dim 128) takes about 3500 cycles, its MMAs 2048 at their rate.  S = Q K^T takes 670 a
// tile for 512: it reads 8 KB of operands per 64 cycles, all that shared memory gives, while the loads' stores want
// some of it (without those 394 us of 455 then; without softmax, too, 348).  So on long parts two CTAs take 512 rows as a
// pair (kv_plan.h): their MMAs have 256 rows, and each CTA holds, and converts, half of every tile's keys and values.  What
// is left, 3100 cycles a step, is a stream's chain: products 1024, the softmax of a tile 1800, of them 930 for its exponentials.
// 2 x 2048 queries of 32 heads over 8192 tokens: 375 us, 1.28 PFLOP/s (single CTAs 418; plain products at their rate: 250).
//
// Every mbarrier wait is bounded (1 s): a role that gives up stops, the others do after it,
// bit 4 (16) of the status word is set and what is missing is not written.
#include "fp4_tile.cuh"
#include "kv_kernels.h"

namespace nvfp4 {
namespace kv {
namespace {

using namespace mm;

constexpr int kSoftmaxWarps = 8, kLoadWarps = 4, kMmaWarp = kSoftmaxWarps + kLoadWarps;
// Four warps to a quarter of the SM, three of the last four idle: of its 4 x 128 registers a thread, softmax takes 2 x 176, loads 112, MMAs 48.
constexpr int kTileThreads = 32 * (kMmaWarp + 4);
constexpr int kSoftmaxRegs = 176, kLoadRegs = 112, kMmaRegs = 48;
constexpr int kKeys = 128, kRows = 128;
constexpr float kBits = 7.0f, kGrowth = 8.0f;

__device__ __forceinline__ float neg_inf() { return __int_as_float(0xff800000); }
__device__ __forceinline__ float ex2(float x) {
    float y;
    asm("ex2.approx.ftz.f32 %0, %1;" : "=f"(y) : "f"(x));
    return y;
}
__device__ __forceinline__ float max3_nan(float a, float b, float c) {
    float d;
    asm("max.NaN.f32 %0, %1, %2, %3;" : "=f"(d) : "f"(a), "f"(b), "f"(c));
    return d;
}
__device__ __forceinline__ uint32_t f16x2(float lo, float hi) {
    uint32_t r;
    asm("cvt.rn.f16x2.f32 %0, %1, %2;" : "=r"(r) : "f"(hi), "f"(lo));
    return r;
}
__device__ __forceinline__ uint32_t mul_h2(uint32_t a, uint32_t b) {
    uint32_t d;
    asm("mul.rn.f16x2 %0, %1, %2;" : "=r"(d) : "r"(a), "r"(b));
    return d;
}
__device__ __forceinline__ uint32_t scale_pair(uint32_t code2) {    // an E4M3 code twice -> its fp16 value twice
    uint32_t h;
    asm("cvt.rn.f16x2.e4m3x2 %0, %1;" : "=r"(h) : "h"((uint16_t)code2));
    return h;
}
__device__ __forceinline__ uint4 e2m1x8_scaled(uint32_t w, uint32_t s) {
    uint4 h;
    asm("{\n\t.reg .b8 a, b, c, d;\n\tmov.b32 {a, b, c, d}, %4;\n\t"
        "cvt.rn.f16x2.e2m1x2 %0, a;\n\tcvt.rn.f16x2.e2m1x2 %1, b;\n\t"
        "cvt.rn.f16x2.e2m1x2 %2, c;\n\tcvt.rn.f16x2.e2m1x2 %3, d;\n\t}"
        : "=r"(h.x), "=r"(h.y), "=r"(h.z), "=r"(h.w) : "r"(w));
    return make_uint4(mul_h2(h.x, s), mul_h2(h.y, s), mul_h2(h.z, s), mul_h2(h.w, s));
}
__device__ __forceinline__ void st_shared16(uint32_t addr, const uint4& v) {
    asm volatile("st.shared.v4.b32 [%0], {%1, %2, %3, %4};" ::"r"(addr), "r"(v.x), "r"(v.y), "r"(v.z), "r"(v.w) : "memory");
}
// A whole sector.
__device__ __forceinline__ void st_global32(void* p, const uint32_t* v) {
    asm volatile("st.global.v8.b32 [%0], {%1, %2, %3, %4, %5, %6, %7, %8};" ::"l"(p), "r"(v[0]), "r"(v[1]), "r"(v[2]), "r"(v[3]),
                 "r"(v[4]), "r"(v[5]), "r"(v[6]), "r"(v[7]) : "memory");
}
// 32 columns of this thread's lane of tensor memory; the values are there after wait_ld32.
__device__ __forceinline__ void tmem_ld32(uint32_t a, float (&v)[32]) {
    asm volatile(
        "tcgen05.ld.sync.aligned.32x32b.x32.b32 "
        "{%0, %1, %2, %3, %4, %5, %6, %7, %8, %9, %10, %11, %12, %13, %14, %15, %16, %17, %18, %19, %20, %21, %22, %23, "
        "%24, %25, %26, %27, %28, %29, %30, %31}, [%32];"
        : "=f"(v[0]), "=f"(v[1]), "=f"(v[2]), "=f"(v[3]), "=f"(v[4]), "=f"(v[5]), "=f"(v[6]), "=f"(v[7]), "=f"(v[8]),
          "=f"(v[9]), "=f"(v[10]), "=f"(v[11]), "=f"(v[12]), "=f"(v[13]), "=f"(v[14]), "=f"(v[15]), "=f"(v[16]), "=f"(v[17]),
          "=f"(v[18]), "=f"(v[19]), "=f"(v[20]), "=f"(v[21]), "=f"(v[22]), "=f"(v[23]), "=f"(v[24]), "=f"(v[25]), "=f"(v[26]),
          "=f"(v[27]), "=f"(v[28]), "=f"(v[29]), "=f"(v[30]), "=f"(v[31])
        : "r"(a)
        : "memory");
}
__device__ __forceinline__ void wait_ld32(float (&v)[32]) {
    asm volatile("tcgen05.wait::ld.sync.aligned;"
                 : "+f"(v[0]), "+f"(v[1]), "+f"(v[2]), "+f"(v[3]), "+f"(v[4]), "+f"(v[5]), "+f"(v[6]), "+f"(v[7]), "+f"(v[8]),
                   "+f"(v[9]), "+f"(v[10]), "+f"(v[11]), "+f"(v[12]), "+f"(v[13]), "+f"(v[14]), "+f"(v[15]), "+f"(v[16]),
                   "+f"(v[17]), "+f"(v[18]), "+f"(v[19]), "+f"(v[20]), "+f"(v[21]), "+f"(v[22]), "+f"(v[23]), "+f"(v[24]),
                   "+f"(v[25]), "+f"(v[26]), "+f"(v[27]), "+f"(v[28]), "+f"(v[29]), "+f"(v[30]), "+f"(v[31])
                 :: "memory");
}
// Values of a load that another wait covers: no use of them moves above this.
__device__ __forceinline__ void hold32(float (&v)[32]) {
#pragma unroll
    for (int i = 0; i < 32; i++) asm volatile("" : "+f"(v[i]));
}
__device__ __forceinline__ void tmem_st16(uint32_t a, const uint32_t (&v)[16]) {
    asm volatile(
        "tcgen05.st.sync.aligned.32x32b.x16.b32 [%0], "
        "{%1, %2, %3, %4, %5, %6, %7, %8, %9, %10, %11, %12, %13, %14, %15, %16};" ::"r"(a),
        "r"(v[0]), "r"(v[1]), "r"(v[2]), "r"(v[3]), "r"(v[4]), "r"(v[5]), "r"(v[6]), "r"(v[7]), "r"(v[8]), "r"(v[9]), "r"(v[10]),
        "r"(v[11]), "r"(v[12]), "r"(v[13]), "r"(v[14]), "r"(v[15])
        : "memory");
}
__device__ __forceinline__ void tmem_wait_st() { asm volatile("tcgen05.wait::st.sync.aligned;" ::: "memory"); }
template <int N>
__device__ __forceinline__ void regs_up() { asm volatile("setmaxnreg.inc.sync.aligned.u32 %0;" ::"n"(N)); }
template <int N>
__device__ __forceinline__ void regs_down() { asm volatile("setmaxnreg.dec.sync.aligned.u32 %0;" ::"n"(N)); }
// fp16 products; CG: the CTAs that they span.
template <int CG>
__device__ __forceinline__ void mma_ss(uint32_t d, uint64_t a, uint64_t b, uint32_t id, uint32_t accumulate) {
    if (CG == 1)
        asm volatile("{\n\t.reg .pred p;\n\tsetp.ne.b32 p, %4, 0;\n\ttcgen05.mma.cta_group::1.kind::f16 [%0], %1, %2, %3, p;\n\t}"
                     ::"r"(d), "l"(a), "l"(b), "r"(id), "r"(accumulate) : "memory");
    else
        asm volatile("{\n\t.reg .pred p;\n\tsetp.ne.b32 p, %4, 0;\n\ttcgen05.mma.cta_group::2.kind::f16 [%0], %1, %2, %3, p;\n\t}"
                     ::"r"(d), "l"(a), "l"(b), "r"(id), "r"(accumulate) : "memory");
}
template <int CG>
__device__ __forceinline__ void mma_ts(uint32_t d, uint32_t a, uint64_t b, uint32_t id, uint32_t accumulate) {
    if (CG == 1)
        asm volatile("{\n\t.reg .pred p;\n\tsetp.ne.b32 p, %4, 0;\n\ttcgen05.mma.cta_group::1.kind::f16 [%0], [%1], %2, %3, p;\n\t}"
                     ::"r"(d), "r"(a), "l"(b), "r"(id), "r"(accumulate) : "memory");
    else
        asm volatile("{\n\t.reg .pred p;\n\tsetp.ne.b32 p, %4, 0;\n\ttcgen05.mma.cta_group::2.kind::f16 [%0], [%1], %2, %3, p;\n\t}"
                     ::"r"(d), "r"(a), "l"(b), "r"(id), "r"(accumulate) : "memory");
}
// Arrival at the barrier when the MMAs issued so far are done; CG 2: at that of both CTAs.
template <int CG>
__device__ __forceinline__ void commit_to(uint64_t* bar) {
    if (CG == 1)
        mma_commit(smem_u32(bar));
    else
        asm volatile("tcgen05.commit.cta_group::2.mbarrier::arrive::one.shared::cluster.multicast::cluster.b64 [%0], %1;"
                     ::"r"(smem_u32(bar)), "h"((uint16_t)3) : "memory");
}
// Arrival at the first CTA's barrier.  A pair's orders tensor memory's accesses alone (with tcgen05's fences before and after).
template <int CG>
__device__ __forceinline__ void signal(uint64_t* bar) {
    if (CG == 1)
        mbar_arrive(smem_u32(bar));
    else
        asm volatile("mbarrier.arrive.relaxed.cluster.shared::cluster.b64 _, [%0];" ::"r"(at_rank(smem_u32(bar), 0)) : "memory");
}
// A pair's that orders shared memory, too.  From the threads that load or weigh, with their accesses in flight, it costs far more
// (510 and 470 us where 375 is reached so), so one that has none of its own gives it for them.
__device__ __forceinline__ void signal_all(uint64_t* bar) {
    asm volatile("mbarrier.arrive.release.cluster.shared::cluster.b64 _, [%0];" ::"r"(at_rank(smem_u32(bar), 0)) : "memory");
}
__device__ __forceinline__ bool try_wait_cluster(uint32_t bar, uint32_t parity) {
    uint32_t ok;
    asm volatile("{\n\t.reg .pred p;\n\tmbarrier.try_wait.parity.acquire.cluster.shared::cta.b64 p, [%1], %2;\n\tselp.u32 %0, 1, 0, p;\n\t}"
                 : "=r"(ok) : "r"(bar), "r"(parity) : "memory");
    return __all_sync(0xffffffffu, ok != 0);
}
template <int CG>
__device__ __forceinline__ bool wait_signal(uint64_t* b, uint32_t parity) {
    const uint32_t bar = smem_u32(b);
    if (CG == 1) return mbar_wait_warp(bar, parity);
    if (try_wait_cluster(bar, parity)) return true;
    const unsigned long long t0 = now_ns();
    while (!try_wait_cluster(bar, parity))
        if (__any_sync(0xffffffffu, now_ns() - t0 > kWaitNs)) return false;
    return true;
}

// kind::f16 with fp16 operands: D fp32 (bits 4-5 = 1), A and B fp16 (0), B's K along its rows or (bit 16) across them.
__host__ __device__ constexpr uint32_t idesc_f16(int m, int n, bool across) {
    return (1u << 4) | (across ? 1u << 16 : 0u) | ((uint32_t)(n >> 3) << 17) | ((uint32_t)(m >> 4) << 24);
}

template <int D, int CG>
struct Shape {
    static constexpr int kPanels = D / 64;                       // of 64 elements (128 bytes) a row
    static constexpr int kPanel = 128 * 128;                     // 128 rows
    static constexpr int kOp = kPanels * kPanel;                 // an operand: 128 rows of D fp16
    // A CTA's part of a tile of keys and of values: of a pair's, 64 keys, and 64 of the values' elements.
    static constexpr int kKeyPanel = kPanel / CG, kStage = kOp / CG;
    static constexpr int kSmem = 2 * kOp + 4 * kStage + 1024;    // Q twice, two stages of K and V
    static constexpr int kScores = 0, kOut = 256;                // columns of tensor memory
};

struct Bars {
    uint64_t k_full[2], k_empty[2], v_full[2], v_empty[2], s_full[2], p_full[2], o_full, drained, joined, q_full;
};

// A token's codes and scales of K or V on their way.
template <int D>
struct Held {
    uint4 w[D / 32];
    uint32_t s[D / 16];                                          // scale codes, not touched before they are used
    __device__ __forceinline__ void load(const uint8_t* codes, const uint8_t* sf, int page_log2) {
#pragma unroll
        for (int i = 0; i < D / 32; i++) w[i] = *reinterpret_cast<const uint4*>(codes + 16 * i);
#pragma unroll
        for (int i = 0; i < D / 16; i++) s[i] = sf[i << page_log2];
    }
    // into a row of an operand, whose address has the row's swizzle in its chunk bits (16 bytes: 8 elements)
    __device__ __forceinline__ void store(uint32_t row) const {
#pragma unroll
        for (int b = 0; b < D / 16; b++) {
            const uint32_t sc = scale_pair(s[b] | s[b] << 8);
            const uint4& v = w[b / 2];
            const uint32_t at = (row ^ ((2 * b & 7) << 4)) + (b >> 2) * Shape<128, 1>::kPanel;
            st_shared16(at, e2m1x8_scaled(b & 1 ? v.z : v.x, sc));
            st_shared16(at ^ 16, e2m1x8_scaled(b & 1 ? v.w : v.y, sc));
        }
    }
};

// CG 2: a pair of CTAs, whose MMAs span both: tiles of 256 rows, 128 in each.
template <int D, bool PREFIX, bool PART, int CG>
__global__ void __launch_bounds__(kTileThreads, 1) tile_kernel(Attention p, Pass pass, int64_t part0) {
    using H = Shape<D, CG>;
    static_assert(CG == 1 || D == 128, "a pair's values come in 64 elements a CTA");
    constexpr int kTile = CG * kRows;                            // rows of an MMA
    const uint32_t rank = CG == 2 ? cluster_rank() : 0;
    extern __shared__ uint8_t smem_raw[];
    __shared__ Bars s_bars;
    __shared__ uint32_t s_tmem, s_hidden[4][4];
    __shared__ float2 s_ml[kRows];
    __shared__ int s_abort;
    if (!p.second) grid_dependency_wait();
    grid_launch_dependents();                                    // behind the wait: the next pass counts on it
    struct AtEnd {
        int wait;
        __device__ ~AtEnd() {
            if (wait) grid_dependency_wait();
        }
    } at_end{p.second};
    const int tid = threadIdx.x, warp = tid >> 5, lane = tid & 31;
    const int head = blockIdx.y;
    // tiles from the last one on: with a causal mask it has the most keys
    const int64_t per = PREFIX ? pass.parts : pass.parts * p.batch;
    const int64_t block = blockIdx.x / CG, tile = pass.tiles - 1 - block / per, rest = block % per;
    const int64_t part = PREFIX ? rest : rest % pass.parts, b = PREFIX ? 0 : rest / pass.parts;

    int64_t row0 = 0, n, len, width;
    const int32_t* table;
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
    if (p.status && outside && tid == 0 && head == 0) atomicOr(p.status, kStatusBounds);
    const bool causal = !PREFIX && p.causal;
    const int64_t rows = (PREFIX || n < p.max_q ? n : p.max_q) * p.group, first = tile * 2 * kTile;
    if (first >= rows) return;
    const int64_t last = (first + 2 * kTile < rows ? first + 2 * kTile : rows) - 1;
    const int64_t sees = causal ? len - n + last / p.group + 1 : len;
    const int64_t chunk = part_tokens(len, pass.parts, kTileKeys), begin = part * chunk;
    const int64_t end = begin + chunk < sees ? begin + chunk : sees;
    if (PART && begin >= end) return;
    const int tiles = end > begin ? (int)((end - begin + kKeys - 1) / kKeys) : 0;      // a part is less than 2^31 tokens
    // two streams of scores, weights and sums: of both tiles of rows; where there is only one (split), of its even and odd keys
    const bool split = CG == 1 && rows - first <= kRows && tiles > 1;
    const int both = rows - first > kTile || split;

    const uint32_t base = (smem_u32(smem_raw) + 1023) & ~1023u;
    const uint32_t sq = base, sk = base + 2 * H::kOp, sv = sk + 2 * H::kStage;
    if (warp == kMmaWarp) {
        if (CG == 1) {
            tmem_alloc(smem_u32(&s_tmem), 512);
        } else {
            asm volatile("tcgen05.alloc.cta_group::2.sync.aligned.shared::cta.b32 [%0], %1;" ::"r"(smem_u32(&s_tmem)), "r"(512) : "memory");
            asm volatile("tcgen05.relinquish_alloc_permit.cta_group::2.sync.aligned;" ::: "memory");
        }
    }
    if (tid == 0) {
        const int more = CG == 2 && rank == 0;                   // the other CTA's word
        for (int i = 0; i < 2; i++) {
            mbar_init(smem_u32(&s_bars.k_full[i]), 4 + more + (p.starve == 1));
            mbar_init(smem_u32(&s_bars.v_full[i]), 4 + more + (p.starve == 2));
            mbar_init(smem_u32(&s_bars.k_empty[i]), 1);
            mbar_init(smem_u32(&s_bars.v_empty[i]), 1);
            mbar_init(smem_u32(&s_bars.s_full[i]), 1);
            mbar_init(smem_u32(&s_bars.p_full[i]), CG * 4);
        }
        mbar_init(smem_u32(&s_bars.o_full), 1);
        mbar_init(smem_u32(&s_bars.drained), 1);
        mbar_init(smem_u32(&s_bars.joined), 4);
        mbar_init(smem_u32(&s_bars.q_full), kSoftmaxWarps + more);
        s_abort = 0;
        asm volatile("fence.mbarrier_init.release.cluster;" ::: "memory");
    }

    tc_fence_before();
    __syncthreads();
    if (CG == 2) cluster_barrier();                              // both CTAs' barriers and tensor memory are there
    tc_fence_after();
    const uint32_t tmem = s_tmem;

    bool ok = true;
    const int half = warp >> 2;                                  // tile of this warp's rows (softmax warps)
    const int64_t row = CG == 2 ? first + half * kTile + (int)rank * kRows + (tid & 127) : first + (split ? tid & 127 : tid);
    if (warp >= kSoftmaxWarps && warp < kMmaWarp) {
        regs_down<kLoadRegs>();
        // Items: keys of a tile, then its values.  The next two items' bytes are on their way, and the page number after
        // them; nothing looks at a load's result before its item's turn.  A page that is not there (behind the end, outside
        // the pool) is read as page 0: its keys are hidden, its values' scales zero (NaN times a weight of 0 is no 0).
        const int t = tid & 127, page_log2 = p.c.page_log2, page_mask = (1 << page_log2) - 1, pool = (int)p.c.pages;
        const int64_t page_codes = (int64_t)p.c.heads * D << page_log2, page_sf = page_codes / 8;  // bytes of a page
        const uint8_t *codes = p.c.codes + ((int64_t)head * D << page_log2), *sf = p.c.sf + ((int64_t)head * (D / 8) << page_log2);
        // A pair's CTA: of the keys a half of 64 of them to a thread, of the values the CTA's half of each.
        constexpr int E = D / CG;                                // elements of a thread
        const int kt = CG == 2 ? (int)rank * 64 + (t >> 1) : t, kr = CG == 2 ? t >> 1 : t, kh = CG == 2 ? t & 1 : 0;
        const uint8_t *k_codes = codes + kh * (E / 2), *k_sf = sf + ((int64_t)(kh * (E / 16)) << page_log2);
        const uint8_t *v_codes = codes + ((int64_t)(D / 2) << page_log2) + rank * (E / 2);
        const uint8_t *v_sf = sf + ((int64_t)(D / 16 + rank * (E / 16)) << page_log2);
        const int stop = (int)end;
        auto entry = [&](int j, int at) {                        // page number of a token of tile j, unchecked
            const int64_t x = begin + (int64_t)j * kKeys + at;
            return x < stop ? table[x >> page_log2] : 0;
        };
        auto fetch = [&](Held<E>& h, int j, int at, const uint8_t* c, const uint8_t* f, int page) {
            const int off = (int)((uint32_t)begin + (uint32_t)(j * kKeys + at)) & page_mask;
            const int64_t pg = (unsigned)page < (unsigned)pool ? page : 0;
            h.load(c + pg * page_codes + off * (D / 2), f + pg * page_sf + off, page_log2);
        };
        const uint32_t k_row = sk + kh * H::kKeyPanel + kr * 128 + ((kr & 7) << 4), v_row = sv + t * 128 + ((t & 7) << 4);
        Held<E> now, next;
        int page = entry(0, t), page1 = entry(1, t);             // of the values now and next, and after them
        int k_page1 = CG == 2 ? entry(1, kt) : 0;                // of the keys after the next
        if (tiles > 0) {
            fetch(now, 0, kt, k_codes, k_sf, CG == 2 ? entry(0, kt) : page);
            fetch(next, 0, t, v_codes, v_sf, page);
        }
#pragma unroll 1
        for (int i = 0; i < 2 * tiles; i++) {
            const int j = i >> 1, part = i & 1, st = j & 1;
            uint64_t *empty = (part ? s_bars.v_empty : s_bars.k_empty) + st, *full = (part ? s_bars.v_full : s_bars.k_full) + st;
            const bool there = begin + (int64_t)j * kKeys + t < stop, ok_page = (unsigned)page < (unsigned)pool;
            if (part == 1 && !(there && ok_page)) {
#pragma unroll
                for (int k = 0; k < E / 16; k++) now.s[k] = 0;
            }
            if (j >= 2 && !mbar_wait_warp(smem_u32(empty), ((j >> 1) & 1) ^ 1)) { ok = false; break; }
            if (part == 0) {
                const uint32_t mask = __ballot_sync(0xffffffffu, there && !ok_page);
                if (lane == 0) s_hidden[j & 3][warp - kSoftmaxWarps] = mask;
                outside |= there && !ok_page;
            }
            now.store((part ? v_row : k_row) + st * H::kStage);
            fence_proxy_async();
            __syncwarp();
            if (lane == 0) mbar_arrive(smem_u32(full));
            now = next;
            if (j + 1 < tiles) {
                if (part == 0) fetch(next, j + 1, kt, k_codes, k_sf, CG == 2 ? k_page1 : page1);
                else fetch(next, j + 1, t, v_codes, v_sf, page1);
            }
            if (part == 1) {
                page = page1;
                page1 = entry(j + 2, t);
                if (CG == 2) k_page1 = entry(j + 2, kt);
            }
        }
        if (p.status && __any_sync(0xffffffffu, outside) && lane == 0) atomicOr(p.status, kStatusBounds);
    } else if (warp >= kMmaWarp) {
        regs_down<kMmaRegs>();
        if (warp == kMmaWarp && rank == 0) {
        // all lanes run the loop and one is elected to issue, so that descriptors stay in uniform registers
        constexpr uint32_t id_s = idesc_f16(kTile, kKeys, false), id_o = idesc_f16(kTile, D, true);
        auto scores = [&](int x, int st) {
            if (elect_one()) {
                const uint64_t a = smem_desc(sq + x * H::kOp, 16, 1024), bd = smem_desc(sk + st * H::kStage, 16, 1024);
#pragma unroll
                for (int kk = 0; kk < D / 16; kk++)
                    mma_ss<CG>(tmem + H::kScores + x * 128, a + (((kk >> 2) * H::kPanel + (kk & 3) * 32) >> 4),
                               bd + (((kk >> 2) * H::kKeyPanel + (kk & 3) * 32) >> 4), id_s, kk != 0);
                commit_to<CG>(&s_bars.s_full[x]);
            }
            __syncwarp();
        };
        auto commit = [&](uint64_t* bar) {
            if (elect_one()) commit_to<CG>(bar);
            __syncwarp();
        };
        auto outputs = [&](int x, int st, bool first_keys) {
            if (elect_one()) {
                const uint64_t bd = smem_desc(sv + st * H::kStage, H::kPanel, 1024);
#pragma unroll
                for (int kk = 0; kk < kKeys / 16; kk++)
                    mma_ts<CG>(tmem + H::kOut + x * D, tmem + H::kScores + x * 128 + kk * 8, bd + (kk * 16 * 128 >> 4), id_o,
                               (uint32_t)(!first_keys | kk));
            }
            __syncwarp();
        };
        auto wait_for = [&](uint64_t* bar, int parity) {
            ok = ok && wait_signal<CG>(bar, parity & 1);
            tc_fence_after();
            return ok;
        };
        wait_for(&s_bars.q_full, 0);
        if (split) {
            for (int j = 0; j < 2 && wait_for(&s_bars.k_full[j], 0); j++) {
                scores(j, j);
                commit(&s_bars.k_empty[j]);
            }
            for (int j = 0; ok && j < tiles; j++) {
                const int st = j & 1;
                if (!wait_for(&s_bars.v_full[st], j >> 1) || !wait_for(&s_bars.p_full[st], j >> 1)) break;
                outputs(st, st, j < 2);
                commit(&s_bars.v_empty[st]);
                if (j + 2 < tiles && wait_for(&s_bars.k_full[st], (j + 2) >> 1)) {
                    scores(st, st);
                    commit(&s_bars.k_empty[st]);
                }
            }
        } else if (tiles > 0) {
            if (wait_for(&s_bars.k_full[0], 0)) {
                scores(0, 0);
                if (both) scores(1, 0);
                commit(&s_bars.k_empty[0]);
            }
            for (int j = 0; ok && j < tiles; j++) {
                const int st = j & 1, nx = (j + 1) & 1;
                if (!wait_for(&s_bars.v_full[st], j >> 1)) break;
                for (int x = 0; ok && x <= both; x++) {
                    if (!wait_for(&s_bars.p_full[x], j)) break;
                    outputs(x, st, j == 0);
                    if (j + 1 < tiles && (x == 1 || wait_for(&s_bars.k_full[nx], (j + 1) >> 1))) scores(x, nx);
                }
                if (!ok) break;
                commit(&s_bars.v_empty[st]);
                if (j + 1 < tiles) commit(&s_bars.k_empty[nx]);
            }
        }
        // after every MMA issued: to the softmax warps, too, where none is missing
        uint64_t* done = ok ? &s_bars.o_full : &s_bars.drained;
        commit(done);
        if (!mbar_wait_warp(smem_u32(done), 0)) ok = false;
        } else if (CG == 2 && warp == kMmaWarp) {
            // the second CTA's operands are there: said here for its warps
            auto relay = [&](uint64_t* bar, int parity) {
                if (ok) ok = mbar_wait_warp(smem_u32(bar), parity & 1);
                tc_fence_after();
                tc_fence_before();
                if (ok && lane == 0) signal_all(bar);
            };
            relay(&s_bars.q_full, 0);
            if (tiles > 0) relay(&s_bars.k_full[0], 0);
            for (int j = 0; ok && j < tiles; j++) {
                const int st = j & 1, nx = (j + 1) & 1;
                relay(&s_bars.v_full[st], j >> 1);
                if (j + 1 < tiles) relay(&s_bars.k_full[nx], (j + 1) >> 1);
            }
        }
    } else {
        regs_up<kSoftmaxRegs>();
        // queries to fp16, scaled by a power of two a row
        float fac = 0.0f;
        int lim = 1 << 30;                                        // keys that the row sees of this part
        uint32_t w[D / 2];
#pragma unroll
        for (int i = 0; i < D / 2; i++) w[i] = 0;
        if (row < rows) {
            const uint16_t* q = static_cast<const uint16_t*>(p.q.p) + (row0 + row / p.group) * p.q.token +
                                (head * (int64_t)p.group + row % p.group) * p.q.head;
            if (p.q.vec) {
#pragma unroll
                for (int i = 0; i < D / 8; i++) {
                    const uint4 v = *reinterpret_cast<const uint4*>(q + 8 * i);
                    w[4 * i] = v.x, w[4 * i + 1] = v.y, w[4 * i + 2] = v.z, w[4 * i + 3] = v.w;
                }
            } else {
#pragma unroll
                for (int i = 0; i < D / 2; i++) w[i] = q[2 * i] | (uint32_t)q[2 * i + 1] << 16;
            }
            const int64_t all = causal ? len - n + row / p.group + 1 : len;
            const int64_t seen = (all < end ? all : end) - begin;
            lim = seen < 0 ? 0 : (int)seen;
        }
        uint32_t top = 0;
#pragma unroll
        for (int i = 0; i < D / 2; i++) top = max(top, max(w[i] & 0x7FFFu, (w[i] >> 16) & 0x7FFFu));
        int e = (int)(top >> 7) - 127;
        if (e == 128) e = 0;                                     // infinities and NaN stay what they are
        e = e < -126 ? -126 : e > 126 ? 126 : e;
        const float down = __int_as_float((127 - e) << 23), up = __int_as_float((127 + e) << 23);
        fac = ld_f32(p.c.S_k) * p.scale * 1.4426950408889634f * up;
        if (fac == 0.0f) fac = 1e-37f;                           // hidden scores, -inf, stay that
        const float first_fac = fac > kWideFactor ? fac : 1.0f;
        if (fac > kWideFactor) fac = 1.0f;
#pragma unroll
        for (int i = 0; i < D / 8; i++) {
            uint32_t h[4];
#pragma unroll
            for (int j = 0; j < 4; j++) h[j] = f16x2(bf16lo(w[4 * i + j]) * down, bf16hi(w[4 * i + j]) * down);
            const int r = tid & 127;
            st_shared16(sq + half * H::kOp + (i >> 3) * H::kPanel + r * 128 + (((i & 7) ^ (r & 7)) << 4),
                        make_uint4(h[0], h[1], h[2], h[3]));
        }
        fence_proxy_async();
        __syncwarp();
        if (lane == 0) mbar_arrive(smem_u32(&s_bars.q_full));
        if (half == 0 || both) {
        const uint32_t lanes = tmem + ((uint32_t)(warp & 3) << 21);      // this warp's lanes
        const uint32_t ts = lanes + H::kScores + half * 128, to = lanes + H::kOut + half * D;
        float m = neg_inf(), l = 0.0f;
        const int step = split ? 2 : 1;
        int turn = 0;
        for (int j = split ? half : 0; j < tiles; j += step, turn++) {
            if (!mbar_wait_warp(smem_u32(&s_bars.s_full[half]), turn & 1)) { ok = false; break; }
            tc_fence_after();
            const int left = lim - j * kKeys;                    // visible keys from this tile on
            uint32_t hid[4];
#pragma unroll
            for (int c = 0; c < 4; c++) hid[c] = s_hidden[j & 3][c];
            const bool whole = __all_sync(0xffffffffu, left >= kKeys && first_fac == 1.0f && !(hid[0] | hid[1] | hid[2] | hid[3]));
            float v[4][32];
#pragma unroll
            for (int c = 0; c < 4; c++) tmem_ld32(ts + 32 * c, v[c]);
            wait_ld32(v[0]);
#pragma unroll
            for (int c = 1; c < 4; c++) hold32(v[c]);
            if (!whole) {
#pragma unroll
                for (int c = 0; c < 4; c++)
#pragma unroll
                    for (int i = 0; i < 32; i++)
                        v[c][i] = 32 * c + i >= left || (hid[c] >> i & 1) ? neg_inf() : __fmul_rn(v[c][i], first_fac);
                __syncwarp();
            }
            float tops[4];
#pragma unroll
            for (int c = 0; c < 4; c++) {
                float a = max3_nan(v[c][0], v[c][1], v[c][2]), b2 = max3_nan(v[c][3], v[c][4], v[c][5]);
#pragma unroll
                for (int i = 6; i < 30; i += 4) {
                    a = max3_nan(a, v[c][i], v[c][i + 1]);
                    b2 = max3_nan(b2, v[c][i + 2], v[c][i + 3]);
                }
                tops[c] = max3_nan(max3_nan(a, v[c][30], v[c][31]), b2, b2);
            }
            const float top = max3_nan(max3_nan(tops[0], tops[1], tops[2]), tops[3], tops[3]) * fac;
            const bool grown = top > __fadd_rd(m, kGrowth);
            if (__any_sync(0xffffffffu, grown)) {
                const float alpha = !grown ? 1.0f : m == neg_inf() ? 0.0f : ex2(__fadd_rd(kBits, -top) - __fadd_rd(kBits, -m));
                if (grown) m = top;
                l *= alpha;
                __syncwarp();                                    // the lanes together for tensor memory
                if (turn > 0) {
#pragma unroll 1
                    for (int c = 0; c < D; c += 16) {
                        float o[16], z[16];
                        tmem_ld16(to + c, o);
                        tmem_wait_ld(o, z);
                        uint32_t u[16];
#pragma unroll
                        for (int i = 0; i < 16; i++) u[i] = __float_as_uint(o[i] * alpha);
                        tmem_st16(to + c, u);
                    }
                }
            }
            const float shift = m == neg_inf() ? 0.0f : __fadd_rd(kBits, -m);
            const u64 f2 = pack2(fac, fac), s2 = pack2(shift, shift), one2 = pack2(1.0f, 1.0f);
            u64 sums[2] = {0ull, 0ull};
#pragma unroll
            for (int c = 0; c < 4; c++) {
                uint32_t w[16];
#pragma unroll
                for (int i = 0; i < 16; i++) {
                    float a, b2;
                    unpack2(fma2(pack2(v[c][2 * i], v[c][2 * i + 1]), f2, s2), a, b2);
                    a = ex2(a);
                    b2 = ex2(b2);
                    sums[i & 1] = fma2(pack2(a, b2), one2, sums[i & 1]);
                    w[i] = f16x2(a, b2);
                }
                tmem_st16(ts + 16 * c, w);
            }
            float a, b2, c2, d2;
            unpack2(sums[0], a, b2);
            unpack2(sums[1], c2, d2);
            l += (a + b2) + (c2 + d2);
            tmem_wait_st();
            tc_fence_before();
            __syncwarp();
            if (lane == 0) signal<CG>(&s_bars.p_full[half]);
        }
        if (ok && !mbar_wait_warp(smem_u32(&s_bars.o_full), 0)) ok = false;
        tc_fence_after();
        const float norm = m == neg_inf() ? 1.0f : ex2(kBits - (m + __fadd_rd(kBits, -m)));        // what 7 - m lost (kWideFactor)
        l *= norm;
        // split: the second stream's maximum, sum and O through shared memory (the queries' place) to the first
        float w0 = norm, w1 = 0.0f;
        const int r = tid & 127;
        auto other = [&](int q) { return sq + (uint32_t)(r * D * 4) + ((q ^ (r & 7)) << 4); };      // 16 bytes of O
        if (split && ok) {
            if (half == 1) {
                s_ml[r] = make_float2(m, l);
#pragma unroll 1
                for (int c = 0; c < D; c += 16) {
                    float o[16], z[16];
                    tmem_ld16(to + c, o);
                    tmem_wait_ld(o, z);
#pragma unroll
                    for (int i = 0; i < 4; i++)
                        st_shared16(other(c / 4 + i), make_uint4(__float_as_uint(o[4 * i] * norm), __float_as_uint(o[4 * i + 1] * norm),
                                                                 __float_as_uint(o[4 * i + 2] * norm), __float_as_uint(o[4 * i + 3] * norm)));
                }
                __syncwarp();
                if (lane == 0) mbar_arrive(smem_u32(&s_bars.joined));
            } else if (!mbar_wait_warp(smem_u32(&s_bars.joined), 0)) {
                ok = false;
            } else {
                const float2 v = s_ml[r];
                const float top = fmaxf(m, v.x);
                const float w = m == neg_inf() ? 0.0f : ex2(m - top);
                w0 = w * norm;
                w1 = v.x == neg_inf() ? 0.0f : ex2(v.x - top);
                m = top;
                l = l * w + v.y * w1;                            // a NaN sum stays one
            }
        }
        if (ok && !(split && half == 1)) {
            const int64_t token = row0 + row / p.group, h = head * (int64_t)p.group + row % p.group;
            const int64_t at = PART ? ((part0 + part) * p.tokens + token) * p.q_heads + h : token * p.q_heads + h;
            const float f = (PART ? 1.0f : ld_f32(p.c.S_v) / l) * (split ? 1.0f : norm);
            const bool empty = m == neg_inf() && l == 0.0f;      // saw nothing (a NaN among its scores makes the sum NaN)
            const bool valid = row < rows;
            __syncwarp();
#pragma unroll
            for (int c = 0; c < D; c += 16) {
                float o[16], z[16];
                if (tiles > 0) {
                    tmem_ld16(to + c, o);
                    tmem_wait_ld(o, z);
                }
                if (split) {
#pragma unroll
                    for (int i = 0; i < 4; i++) {
                        float4 u;
                        asm volatile("ld.shared.v4.f32 {%0, %1, %2, %3}, [%4];" : "=f"(u.x), "=f"(u.y), "=f"(u.z), "=f"(u.w)
                                     : "r"(other(c / 4 + i)) : "memory");
                        o[4 * i] = o[4 * i] * w0 + u.x * w1, o[4 * i + 1] = o[4 * i + 1] * w0 + u.y * w1;
                        o[4 * i + 2] = o[4 * i + 2] * w0 + u.z * w1, o[4 * i + 3] = o[4 * i + 3] * w0 + u.w * w1;
                    }
                }
#pragma unroll
                for (int i = 0; i < 16; i++) o[i] = empty ? 0.0f : o[i] * f;
                if (valid && PART) {
                    float* d = static_cast<float*>(p.workspace) + at * D + c;
                    uint32_t u[16];
#pragma unroll
                    for (int i = 0; i < 16; i++) u[i] = __float_as_uint(o[i]);
                    st_global32(d, u);
                    st_global32(d + 8, u + 8);
                } else if (valid) {
                    uint32_t w[8];
#pragma unroll
                    for (int i = 0; i < 8; i++)
                        asm("cvt.rn.bf16x2.f32 %0, %1, %2;" : "=r"(w[i]) : "f"(o[2 * i + 1]), "f"(o[2 * i]));
                    uint16_t* d = static_cast<uint16_t*>(p.out.p) + token * p.out.token + h * p.out.head + c;
                    if (p.out.vec == 2) {
                        st_global32(d, w);
                    } else {
#pragma unroll
                        for (int i = 0; i < 16; i++) d[i] = (uint16_t)(w[i / 2] >> (16 * (i & 1)));
                    }
                }
                __syncwarp();                                    // lanes without a row stored nothing
            }
            if (valid) {
                // a NaN sum shows in both
                if (PART)
                    reinterpret_cast<float2*>(static_cast<char*>(p.workspace) + p.plan.values)[at] =
                        make_float2(l != l ? l : empty ? neg_inf() : m, l);
                else if (p.lse)
                    p.lse[at] = empty ? neg_inf() : (m + log2f(l) - kBits) * 0.6931471805599453f;
            }
        }
    }
    }
    if (!ok) atomicOr(&s_abort, 1);
    __syncwarp();
    tc_fence_before();
    __syncthreads();
    tc_fence_after();
    if (CG == 2) cluster_barrier();                              // neither signals the other's barriers any more
    if (warp == kMmaWarp) {
        if (CG == 1) tmem_dealloc(tmem, 512);
        else asm volatile("tcgen05.dealloc.cta_group::2.sync.aligned.b32 %0, %1;" ::"r"(tmem), "r"(512) : "memory");
    }
    if (tid == 0 && s_abort && p.status) atomicOr(p.status, kStatusTimeout);
}

template <int D, bool PREFIX, bool PART, int CG>
cudaError_t launch(const Attention& p, const Pass& pass, int64_t part0, cudaStream_t s) {
    static std::atomic<uint64_t> opted;                          // devices whose shared memory limit is raised
    constexpr int kSmem = Shape<D, CG>::kSmem;
    const auto kernel = tile_kernel<D, PREFIX, PART, CG>;
    int dev = 0;
    cudaError_t e = cudaGetDevice(&dev);
    if (e != cudaSuccess) return e;
    const uint64_t bit = dev < 64 ? 1ull << dev : 0;
    if (!(opted.load(std::memory_order_relaxed) & bit) || !bit) {
        e = cudaFuncSetAttribute(kernel, cudaFuncAttributeMaxDynamicSharedMemorySize, kSmem);
        if (e != cudaSuccess) return e;
        opted.fetch_or(bit, std::memory_order_relaxed);
    }
    cudaLaunchConfig_t cfg = {};
    cfg.gridDim = dim3((unsigned)(pass.tiles * pass.parts * (PREFIX ? 1 : p.batch) * CG), (unsigned)p.c.heads);
    cfg.blockDim = dim3(kTileThreads);
    cfg.dynamicSmemBytes = kSmem;
    cfg.stream = s;
    cudaLaunchAttribute attr[2];
    attr[0].id = cudaLaunchAttributeProgrammaticStreamSerialization;
    attr[0].val.programmaticStreamSerializationAllowed = 1;
    attr[1].id = cudaLaunchAttributeClusterDimension;
    attr[1].val.clusterDim.x = CG;
    attr[1].val.clusterDim.y = attr[1].val.clusterDim.z = 1;
    cfg.attrs = attr;
    cfg.numAttrs = CG;
    return cudaLaunchKernelEx(&cfg, kernel, p, pass, part0);
}

template <int D, int CG>
cudaError_t dispatch(const Attention& p, const Pass& pass, bool prefix, int64_t part0, cudaStream_t s) {
    if (prefix) return launch<D, true, true, CG>(p, pass, part0, s);
    return p.plan.through ? launch<D, false, true, CG>(p, pass, part0, s) : launch<D, false, false, CG>(p, pass, part0, s);
}

}  // namespace

cudaError_t launch_tiles(const Attention& p, const Pass& pass, bool prefix, int64_t part0, cudaStream_t s) {
    if (p.c.dim == 64) return dispatch<64, 1>(p, pass, prefix, part0, s);
    return pass.rows == kPairRows ? dispatch<128, 2>(p, pass, prefix, part0, s) : dispatch<128, 1>(p, pass, prefix, part0, s);
}

}  // namespace kv
}  // namespace nvfp4

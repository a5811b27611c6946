// Products of few tokens on the tensor cores (tcgen05.mma.kind::mxf4nvf4, block scales
// applied by the MMA), bound by reading the weight once:
//
//   out[t][n] = epilogue( sum_k q[t][k] p[n][k] ),   p: weights, q: at most TN tokens.
//
// The weight's rows are the MMA's M side, so that one token costs an MMA of N = 16.  Lane
// i of tensor memory is then column n0 + i of the result and a warp's stores are consecutive.
// The gated form keeps two accumulators, gate and up.
//   * one warp loads stages (128 bytes of each operand's rows along K, and their scale
//     atoms) by TMA into a ring; out-of-range rows, columns and atoms arrive as zeros;
//   * one warp copies each stage's scale atoms to tensor memory (tcgen05.cp) and issues its
//     MMAs; copies and MMAs run in the order they are issued;
//   * four warps read the accumulators and write the result.
// Two CTAs to an SM, and a cluster of up to eight splits K so that their loads fill the SMs.  Each
// rank sends its sums for a token to the rank that finishes that token, which adds
// them in rank order: one cluster barrier after the sends, none after the reads.
//
// Every mbarrier wait is bounded (1 s); on a timeout the CTA sets bit 16 of the status
// word, drains its copies, frees its tensor memory and returns; its results are not there.
#include "fp4_tile.cuh"

namespace nvfp4 {
namespace mm {
namespace {

constexpr int kThreadsTile = 192;                            // 4 epilogue warps, loads, MMAs
constexpr int kMaxStages = 8;
constexpr int kTileSmem = 112 * 1024;                        // of a CTA, two to an SM

struct TileParams {
    CUtensorMap p, p2, q, sp, sp2, sq;
    int64_t k;
    int stages, log_split, starve;
    Epilogue e;
};

template <int KIND, int MODE, int TN>
struct Tile {
    static constexpr int kG = MODE == kPlain ? 1 : 2;        // accumulators
    static constexpr int kP = 128 * kRow, kQ = TN * kRow, kS = atoms(KIND) * kAtom;
    static constexpr int kStage = kG * kP + kQ + (kG + 1) * kS;
    static constexpr int kRed = kG * TN * 128 * 4;           // sums of all ranks for this rank's tokens
    // More than 16 KB of them would cost the second CTA of an SM: they take the ring's place,
    // once a further cluster barrier says that every rank is done with its own.
    static constexpr bool kOver = kRed > 16 * 1024;
    // tensor memory: accumulators, then the scales of p, p2, q (4 columns an atom)
    static constexpr int kSfCol = kG * TN, kSfW = atoms(KIND) * 4;
    static constexpr int kCols = kSfCol + (kG + 1) * kSfW;
    static constexpr int kTmem = kCols <= 32 ? 32 : kCols <= 64 ? 64 : kCols <= 128 ? 128 : 256;
    static constexpr int kOwn = kOver ? 0 : kRed;
    // stages of a CTA that has half an SM, or a whole one
    static constexpr int kHalf = (kTileSmem - 1024 - 256 - kOwn) / kStage;
    static constexpr int kWhole = (2 * kTileSmem - 1024 - 256 - kOwn) / kStage > kMaxStages ? kMaxStages
                                                                                          : (2 * kTileSmem - 1024 - 256 - kOwn) / kStage;
    static constexpr int smem(int stages) { return stages * kStage + kOwn + 1024; }
    static_assert(kHalf >= 2 && (!kOver || kRed <= kHalf * kStage), "shared memory");
};

// Column n of tokens t.. below T, K of them at most.  Whole warps call it (the MXFP4 form reduces
// over the 32 columns of a warp, one block).  All values first, then all stores: with the branches
// on what is wanted inside a token's work, tokens ran one after the other (240 cycles each).
template <int MODE, int K>
__device__ __forceinline__ void emit(const Epilogue& e, int t, int T, int64_t n, const float (&a)[K], const float (&b)[K],
                                     float sp, float sp2, float sq, bool& bad) {
    if constexpr (MODE == kPlain) {
        if (n >= e.N) return;
        if (e.out_f32) {
            float* at = static_cast<float*>(e.out) + t * e.ldo + n;
#pragma unroll
            for (int i = 0; i < K; i++)
                if (t + i < T) at[i * e.ldo] = a[i] * sp * sq;
        } else {
            uint16_t* at = static_cast<uint16_t*>(e.out) + t * e.ldo + n;
#pragma unroll
            for (int i = 0; i < K; i++)
                if (t + i < T) at[i * e.ldo] = bf16_bits(a[i] * sp * sq);
        }
    } else {
        uint16_t h[K];
        float g[K], unused;
#pragma unroll
        for (int i = 0; i < K; i++) g[i] = a[i] * sp * sq;
        if (e.act == 1) {
#pragma unroll
            for (int i = 0; i < K; i++) g[i] = activate<false>(1, g[i], unused);
        } else {
#pragma unroll
            for (int i = 0; i < K; i++) g[i] = activate<false>(0, g[i], unused);
        }
#pragma unroll
        for (int i = 0; i < K; i++) h[i] = bf16_bits(g[i] * (b[i] * sp2 * sq));
        if (e.out && n < e.N) {
            uint16_t* at = static_cast<uint16_t*>(e.out) + t * e.ldo + n;
#pragma unroll
            for (int i = 0; i < K; i++)
                if (t + i < T) at[i * e.ldo] = h[i];
        }
        if (e.h_codes) {
            const int lane = threadIdx.x & 31;
            const bool live = n < e.N;                           // N % 32 == 0: the same for a warp
#pragma unroll
            for (int i = 0; i < K; i++) {
                const uint32_t m = __reduce_max_sync(0xFFFFFFFFu, live ? (uint32_t)(h[i] & 0x7FFF) << 16 : 0u), ex = m >> 23;
                const bool finite = ex != 255;
                const uint32_t code = finite && ex > 2 ? ex - 2 : 0;
                const float hv = bf16_value(h[i]);
                const float x = finite ? hv * __uint_as_float((254u - code) << 23) : copysignf(0.0f, hv);
                uint32_t w = (e2m1x8(pack2(x, 0.0f), 0, 0, 0) & 0xFu) << (4 * (lane & 7));
                w |= __shfl_xor_sync(0xFFFFFFFFu, w, 1);
                w |= __shfl_xor_sync(0xFFFFFFFFu, w, 2);
                w |= __shfl_xor_sync(0xFFFFFFFFu, w, 4);
                const int64_t r = t + i;
                if (r >= T) continue;
                bad |= !finite;
                if (live && (lane & 7) == 0) *reinterpret_cast<uint32_t*>(e.h_codes + r * (e.N / 2) + n / 2) = w;
                if (lane == 0) e.h_sf[swizzle_offset(r, n >> 5, e.h_kpad4)] = (uint8_t)code;   // columns past N: zero
            }
        }
    }
}

template <int KIND, int MODE, int TN>
__global__ void __launch_bounds__(kThreadsTile, 2) tile_kernel(const __grid_constant__ TileParams P) {
    using C = Tile<KIND, MODE, TN>;
    extern __shared__ uint8_t smem_raw[];
    __shared__ __align__(8) uint64_t bars[2 * kMaxStages + 1];
    __shared__ int s_abort;
    __shared__ uint32_t s_tmem;
    uint8_t* base = reinterpret_cast<uint8_t*>((reinterpret_cast<uintptr_t>(smem_raw) + 1023) & ~uintptr_t(1023));
    const int tid = threadIdx.x, warp = warp_index(), lane = tid & 31;
    const int lsplit = P.log_split, split = 1 << lsplit, rank = (int)blockIdx.x;   // the cluster is grid dimension x
    const int stages = P.stages;
    const int n0 = (int)blockIdx.y * 128;
    const int nst = (int)((P.k + stage_k(KIND) - 1) / stage_k(KIND));
    const int from = (int)((int64_t)nst * rank / split), to = (int)((int64_t)nst * (rank + 1) / split);
    const uint32_t full0 = smem_u32(bars), empty0 = full0 + 8 * kMaxStages, dbar = empty0 + 8 * kMaxStages;

    if (warp == 5) tmem_alloc(smem_u32(&s_tmem), C::kTmem);
    if (tid == 0) {
        for (int b = 0; b < stages; b++) {
            mbar_init(full0 + 8 * b, 1 + P.starve);
            mbar_init(empty0 + 8 * b, 1);
        }
        mbar_init(dbar, 1);
        s_abort = 0;
        asm volatile("fence.mbarrier_init.release.cluster;" ::: "memory");
    }
    tc_fence_before();
    __syncthreads();
    tc_fence_after();
    if (split > 1 && !C::kOver) asm volatile("barrier.cluster.arrive.relaxed.aligned;" ::: "memory");   // may be sent to
    grid_launch_dependents();                                // tensor memory is this CTA's by now
    grid_dependency_wait();
    const uint32_t tmem = s_tmem;

    if (warp == 4) {
        Ring ring(smem_u32(base));
        bool ok = true;
        int issued = 0;
        for (int s = from; s < to; s++) {
            const int r = ring.slot;
            if (issued >= stages && !mbar_wait_warp(empty0 + 8 * r, ring.parity ^ 1)) {
                ok = false;
                break;
            }
            if (elect_one()) {
                const uint32_t bar = full0 + 8 * r, st = ring.at, sf = st + C::kG * C::kP + C::kQ;
                mbar_expect_tx(bar, C::kStage);
                tma_load_2d(st, &P.p, s * 128, n0, bar);
                if (C::kG == 2) tma_load_2d(st + C::kP, &P.p2, s * 128, n0, bar);
                tma_load_2d(st + C::kG * C::kP, &P.q, s * 128, 0, bar);
                tma_load_3d(sf, &P.sp, 0, s * atoms(KIND), n0 >> 7, bar);
                if (C::kG == 2) tma_load_3d(sf + C::kS, &P.sp2, 0, s * atoms(KIND), n0 >> 7, bar);
                tma_load_3d(sf + C::kG * C::kS, &P.sq, 0, s * atoms(KIND), 0, bar);
            }
            __syncwarp();
            if (issued < stages) issued++;
            ring.next(stages, C::kStage);
        }
        // every slot in use landed
        if (issued < stages) ring = Ring(ring.first, 1);          // each used once
        for (int j = 0; j < issued; j++, ring.next(stages, C::kStage))
            if (!mbar_wait_warp(full0 + 8 * ring.slot, ring.parity ^ 1)) {
                ok = false;
                break;
            }
        if (!ok && lane == 0) atomicOr(&s_abort, 1);
    } else if (warp == 5) {
        constexpr uint32_t id = idesc(KIND, 128, TN);
        Ring ring(smem_u32(base));
        bool ok = true;
        for (int s = from; s < to; s++) {
            const int r = ring.slot;
            if (!mbar_wait_warp(full0 + 8 * r, ring.parity)) {
                ok = false;
                break;
            }
            tc_fence_after();
            if (elect_one()) {
                const uint32_t st = ring.at, sf = st + C::kG * C::kP + C::kQ;
#pragma unroll
                for (int a = 0; a < (C::kG + 1) * atoms(KIND); a++) cp_atom<1>(tmem + C::kSfCol + 4 * a, atom_desc(sf + a * kAtom));
                const int left = (int)((P.k - (int64_t)s * stage_k(KIND) + mma_k(KIND) - 1) / mma_k(KIND));
#pragma unroll
                for (int kk = 0; kk < 4; kk++) {
                    if (kk >= left) break;                   // K ends inside the stage
                    const uint64_t qd = smem_desc(st + C::kG * C::kP + kk * 32, 16, 1024);
                    const uint32_t w = KIND == kMxfp4 ? id | sf_id(2 * (kk & 1)) : id;
                    const uint32_t col = tmem + C::kSfCol + 4 * (KIND == kNvfp4 ? kk : kk >> 1);
#pragma unroll
                    for (int g = 0; g < C::kG; g++)
                        mma<KIND, 1>(tmem + g * TN, smem_desc(st + g * C::kP + kk * 32, 16, 1024), qd, w,
                                     (uint32_t)((s - from) | kk), col + g * C::kSfW, col + C::kG * C::kSfW);
                }
                mma_commit(empty0 + 8 * r);
                if (s == to - 1) mma_commit(dbar);
            }
            __syncwarp();
            ring.next(stages, C::kStage);
        }
        if (!ok && lane == 0) atomicOr(&s_abort, 1);
    } else if (!mbar_wait_warp(dbar, 0)) {
        if (lane == 0) atomicOr(&s_abort, 1);
    }
    tc_fence_after();
    __syncthreads();
    const Epilogue& e = P.e;
    bool ok = s_abort == 0;
    const int T = (int)e.T, lper = (TN == 16 ? 4 : TN == 32 ? 5 : 6) - lsplit, per = 1 << lper;   // tokens a rank finishes
    bool bad = false;
    float sp = 1.0f, sp2 = 1.0f, sq = 1.0f;
    const int64_t n = n0 + 32 * warp + lane;
    if (warp < 4) {
        sp = scale_or_1(e.s_p);
        if (C::kG == 2) sp2 = scale_or_1(e.s_p2);
        sq = scale_or_1(e.s_q);
    }
    if (split > 1) {
        if (C::kOver) asm volatile("barrier.cluster.arrive.release.aligned;" ::: "memory");   // done with the ring
        asm volatile("barrier.cluster.wait.acquire.aligned;" ::: "memory");
    }
    const int red_at = C::kOver ? 0 : stages * C::kStage;
    const uint32_t red = smem_u32(base) + red_at;         // [accumulator][token of this rank][rank][128]
    if (warp < 4 && ok) {
        const uint32_t acc = tmem + ((uint32_t)(32 * warp) << 16);
#pragma unroll 1
        for (int c = 0; c < TN && c < T; c += 16) {
            float a[16], b[16];
            tmem_ld16(acc + c, a);
            if (C::kG == 2) tmem_ld16(acc + TN + c, b);
            tmem_wait16(a);
            if (C::kG == 2) tmem_wait16(b);
            if (split > 1) {
#pragma unroll
                for (int i = 0; i < 16; i++) {
                    const int t = c + i;
                    if (t >= T) continue;
                    const uint32_t at = at_rank(red + (uint32_t)((((t & (per - 1)) << lsplit) + rank) * 512 + tid * 4), (uint32_t)(t >> lper));
                    st_cluster(at, a[i]);
                    if (C::kG == 2) st_cluster(at + TN * 512, b[i]);
                }
            } else {
                if (T - c <= 2) {
                    const float a2[2] = {a[0], a[1]}, b2[2] = {b[0], b[1]};
                    emit<MODE, 2>(e, c, T, n, a2, b2, sp, sp2, sq, bad);
                } else {
                    emit<MODE, 16>(e, c, T, n, a, b, sp, sp2, sq, bad);
                }
            }
        }
    }
    if (split > 1) {
        // every rank's sums are here, or the word that one has none
        if (!ok && tid < split) st_cluster(at_rank(smem_u32(&s_abort), tid), 1);
        __syncwarp();
        cluster_barrier();
        ok = *reinterpret_cast<volatile int*>(&s_abort) == 0;
        if (warp < 4 && ok) {
            const float* mine = reinterpret_cast<const float*>(base + red_at) + tid;
            // two tokens at a time: a rank has at least two
#pragma unroll 1
            for (int j = 0; j < per && rank * per + j < T; j += 2) {
                float a[2] = {0.0f, 0.0f}, b[2] = {0.0f, 0.0f};
                for (int r = 0; r < split; r++) {
#pragma unroll
                    for (int i = 0; i < 2; i++) {
                        a[i] += mine[((j + i) * split + r) * 128];
                        if (C::kG == 2) b[i] += mine[(TN + (j + i) * split + r) * 128];
                    }
                }
                emit<MODE, 2>(e, rank * per + j, T, n, a, b, sp, sp2, sq, bad);
            }
        }
    }
    if (MODE == kGated && e.h_codes && warp < 4 && rank == 0)    // scale rows of the tile that hold no token
        for (int r = T + lane; r < 128; r += 32) e.h_sf[swizzle_offset(r, (n0 >> 5) + warp, e.h_kpad4)] = 0;
    if (tid == 0 && !ok && e.status) atomicOr(e.status, kStatusTimeout);
    if (bad && e.status) atomicOr(e.status, 1);
    tc_fence_before();
    __syncthreads();
    if (warp == 5) tmem_dealloc(tmem, C::kTmem);
}

// ---------------------------------------------------------------------------
template <int KIND, int MODE, int TN>
cudaError_t launch_tile(const Product& p, int sms, cudaStream_t s) {
    using C = Tile<KIND, MODE, TN>;
    TileParams P;
    const bool ok = make_operand_map(&P.p, p.p, KIND, p.k, 128) && make_operand_map(&P.q, p.q, KIND, p.k, TN) &&
                    (C::kG == 1 || make_operand_map(&P.p2, p.p2, KIND, p.k, 128)) && make_scale_map(&P.sp, p.p, KIND, p.k) &&
                    make_scale_map(&P.sq, p.q, KIND, p.k) && (C::kG == 1 || make_scale_map(&P.sp2, p.p2, KIND, p.k));
    if (!ok) return cudaErrorNotSupported;
    P.k = p.k;
    P.starve = p.starve;
    P.e = make_epilogue(p);
    const int64_t tn = (p.p.rows + 127) / 128;
    const TilePlan b = tile_plan(p.sizes(), sms);
    P.log_split = b.log_split;
    const int split = 1 << b.log_split;
    P.stages = b.whole ? C::kWhole : C::kHalf;
    const int smem = C::smem(P.stages);
    static std::atomic<bool> attr_set[64];
    int dev = 0;
    cudaError_t e = cudaGetDevice(&dev);
    if (e != cudaSuccess) return e;
    const auto kernel = tile_kernel<KIND, MODE, TN>;
    if (dev < 0 || dev >= 64 || !attr_set[dev].load(std::memory_order_acquire)) {
        e = cudaFuncSetAttribute(kernel, cudaFuncAttributeMaxDynamicSharedMemorySize, C::smem(C::kWhole));
        if (e != cudaSuccess) return e;
        if (dev >= 0 && dev < 64) attr_set[dev].store(true, std::memory_order_release);
    }
    cudaLaunchConfig_t cfg = {};
    cfg.gridDim = dim3((unsigned)split, (unsigned)tn);
    cfg.blockDim = dim3(kThreadsTile);
    cfg.dynamicSmemBytes = (size_t)smem;
    cfg.stream = s;
    cudaLaunchAttribute attr[2];
    attr[0].id = cudaLaunchAttributeProgrammaticStreamSerialization;
    attr[0].val.programmaticStreamSerializationAllowed = 1;
    attr[1].id = cudaLaunchAttributeClusterDimension;
    attr[1].val.clusterDim.x = (unsigned)split;
    attr[1].val.clusterDim.y = 1;
    attr[1].val.clusterDim.z = 1;
    cfg.attrs = attr;
    cfg.numAttrs = 2;
    return cudaLaunchKernelEx(&cfg, kernel, P);
}

template <int KIND, int MODE>
cudaError_t launch_by_tokens(const Product& p, int sms, cudaStream_t s) {
    if (p.q.rows <= 16) return launch_tile<KIND, MODE, 16>(p, sms, s);
    if (p.q.rows <= 32) return launch_tile<KIND, MODE, 32>(p, sms, s);
    return launch_tile<KIND, MODE, 64>(p, sms, s);
}

}  // namespace
}  // namespace mm

cudaError_t launch_product(const Product& p, int sms, cudaStream_t s) {
    if (!mm::few_tokens(p.sizes(), sms)) return launch_pair(p, sms, s);
    if (p.mode == kPlain)
        return p.kind == kMxfp4 ? mm::launch_by_tokens<kMxfp4, kPlain>(p, sms, s) : mm::launch_by_tokens<kNvfp4, kPlain>(p, sms, s);
    return p.kind == kMxfp4 ? mm::launch_by_tokens<kMxfp4, kGated>(p, sms, s) : mm::launch_by_tokens<kNvfp4, kGated>(p, sms, s);
}

}  // namespace nvfp4

// Products on the tensor cores of quantised operands (tcgen05.mma.kind::mxf4nvf4, block
// scales applied by the MMA) and of the bf16 operands of their gradients (kind::f16):
//
//   out[t][n] = epilogue( sum_k q[t][k] p[n][k] ),   p: weights, q: tokens.
//
// tile_kernel: a CTA forms 128 columns n by TN tokens, the weight's rows on the MMA's M
// side whatever the number of tokens, so that one token costs an MMA of N = 16 and the
// weight is read once.  Lane i of tensor memory is then column n0 + i of the result and a
// warp's stores are consecutive.  The gated forms keep two accumulators, gate and up.
//   * one warp loads stages (128 bytes of each operand's rows along K, and their scale
//     atoms) by TMA into a ring; out-of-range rows, columns and atoms arrive as zeros;
//   * one warp copies each stage's scale atoms to tensor memory (tcgen05.cp) and issues its
//     MMAs; copies and MMAs run in the order they are issued;
//   * four warps read the accumulators and write the result.
// Where there are fewer tiles than SMs, a cluster of CTAs splits K; each leaves its sums in
// its shared memory and adds a share of the columns over all of them in rank order.
//
// Every mbarrier wait is bounded (1 s); on a timeout the CTA sets bit 16 of the status
// word, drains its copies, frees its tensor memory and returns without writing.
#include "fp4_tile.cuh"

namespace nvfp4 {
namespace mm {
namespace {

constexpr int kThreadsTile = 192;                            // 4 epilogue warps, loads, MMAs
constexpr int kMaxStages = 8;

struct TileParams {
    CUtensorMap p, p2, q, sp, sp2, sq;
    int64_t k;
    int stages;
    Epilogue e;
};

template <int KIND, int MODE, int TN>
struct Tile {
    static constexpr int kG = MODE == kPlain ? 1 : 2;        // accumulators
    static constexpr int kP = 128 * kRow, kQ = TN * kRow, kS = atoms(KIND) * kAtom;
    static constexpr int kStage = kG * kP + kQ + (kG + 1) * kS;
    // tensor memory: accumulators, then the scales of p, p2, q (4 columns an atom)
    static constexpr int kSfCol = kG * TN, kSfW = atoms(KIND) * 4;
    static constexpr int kCols = kSfCol + (kG + 1) * kSfW;
    static constexpr int kTmem = kCols <= 32 ? 32 : kCols <= 64 ? 64 : kCols <= 128 ? 128 : kCols <= 256 ? 256 : 512;
    static int stages() {
        const int n = (200 * 1024) / kStage;
        return n > kMaxStages ? kMaxStages : n;
    }
    static int smem(int stages) {
        const int ring = stages * kStage, red = kG * TN * 128 * 4;
        return (ring > red ? ring : red) + 1024 + 256;
    }
};

// One result column n of token t.  Whole warps call it (the MXFP4 form reduces over the
// 32 columns of a warp, one block).
template <int MODE>
__device__ __forceinline__ void emit(const Epilogue& e, int64_t t, int64_t n, float a, float b, float sp, float sp2,
                                     float sq, bool& bad) {
    if (MODE == kPlain) {
        if (t < e.T && n < e.N) {
            const float v = a * sp * sq;
            if (e.out_f32)
                static_cast<float*>(e.out)[t * e.ldo + n] = v;
            else
                static_cast<uint16_t*>(e.out)[t * e.ldo + n] = bf16_bits(v);
        }
        return;
    }
    float unused;
    const float g = a * sp * sq, u = b * sp2 * sq;
    const uint16_t h = bf16_bits(activate<false>(e.act, g, unused) * u);
    if (e.out && t < e.T && n < e.N) static_cast<uint16_t*>(e.out)[t * e.ldo + n] = h;
    if (MODE == kGated && e.h_codes) {
        const int lane = threadIdx.x & 31;
        const bool live = t < e.T && n < e.N;                // N % 32 == 0: the same for a warp
        const uint32_t m = __reduce_max_sync(0xFFFFFFFFu, live ? (uint32_t)(h & 0x7FFF) << 16 : 0u), ex = m >> 23;
        const bool finite = ex != 255;
        bad |= !finite;
        const uint32_t code = finite && ex > 2 ? ex - 2 : 0;
        const float hv = bf16_value(h);
        const float x = finite ? hv * __uint_as_float((254u - code) << 23) : copysignf(0.0f, hv);
        uint32_t w = (e2m1x8(pack2(x, 0.0f), 0, 0, 0) & 0xFu) << (4 * (lane & 7));
        w |= __shfl_xor_sync(0xFFFFFFFFu, w, 1);
        w |= __shfl_xor_sync(0xFFFFFFFFu, w, 2);
        w |= __shfl_xor_sync(0xFFFFFFFFu, w, 4);
        if (live && (lane & 7) == 0) *reinterpret_cast<uint32_t*>(e.h_codes + t * (e.N / 2) + n / 2) = w;
        if (lane == 0) e.h_sf[swizzle_offset(t, n >> 5, e.h_kpad4)] = (uint8_t)code;   // padding: zero
    }
}

// Sixteen tokens t0.. of column n: the gradients of the gated form.
__device__ __forceinline__ void emit_grad16(const Epilogue& e, int64_t t0, int64_t n, const float (&a)[16],
                                            const float (&b)[16], float sp, float sp2, float sq) {
    uint32_t dgw[8], duw[8];
#pragma unroll
    for (int i = 0; i < 16; i++) {
        const int64_t t = t0 + i;
        const bool live = t < e.T && n < e.N;
        const float g = a[i] * sp * sq, u = b[i] * sp2 * sq;
        const float dh = live ? bf16_value(e.dh[t * e.lddh + n]) : 0.0f;
        float da;
        const float ag = activate<true>(e.act, g, da);
        const float dg = live ? dh * u * da : 0.0f, du = live ? dh * ag : 0.0f;
        if (e.out && live) static_cast<uint16_t*>(e.out)[t * e.ldo + n] = bf16_bits(ag * u);
        if (e.dgu && t < e.T) {                              // n < fp: fp is a multiple of the tile
            e.dgu[t * 2 * e.fp + n] = live ? bf16_bits(dg * sp) : (uint16_t)0;
            e.dgu[t * 2 * e.fp + e.fp + n] = live ? bf16_bits(du * sp2) : (uint16_t)0;
        }
        const uint32_t bg = bf16_bits(dg), bu = bf16_bits(du);
        dgw[i >> 1] = i & 1 ? dgw[i >> 1] | bg << 16 : bg;
        duw[i >> 1] = i & 1 ? duw[i >> 1] | bu << 16 : bu;
    }
    if (e.dgu_t) {
#pragma unroll
        for (int j = 0; j < 2; j++) {
            if (t0 + 8 * j >= e.ldt) continue;               // ldt is a multiple of 8
            *reinterpret_cast<uint4*>(e.dgu_t + n * e.ldt + t0 + 8 * j) =
                make_uint4(dgw[4 * j], dgw[4 * j + 1], dgw[4 * j + 2], dgw[4 * j + 3]);
            *reinterpret_cast<uint4*>(e.dgu_t + (e.fp + n) * e.ldt + t0 + 8 * j) =
                make_uint4(duw[4 * j], duw[4 * j + 1], duw[4 * j + 2], duw[4 * j + 3]);
        }
    }
}

template <int KIND, int MODE, int TN>
__global__ void __launch_bounds__(kThreadsTile, 1) tile_kernel(const __grid_constant__ TileParams P) {
    using C = Tile<KIND, MODE, TN>;
    extern __shared__ uint8_t smem_raw[];
    __shared__ __align__(8) uint64_t bars[2 * kMaxStages + 1];
    __shared__ int s_abort;
    __shared__ uint32_t s_tmem;
    uint8_t* base = reinterpret_cast<uint8_t*>((reinterpret_cast<uintptr_t>(smem_raw) + 1023) & ~uintptr_t(1023));
    const int tid = threadIdx.x, warp = warp_index(), lane = tid & 31;
    const int split = (int)gridDim.x, rank = (int)blockIdx.x;   // the cluster is grid dimension x
    const int64_t n0 = (int64_t)blockIdx.y * 128, t0 = (int64_t)blockIdx.z * TN;
    const int nst = (int)((P.k + stage_k(KIND) - 1) / stage_k(KIND));
    const int from = (int)((int64_t)nst * rank / split), to = (int)((int64_t)nst * (rank + 1) / split);
    const uint32_t full0 = smem_u32(bars), empty0 = full0 + 8 * kMaxStages, dbar = empty0 + 8 * kMaxStages;

    if (warp == 5) tmem_alloc(smem_u32(&s_tmem), C::kTmem);
    if (tid == 0) {
        for (int b = 0; b < P.stages; b++) {
            mbar_init(full0 + 8 * b, 1);
            mbar_init(empty0 + 8 * b, 1);
        }
        mbar_init(dbar, 1);
        s_abort = 0;
        asm volatile("fence.mbarrier_init.release.cluster;" ::: "memory");
    }
    tc_fence_before();
    __syncthreads();
    tc_fence_after();
    grid_launch_dependents();                                // tensor memory is this CTA's by now
    grid_dependency_wait();
    const uint32_t tmem = s_tmem;

    if (warp == 4) {
        Ring ring;
        bool ok = true;
        int issued = 0;
        for (int s = from; s < to; s++) {
            const int r = ring.slot;
            if (issued >= P.stages && !mbar_wait_warp(empty0 + 8 * r, ring.parity ^ 1)) {
                ok = false;
                break;
            }
            if (elect_one()) {
                const uint32_t bar = full0 + 8 * r, st = smem_u32(base) + r * C::kStage;
                const int kc = s * (KIND == kBf16 ? 64 : 128);   // elements of the map: bf16 or bytes
                mbar_expect_tx(bar, C::kStage);
                tma_load_2d(st, &P.p, kc, (int)n0, bar);
                if (C::kG == 2) tma_load_2d(st + C::kP, &P.p2, kc, (int)n0, bar);
                tma_load_2d(st + C::kG * C::kP, &P.q, kc, (int)t0, bar);
                if (KIND != kBf16) {
                    const uint32_t sf = st + C::kG * C::kP + C::kQ;
                    tma_load_3d(sf, &P.sp, 0, s * atoms(KIND), (int)(n0 >> 7), bar);
                    if (C::kG == 2) tma_load_3d(sf + C::kS, &P.sp2, 0, s * atoms(KIND), (int)(n0 >> 7), bar);
                    tma_load_3d(sf + C::kG * C::kS, &P.sq, 0, s * atoms(KIND), (int)(t0 >> 7), bar);
                }
            }
            __syncwarp();
            if (issued < P.stages) issued++;
            ring.next(P.stages);
        }
        // every slot in use landed
        if (issued < P.stages) ring = Ring{0, 1};            // each used once
        for (int j = 0; j < issued; j++, ring.next(P.stages))
            if (!mbar_wait_warp(full0 + 8 * ring.slot, ring.parity ^ 1)) ok = false;
        if (!ok && lane == 0) atomicOr(&s_abort, 1);
    } else if (warp == 5) {
        constexpr uint32_t id = idesc(KIND, 128, TN);
        Ring ring;
        bool ok = true;
        for (int s = from; s < to; s++) {
            const int r = ring.slot;
            if (!mbar_wait_warp(full0 + 8 * r, ring.parity)) {
                ok = false;
                break;
            }
            tc_fence_after();
            if (elect_one()) {
                const uint32_t st = smem_u32(base) + r * C::kStage, sf = st + C::kG * C::kP + C::kQ;
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
            }
            __syncwarp();
            ring.next(P.stages);
        }
        if (elect_one()) mma_commit(dbar);                   // after every MMA issued, also on a timeout
        __syncwarp();
        if (!ok && lane == 0) atomicOr(&s_abort, 1);
    }
    __syncthreads();
    if (!mbar_wait(dbar, 0)) atomicOr(&s_abort, 1);
    tc_fence_after();
    __syncthreads();
    const bool ok = s_abort == 0;
    bool bad = false;
    if (warp < 4) {
        const Epilogue& e = P.e;
        const float sp = scale_or_1(e.s_p), sp2 = C::kG == 2 ? scale_or_1(e.s_p2) : 1.0f, sq = scale_or_1(e.s_q);
        const int64_t n = n0 + 32 * warp + lane;
        const uint32_t acc = tmem + ((uint32_t)(32 * warp) << 16);
        float* red = reinterpret_cast<float*>(base);
        if (ok)
#pragma unroll 1
            for (int c = 0; c < TN; c += 16) {
                float a[16], b[16];
                tmem_ld16(acc + c, a);
                if (C::kG == 2) tmem_ld16(acc + TN + c, b);
                tmem_wait16(a);
                if (C::kG == 2) tmem_wait16(b);
                if (split > 1) {
#pragma unroll
                    for (int i = 0; i < 16; i++) {
                        red[(c + i) * 128 + tid] = a[i];
                        if (C::kG == 2) red[(TN + c + i) * 128 + tid] = b[i];
                    }
                } else if (MODE == kGatedGrad) {
                    emit_grad16(e, t0 + c, n, a, b, sp, sp2, sq);
                } else {
#pragma unroll
                    for (int i = 0; i < 16; i++) emit<MODE>(e, t0 + c + i, n, a[i], C::kG == 2 ? b[i] : 0.0f, sp, sp2, sq, bad);
                }
            }
    }
    if (split > 1) {
        cluster_barrier();                                   // every rank's sums are in its shared memory
        if (warp < 4 && ok) {
            const Epilogue& e = P.e;
            const float sp = scale_or_1(e.s_p), sp2 = C::kG == 2 ? scale_or_1(e.s_p2) : 1.0f, sq = scale_or_1(e.s_q);
            const int64_t n = n0 + 32 * warp + lane;
            const uint32_t mine = smem_u32(base) + 4 * tid;
#pragma unroll 2
            for (int c = TN * rank / split; c < TN * (rank + 1) / split; c++) {
                float a = 0.0f, b = 0.0f;
                for (int r = 0; r < split; r++) {
                    const uint32_t from_r = at_rank(mine + c * 512, r);
                    a += ld_cluster(from_r);
                    if (C::kG == 2) b += ld_cluster(from_r + TN * 512);
                }
                emit<MODE>(e, t0 + c, n, a, b, sp, sp2, sq, bad);
            }
        }
        cluster_barrier();                                   // read before any rank's shared memory goes
    }
    if (MODE == kGated && TN < 128 && P.e.h_codes && warp < 4 && rank == 0)    // scale rows of the tile that hold no token
        for (int r = TN + lane; r < 128; r += 32) P.e.h_sf[swizzle_offset(t0 + r, (n0 >> 5) + warp, P.e.h_kpad4)] = 0;
    if (tid == 0 && !ok && P.e.status) atomicOr(P.e.status, kStatusTimeout);
    if (bad && P.e.status) atomicOr(P.e.status, 1);
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
                    (C::kG == 1 || make_operand_map(&P.p2, p.p2, KIND, p.k, 128)) &&
                    (KIND == kBf16 || (make_scale_map(&P.sp, p.p, KIND, p.k) && make_scale_map(&P.sq, p.q, KIND, p.k) &&
                                       (C::kG == 1 || make_scale_map(&P.sp2, p.p2, KIND, p.k))));
    if (!ok) return cudaErrorNotSupported;
    P.k = p.k;
    P.e = make_epilogue(p);
    const int nst = (int)((p.k + stage_k(KIND) - 1) / stage_k(KIND));
    const int64_t tn = (p.p.rows + 127) / 128, tt = (p.q.rows + TN - 1) / TN;
    int split = 1;
    if (MODE != kGatedGrad)
        while (split < 8 && 2 * split * tn * tt <= sms && 2 * split <= nst && 2 * split <= TN) split *= 2;
    P.stages = C::stages();
    const int smem = C::smem(P.stages);
    static std::atomic<bool> attr_set[64];
    int dev = 0;
    cudaError_t e = cudaGetDevice(&dev);
    if (e != cudaSuccess) return e;
    const auto kernel = tile_kernel<KIND, MODE, TN>;
    if (dev < 0 || dev >= 64 || !attr_set[dev].load(std::memory_order_acquire)) {
        e = cudaFuncSetAttribute(kernel, cudaFuncAttributeMaxDynamicSharedMemorySize, smem);
        if (e != cudaSuccess) return e;
        if (dev >= 0 && dev < 64) attr_set[dev].store(true, std::memory_order_release);
    }
    cudaLaunchConfig_t cfg = {};
    cfg.gridDim = dim3((unsigned)split, (unsigned)tn, (unsigned)tt);
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
    // the fewest tokens to a tile that hold all, else 128: an atom's rows start a tile
    if (p.q.rows <= 16) return launch_tile<KIND, MODE, 16>(p, sms, s);
    if (p.q.rows <= 32) return launch_tile<KIND, MODE, 32>(p, sms, s);
    if (p.q.rows <= 64) return launch_tile<KIND, MODE, 64>(p, sms, s);
    return launch_tile<KIND, MODE, 128>(p, sms, s);
}

template <int KIND>
cudaError_t launch_by_mode(const Product& p, int sms, cudaStream_t s) {
    switch (p.mode) {
        case kPlain: return launch_by_tokens<KIND, kPlain>(p, sms, s);
        case kGated: return launch_by_tokens<KIND, kGated>(p, sms, s);
        default: return launch_tile<KIND, kGatedGrad, 128>(p, sms, s);
    }
}

}  // namespace
}  // namespace mm

cudaError_t launch_product(const Product& p, int sms, cudaStream_t s) {
    if (p.q.rows > 128) return launch_pair(p, sms, s);
    switch (p.kind) {
        case kNvfp4: return mm::launch_by_mode<kNvfp4>(p, sms, s);
        case kMxfp4: return mm::launch_by_mode<kMxfp4>(p, sms, s);
        default: return mm::launch_tile<kBf16, kPlain, 128>(p, sms, s);
    }
}

}  // namespace nvfp4
